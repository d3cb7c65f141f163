// Routed operators (router, experts' products, 4-bit weights): what their sources share.
#pragma once
#include <atomic>
#include <cstdint>

#include "../../include/tilefusion.h"

namespace tf {

// Row counts go up to 2^31 - 1: sums of them are 64 bits wide, differences need no more than 32.
constexpr int64_t ceil_div(int64_t n, int64_t per) { return (n + per - 1) / per; }
// The most workgroups of a launch, whose threads must be fewer than 2^32.
constexpr int64_t most_workgroups(int64_t threads) { return (((int64_t)1 << 32) - 1) / threads; }
constexpr bool last_pass(int32_t first, int32_t total, int32_t most) { return total - first <= most; }

// The devices for which something that lasts has been done; any thread may ask.  (Beyond the 64th it is done each time.)
class DoneOnDevices {
    std::atomic<uint64_t> done_{0};

  public:
    bool has(int device) const { return device >= 0 && device < 64 && (done_.load(std::memory_order_acquire) >> device & 1); }
    void add(int device) {
        if (device >= 0 && device < 64) done_.fetch_or((uint64_t)1 << device, std::memory_order_release);
    }
};

// ---------------------------------------------------------------------------------- 4-bit layout
//
// A matrix is cut into blocks of 16 rows x 128 columns, 1 KiB each, block row after block row: what one wave
// loads with one instruction, sixteen bytes a lane.  Lane 16 g + r holds in word j the eight columns
// 128 kb + 32 j + 8 g + {0 .. 7} of row r: an operand of the j-th 16 x 16 x 32 matrix instruction.  Scales are in blocks of
// the same rows and columns, row after row, group after group.  Columns beyond the matrix have code 0 and scale 0, rows beyond
// it likewise.
constexpr int kQ4Block = 128;
inline int64_t q4_tiles(int64_t rows) { return (rows + 15) / 16; }
inline int64_t q4_blocks(int64_t cols) { return (cols + kQ4Block - 1) / kQ4Block; }
inline int64_t q4_code_bytes(int64_t rows, int64_t cols) { return q4_tiles(rows) * q4_blocks(cols) * 1024; }
inline int64_t q4_scale_bytes(int64_t rows, int64_t cols, int group) {
    return q4_tiles(rows) * q4_blocks(cols) * 16 * (kQ4Block / group) * 2;
}

struct Q4Launch {
    int64_t n_mats, n_rows, n_cols;
    int32_t kind, group;
    void *codes, *scales;
    const int8_t *src_codes;      // pack
    const void *src_scales;
    void *weights;                // quantize: read, unpack: written
    int32_t dtype;
    int32_t *bad;                 // pack: set where a code is out of range
};
int launch_q4_pack(const Q4Launch &a, void *stream);
int launch_q4_quantize(const Q4Launch &a, void *stream);
int launch_q4_unpack(const Q4Launch &a, void *stream);

// ----------------------------------------------------------------------------------------- router

constexpr int kRouteMaxExperts = 1024, kRouteMaxK = 64;
struct RouteLaunch {
    const void *scores;
    int64_t ld;
    const float *bias;
    int32_t *rowptr, *colidx;
    float *vals;
    int32_t n_tokens, n_experts, k, dtype, scoring;
    float scale;
    int32_t first;                // token that a launch begins with
};
int launch_route(const RouteLaunch &a, void *stream);

// ------------------------------------------------------------------------------ experts' products

// What a launch does with the sums of rows of tokens: the activated hidden row of an entry, or rows of Y.  (Those of hidden
// rows are fp32 sums of entries, which the last workgroup adds up to rows of D.)
enum ExpertOut { kOutHidden = 0, kOutRows = 2 };

constexpr int64_t kMaxColumns = (int64_t)1 << 24;     // of weights: sixteen rows of them are below 2^31 bytes apart
struct ExpertLaunch {
    const void *W, *scales;       // dense: row-major; 4 bits: codes and scales as above
    int64_t w_mat, s_mat;         // bytes from one expert's to the next one's
    int32_t n_rows, n_cols;       // of one expert's matrix that a launch computes with (gate not counted)
    int32_t kind, group;          // kind -1: dense
    int32_t dtype;
    int32_t x_hidden;             // 1: X are hidden rows of entries, 0: rows of tokens
    const void *X;
    int64_t ldx;                  // elements
    int64_t x_part;               // bytes from the high parts of hidden rows to the low ones
    const int32_t *rowptr, *colidx;   // rowptr NULL: one matrix, entry q is row q of X
    int32_t n_tokens, n_entries, n_experts;
    int32_t first_token;          // that a launch of the sum over entries begins with
    int32_t out_kind, activation, gated;
    void *out;
    int64_t ldo, out_part;        // elements; bytes
    const float *vals;            // hidden rows: values of the entries, rows of D
    void *D;
    int64_t ldd;
    uint32_t *arrived;            // for each block of columns: workgroups that have stored their sums (all zero between launches)
    int32_t k_waves;              // waves of a workgroup that share the columns of the same rows: 1, 2, 4 or 8
    int32_t pass_entries;         // the most entries that a workgroup multiplies at a time (LDS and k_waves are chosen for them): 4, 16, 32 or 64
};
int launch_experts(const ExpertLaunch &a, void *stream);
int launch_experts_bf16(const ExpertLaunch &a, void *stream);
int launch_experts_f16(const ExpertLaunch &a, void *stream);
int launch_experts_f32(const ExpertLaunch &a, void *stream);

// Elements from one hidden row to the next: rows begin on lines of memory.  (What lies between them is neither written nor read.)
inline int64_t hidden_ld(int64_t n_hidden) { return (n_hidden + kQ4Block - 1) / kQ4Block * kQ4Block; }

// ----------------------------------------------------------------------------------------- errors
// (tf_api.cpp) Sets what tf_last_error returns.
tf_status report(tf_status st, const char *msg);
tf_status report_hip(int hip_error, const char *what);

}  // namespace tf
