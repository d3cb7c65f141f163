// Device helpers of the routed operators.
#pragma once
#include <hip/hip_runtime.h>

#include "tf_moe.h"

namespace tf {
namespace {

typedef float Float4 __attribute__((ext_vector_type(4)));
typedef uint32_t Words4 __attribute__((ext_vector_type(4)));
typedef __bf16 Bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 Half8 __attribute__((ext_vector_type(8)));

// Element types by their tf_dtype.
template <int EL> struct El;
template <> struct El<TF_F32> {
    typedef float T;
    static __device__ __forceinline__ float get(float x) { return x; }
    static __device__ __forceinline__ float put(float x) { return x; }
};
template <> struct El<TF_BF16> {
    typedef uint16_t T;
    static __device__ __forceinline__ float get(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
    static __device__ __forceinline__ uint16_t put(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
};
template <> struct El<TF_F16> {
    typedef uint16_t T;
    static __device__ __forceinline__ float get(uint16_t x) { return (float)__builtin_bit_cast(_Float16, x); }
    static __device__ __forceinline__ uint16_t put(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
};

// Sixteen bytes at any element's address.
typedef uint32_t AnyWords4 __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Place of column i (0 .. 7) of a word: the bit position of its sign and that of its lowest magnitude bit.
// E2M1: nibble i, as the card's conversion takes them.  INT: columns 0 .. 3 are the bytes of the word
// masked with 0x87, columns 4 .. 7 those of the word rotated right by four bits.
__host__ __device__ inline int q4_low_bit(int kind, int i) { return kind == TF_Q4_E2M1 ? 4 * i : i < 4 ? 8 * i : 8 * (i - 4) + 4; }
__host__ __device__ inline int q4_sign_bit(int kind, int i) {
    return kind == TF_Q4_E2M1 ? 4 * i + 3 : i < 4 ? 8 * i + 7 : (8 * (i - 4) + 11) % 32;
}

}  // namespace
}  // namespace tf
