"""Arithmetic of the routed operators' host code, at sizes that no test would allocate: small C++ programs over their header."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2407_00243_amd", "csrc")


def run_cpp(tmp_path, body):
    """Compiles and runs `body` as main(); CHECK(x) ends it with the line number."""
    src, exe = str(tmp_path / "main.cpp"), str(tmp_path / "main")
    with open(src, "w") as f:
        f.write('#include <cstdio>\n#include <initializer_list>\n#include "tf_moe.h"\nusing namespace tf;\n'
                "#define CHECK(x) do { if (!(x)) { std::printf(\"line %d: %s\\n\", __LINE__, #x); return 1; } } while (0)\n"
                "int main() {\n" + body + "\nreturn 0;\n}\n")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", CSRC, src,
                    "-o", exe], check=True)
    res = subprocess.run([exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout + res.stderr


def test_passes_over_rows_up_to_the_last_count(tmp_path):
    """Passes over the rows of a product cover them once, whatever their count; blocks of a launch likewise."""
    run_cpp(tmp_path, """
    for (int64_t total : {(int64_t)1, (int64_t)4, (int64_t)5, (int64_t)0x7fffffff - 64, (int64_t)0x7fffffff - 1, (int64_t)0x7fffffff})
        for (int32_t most : {4, 16, 32, 64}) {
            CHECK(ceil_div(total, most) * most >= total && (ceil_div(total, most) - 1) * most < total);
            int64_t passes = 0, rows = 0;
            for (int32_t first = 0;; first += most) {
                ++passes;
                rows += total - first < most ? total - first : most;
                if (last_pass(first, (int32_t)total, most)) break;
            }
            CHECK(passes == ceil_div(total, most) && rows == total);
        }""")


def test_launches_stay_below_32_bits_of_threads(tmp_path):
    run_cpp(tmp_path, """
    for (int64_t threads : {256, 512}) {
        CHECK(most_workgroups(threads) * threads < (int64_t)1 << 32);
        CHECK((most_workgroups(threads) + 1) * threads >= (int64_t)1 << 32);
    }""")


def test_what_is_done_once_for_each_device(tmp_path):
    run_cpp(tmp_path, """
    DoneOnDevices done;
    for (int d : {0, 5, 63}) {
        CHECK(!done.has(d));
        CHECK(!done.has(d));            // (asking, as before a call that then fails, changes nothing)
        done.add(d);
        CHECK(done.has(d) && !done.has(d - 1) && !done.has(d + 1));
    }
    for (int d : {-1, 64, 1000}) {
        done.add(d);
        CHECK(!done.has(d));
    }
    CHECK(done.has(0) && done.has(5) && done.has(63) && !done.has(1));""")
