"""Host code that the attention kernels take their decisions with, compiled for the host.  No GPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def run_host(tmp_path, source):
    src, exe = tmp_path / "t.cpp", str(tmp_path / "t")
    src.write_text(source)
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-I",
                    os.path.join(ROOT, "paper_2405_03133_amd", "csrc"), "-o", exe, str(src)], check=True)
    out = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "bad 0", out.stdout[-2000:]


STEP = r"""
#include <stdio.h>
#include "paged_index.h"
using namespace lory::paged;
int main()
{
    long bad = 0;
    for (int keys = 16; keys <= 32; keys += 16) {
        // a step whose first n keys have a page: lane i of 64 owns key i % keys
        for (int n = 0; n <= keys; ++n) {
            uint64_t ballot = 0;
            for (int lane = 0; lane < 64; ++lane)
                if (lane % keys < n) ballot |= (uint64_t)1 << lane;
            const uint32_t valid = valid_keys(ballot, keys);
            bad += (valid == all_keys(keys)) != (n == keys);   // the full step is not masked, any other is
            for (int key = 0; key < keys; ++key) bad += ((valid >> key) & 1) != (key < n);
        }
    }
    printf("bad %ld\n", bad);
    return bad != 0;
}
"""


def test_a_step_with_all_its_keys_is_known_as_one(tmp_path):
    run_host(tmp_path, STEP)


ALONE = r"""
#include <stdio.h>
#include "qk_rope_plan.h"
using lory::rope::alone;
int main()
{
    long bad = 0;
    // tokens and values: one launch is up to a microsecond and more slower from a graph; it is faster, or slower by half of one at most
    const long two[][2] = {{10, 10240}, {8, 10240}, {6, 15360}, {12, 15360}, {7, 17920}, {8, 20480}, {16, 20480}, {17, 136}};
    const long one[][2] = {{1, 512}, {5, 2560}, {1, 2560}, {12, 6144}, {4, 5120}, {2, 5120}, {1, 5120}, {3, 7680}, {16, 8192}};
    for (auto &c : two) bad += alone(c[0], c[1]);
    for (auto &c : one) bad += !alone(c[0], c[1]);
    bad += alone(0, 0) || alone(1l << 25, (1l << 25) * 131070 * 256);
    printf("bad %ld\n", bad);
    return bad != 0;
}
"""


def test_one_workgroup_takes_a_gradient_only_where_replays_stand_it(tmp_path):
    run_host(tmp_path, ALONE)
