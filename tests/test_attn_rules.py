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
