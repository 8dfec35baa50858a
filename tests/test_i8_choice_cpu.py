"""Which kernel an 8-bit linear layer goes to: the rule is host code; the sizes that the GPU tests reach each kernel with, and measured
sizes on both sides of its steps."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ["split32x32", "split32x64", "private", "direct64", "direct128", "direct256"]


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    d = tmp_path_factory.mktemp("i8_choice")
    src = d / "choice.cpp"
    src.write_text("""
#include <cstdio>
#include "gemm_i8_choice.hpp"
int main() {
    long long m, n; int k, cus;
    while (scanf("%lld %lld %d %d", &m, &n, &k, &cus) == 4) printf("%d\\n", (int)rs::gemm_i8_choose(m, n, k, cus));
}
""")
    exe = d / "choice"
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2508_00367_amd", "csrc"), str(src), "-o", str(exe)])

    def ask(sizes, cus=256):
        text = "\n".join("%d %d %d %d" % (M, N, K, cus) for M, K, N in sizes)
        out = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True).stdout
        return [NAMES[int(x)] for x in out.split()]
    return ask


def test_the_sizes_of_the_gpu_tests_reach_every_kernel(choose):
    from test_gpu_linear_i8 import EVERY_KERNEL
    assert choose(EVERY_KERNEL) == ["split32x32", "split32x64", "split32x64", "private", "private", "private", "direct64", "direct64",
                                    "direct128", "direct128", "direct256", "direct256"]
    assert choose([(33, 128, 70), (300, 128, 1100), (1100, 128, 3000), (1100, 1025, 3000)]) == ["split32x32", "split32x64", "direct64", "direct64"]
    assert choose([(300, 1025, 1100)]) == ["private"]


MEASURED = [((1, 768, 2304), "split32x32"), ((64, 768, 2304), "split32x32"), ((197, 4096, 1024), "split32x32"), ((394, 768, 768), "split32x64"),
            ((394, 4096, 1024), "private"), ((394, 1024, 4096), "private"), ((1576, 4096, 1024), "private"), ((2200, 4096, 1024), "direct64"),
            ((2200, 768, 768), "direct64"), ((3152, 4096, 1024), "direct64"), ((2200, 1024, 4096), "direct64"), ((4400, 1024, 4096), "direct64"),
            ((9000, 768, 2304), "direct64"), ((12608, 384, 1536), "direct64"), ((25216, 768, 768), "direct64"), ((9000, 384, 1536), "direct128"),
            ((1576, 1024, 4096), "direct128"), ((3152, 2048, 2048), "direct128"), ((50432, 768, 768), "direct128"), ((50432, 768, 2304), "direct128"),
            ((16388, 1024, 4096), "direct128"), ((12552, 4096, 1024), "direct256"), ((32768, 4096, 4096), "direct256"),
            ((50432, 768, 64), "private"), ((34508, 2048, 128), "private"), ((50432, 192, 64), "direct128"), ((50432, 768, 128), "direct128"),
            ((6000, 4096, 4096), "direct128"), ((16384, 2048, 2048), "direct256"), ((20000, 4096, 1024), "direct128"), ((14000, 4096, 1024), "direct256")]


@pytest.mark.parametrize("size,want", MEASURED)
def test_measured_sizes(choose, size, want):
    assert choose([size]) == [want]


def test_sizes_at_the_ends_have_a_kernel(choose):
    got = choose([(1, 1, 1), (2147483647, 131071, 1048576), (2147483647, 1, 1), (1, 131071, 1048576)])
    assert got[0] == "split32x32" and got[1] in ("direct128", "direct256") and got[2] == "direct128"
