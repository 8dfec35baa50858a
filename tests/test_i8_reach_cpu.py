"""Which kernels the GPU tests of single properties of 8-bit linear layers reach: the choice by shape is host code."""
from test_i8_choice_cpu import choose  # noqa: F401

SPLIT1, SPLIT2, PRIVATE, D64, D128, D256 = "split32x32", "split32x64", "private", "direct64", "direct128", "direct256"


def test_the_gelu_tests_reach_every_kernel(choose):  # noqa: F811
    from test_gpu_i8_gelu import KERNELS
    assert choose(KERNELS) == [SPLIT1, SPLIT1, SPLIT2, PRIVATE, PRIVATE, D64, D64, D128, D128, D256, D256]


def test_the_store_tests_reach_the_tiles(choose):  # noqa: F811
    from test_gpu_i8_stores import PIECES
    assert choose(PIECES) == [PRIVATE, D64, D128, D256]
    assert all(N * size % 16 == 0 and N * size % 128 for _, _, N in PIECES for size in (2, 4))
