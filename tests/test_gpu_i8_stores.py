"""Rows of the output that are whole 16-byte pieces and no whole lines, in the kernels with large tiles: another store than those of
whole lines and of rows that start anywhere."""
import sys

import pytest
import torch

import paper_2508_00367_amd as rs
from test_gpu_linear_i8 import EPI, check, make, packed, run_linear

pytestmark = pytest.mark.gpu

# (M, K, N) for the private kernel and the direct ones of 64, 128 and 256 rows, N * size a multiple of 16 bytes and not of 128 in both
# types: tests/test_i8_reach_cpu.py
PIECES = [(900, 200, 1008), (1700, 1300, 2056), (2500, 1100, 3000), (3000, 2048, 4008)]


def _say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("epi", ["bias", "gelu", "res"])
@pytest.mark.parametrize("M,K,N", PIECES)
def test_rows_of_pieces(M, K, N, epi, dtype):
    """The outer rows and columns and a sample of the others, where the ends of tiles, waves and lines are."""
    _say("rows of pieces", M, K, N, epi, dtype)
    a, a_s, w, w_s, bias, res = make(M, K, N, dtype, epi, seed=M + N)
    out = run_linear(a, a_s, w, w_s, bias, res, dtype, epi)
    rows = sorted(set(range(70)) | set(range(M - 140, M)) | set(range(0, M, 37)))
    check(out[rows], a[rows], a_s[rows], w, w_s, bias, None if res is None else res[rows], dtype, epi)
    cols = sorted(set(range(70)) | set(range(N - 70, N)))
    check(out[:, cols], a, a_s, w[:, cols], w_s[cols], bias[cols], None if res is None else res[:, cols], dtype, epi)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", PIECES + [(40, 300, 200), (788, 768, 768), (900, 200, 1001), (2500, 1100, 3001)])
def test_out_is_res(M, K, N, dtype):
    """In place the same bits as beside it: no wave needs residual rows that another has overwritten."""
    a, a_s, w, w_s, bias, res = make(M, K, N, dtype, "res", seed=M)
    want = run_linear(a, a_s, w, w_s, bias, res, dtype, "res")
    pw = packed(w)
    for _ in range(3):
        inout = res.clone()
        rs.rs_linear_i8_fwd(a, a_s, pw, w_s, bias, inout, inout, EPI["res"])
        assert torch.equal(inout, want)
