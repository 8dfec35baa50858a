"""GELU behind an 8-bit layer, value by value: x Phi(x) to the rounding of the type, in the tail too, on every kernel."""
import math

import numpy as np
import pytest
import torch

import paper_2508_00367_amd as rs
from i8_testlib import DT, U16, U32, f64

pytestmark = pytest.mark.gpu

# Sizes (M, K, N) that reach every kernel, whole 16-byte pieces and others: tests/test_i8_reach_cpu.py has which is which.
KERNELS = [(40, 16, 24), (40, 16, 21), (300, 16, 1024), (788, 16, 768), (900, 16, 1001), (1576, 16, 2304), (1700, 16, 2051), (1576, 1024, 4096),
           (2500, 1100, 3001), (3000, 2048, 4096), (3000, 2050, 4001)]


def gelu64(v):
    """v Phi(v), Phi by erfc on the side where it is small: nothing cancels."""
    return np.array([x * 0.5 * math.erfc(-x * math.sqrt(0.5)) for x in v])


def layer(values, M, K, N, dtype):
    """[M, N] of GELU(values[m]): one product of 1 and +-1 with the scale |value|, exact whatever the order."""
    a = torch.zeros(M, (K + 15) // 16 * 16, dtype=torch.int8, device="cuda")
    v = torch.tensor(np.resize(values, M), dtype=torch.float32)
    a[:, 0] = torch.where(v < 0, -1, 1).to(torch.int8).cuda()
    w = torch.zeros(K, N, dtype=torch.int8, device="cuda")
    w[0] = 1
    packed = torch.empty(rs.rs_packed_linear_i8_size(K, N), dtype=torch.uint8, device="cuda")
    rs.rs_pack_linear_i8(w, packed)
    out = torch.full((M, N), 7.0, dtype=DT[dtype], device="cuda")
    rs.rs_linear_i8_fwd(a[:, :K], v.abs().cuda(), packed, torch.ones(N, device="cuda"), None, None, out, rs.RS_EPI_BIAS_GELU)
    torch.cuda.synchronize()
    return v.double().numpy(), out


def bound(v, ref, dtype):
    """bf16: x Phi(x) = max(x, 0) - |x| 2^q(|x|), q of degree 7.  Its fit to log2 Phi is 8e-6 of Phi off up to 2, 2e-5 to 4, 1.4e-4 to 6, 1.7e-3 to 9;
    its 7 fused steps are 7 roundings of the sum of its terms' magnitudes, 6, 20, 57 and 230 there, times ln 2; the exponential and the product,
    4 more.  Beyond 9 both the value and the form are under 1.1e-18.  One rounding of the sum, one to bf16 (1e-37: what underflows).
    fp32: 0.5 x (1 + erf(x / sqrt(2))), in which 1 + erf cancels for negative x: roundings of magnitude |x|, 8 of them."""
    if dtype == "f32":
        return 8 * U32 * np.abs(v) + U32 * np.abs(ref) + 1e-37
    a = np.abs(v)
    fit, size = (np.select([a <= 2, a <= 4, a <= 6, a <= 9], t, 0.0) for t in ([8e-6, 2e-5, 1.4e-4, 1.7e-3], [6, 20, 57, 230]))
    small = np.array([x * 0.5 * math.erfc(x * math.sqrt(0.5)) for x in a])
    tol = np.where(a <= 9, small * (fit + (5 * size + 4) * U32), 1.1e-18) + U32 * np.abs(ref)
    return tol + U16 * (np.abs(ref) + tol) + 1e-37


VALUES = np.concatenate([np.linspace(-13, 13, 521), [-1e-3, 1e-3, -1e-20, 1e-20, -2.0 ** -126, 0.0, -14.0, -40.0, -1e5, 1e5, -1e30, 1e30]])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", KERNELS)
def test_gelu_of_every_value(M, K, N, dtype):
    for part in range(0, len(VALUES), M):
        v, out = layer(VALUES[part:part + M], M, K, N, dtype)
        ref = gelu64(v)
        got = f64(out)
        assert np.all(got == got[:, :1])
        off = np.abs(got[:, 0] - ref)
        assert np.all(off <= bound(v, ref, dtype)), (v[np.argmax(off / bound(v, ref, dtype))], np.max(off / bound(v, ref, dtype)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gelu_of_infinities_and_nan(dtype):
    """+inf stays, NaN stays; -inf is NaN or 0 (the limit), by the form taken; the other rows are what they were."""
    v, out = layer(np.array([np.inf, np.nan, -np.inf, 1.0]), 4, 16, 40, dtype)
    got = f64(out)
    assert np.all(np.isposinf(got[0])) and np.all(np.isnan(got[1]))
    assert np.all(np.isnan(got[2]) | (got[2] == 0))
    assert np.all(np.abs(got[3] - gelu64([1.0])) <= bound(np.array([1.0]), gelu64([1.0]), dtype))
