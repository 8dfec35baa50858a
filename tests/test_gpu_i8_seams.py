"""More rows than one launch, or one pass of a grid, takes: what the second one reads and writes, on both sides of the seam."""
import sys

import numpy as np
import pytest
import torch

import paper_2508_00367_amd as rs
from i8_testlib import DT, quantize
from test_gpu_linear_i8 import check, packed
from test_gpu_residual_norm import check8, reference, within

pytestmark = pytest.mark.gpu


def _say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def test_linear_rows_of_a_second_launch():
    """One feature: 2^29 rows a launch (2^22 tiles of 128 x 64).  Scales, residual and outputs of the rows behind them."""
    M, K, N = (1 << 29) + 5, 16, 1
    _say("linear_i8", M, K, N)
    a = torch.randint(-128, 128, (M, K), dtype=torch.int8, device="cuda")
    a_scale = torch.rand(M, device="cuda").mul_(0.02).add_(1e-3)
    res = torch.randn(M, N, device="cuda", dtype=torch.bfloat16)
    w = torch.randint(-128, 128, (K, N), dtype=torch.int8, device="cuda")
    w_scale, bias = torch.rand(N, device="cuda") + 0.01, torch.randn(N, device="cuda").bfloat16()
    buf = torch.full((M + 16, N), -777.0, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    rs.rs_linear_i8_fwd(a, a_scale, packed(w), w_scale, bias, res, buf[8:M + 8], rs.RS_EPI_BIAS_RES)
    torch.cuda.synchronize()
    assert bool((buf[:8] == -777).all()) and bool((buf[M + 8:] == -777).all())
    for lo, hi in ((0, 300), ((1 << 28) - 200, (1 << 28) + 200), ((1 << 29) - 300, M)):
        check(buf[8 + lo:8 + hi], a[lo:hi], a_scale[lo:hi], w, w_scale, bias, res[lo:hi], "bf16", "res")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantized_rows_of_a_second_launch(dtype):
    """Four rows a workgroup, 2^23 workgroups a launch."""
    M, K = (1 << 25) + 5, 7
    _say("quantize_rows", M, K, dtype)
    x = torch.randn(M, K, device="cuda", dtype=DT[dtype])
    q, scale = torch.full((M + 1, 16), 55, dtype=torch.int8, device="cuda"), torch.full((M + 1,), -1.0, device="cuda")
    torch.cuda.synchronize()
    rs.rs_quantize_rows(x, q[:M, :K], scale[:M])
    torch.cuda.synchronize()
    assert bool((q[M] == 55).all()) and float(scale[M]) == -1.0 and bool((scale[:M] > 0).all())
    for lo, hi in ((0, 9), ((1 << 24) - 5, (1 << 24) + 5), ((1 << 25) - 9, M)):
        rq, rscale = quantize(x[lo:hi].float().cpu().numpy(), 1)
        assert np.array_equal(q[lo:hi, :K].cpu().numpy(), rq) and np.array_equal(scale[lo:hi].cpu().numpy(), rscale)
        assert bool((q[lo:hi, K:] == 0).all())


def test_norm_rows_of_a_second_pass_one_a_workgroup():
    """2056 channels: a workgroup a row, 2^20 workgroups; the scratch of the sums is used again.  Element 2^31 lies in row 1044495."""
    N, D = 1100000, 2056
    _say("residual_norm", N, D)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    t = lambda *s, std=1.0, mean=0.0: torch.empty(*s, dtype=torch.bfloat16, device="cuda").normal_(mean, std, generator=g)  # noqa: E731
    x, f = t(1, N, D), t(1, N, D)
    v = dict(post_g=t(D, std=0.2, mean=1.0), post_b=t(D, std=0.2), gate=t(D, std=0.5), pre_g=t(D, std=0.2, mean=1.0))
    cfg = rs.make_residual_norm_cfg(1, N, D, torch.bfloat16, rs.RS_NORM_LAYER, rs.RS_NORM_RMS, 1e-6, 1e-5, 1.0, 1.0)
    y, u_q, u_s = torch.empty_like(x), torch.full((N + 1, D + 8), 55, dtype=torch.int8, device="cuda"), torch.empty(N, device="cuda")
    torch.cuda.synchronize()
    rs.rs_residual_norm_fwd(cfg, rs.make_residual_norm_weights(v), x, f, y, None, u_q[:N, :D], u_s)
    torch.cuda.synchronize()
    assert bool((u_q[N] == 55).all())
    for lo, hi in ((0, 4), (1044494, 1044498), ((1 << 20) - 3, (1 << 20) + 5), (N - 4, N)):
        rows = slice(lo, hi)
        ry, ru, ey, eu = reference(x[:, rows], f[:, rows], v, "layer", "rms", False, 1.0, 1.0)
        within(y[:, rows], ry, ey, "bf16")
        check8(u_q[rows], u_s[rows], ru, eu, D)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_rows_of_a_second_pass_many_a_wave(dtype):
    """8 channels: 32 rows a workgroup, every row an image with vectors of its own."""
    B, D = (1 << 25) + 5, 8
    _say("residual_norm", B, D, dtype)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    t = lambda *s, std=1.0, mean=0.0: torch.empty(*s, dtype=DT[dtype], device="cuda").normal_(mean, std, generator=g)  # noqa: E731
    x, f = t(B, 1, D), t(B, 1, D)
    v = dict(gate=t(B, D, std=0.5), mod_scale=t(B, D, std=0.3), mod_shift=t(B, D, std=0.3))
    cfg = rs.make_residual_norm_cfg(B, 1, D, DT[dtype], rs.RS_NORM_RMS, rs.RS_NORM_LAYER, 1e-6, 1e-5, 0.5, 2.0, D, D)
    y, u = (torch.full((B + 1, D), -777.0, dtype=DT[dtype], device="cuda") for _ in range(2))
    torch.cuda.synchronize()
    rs.rs_residual_norm_fwd(cfg, rs.make_residual_norm_weights(v), x, f, y[:B], u[:B])
    torch.cuda.synchronize()
    assert bool((y[B] == -777).all()) and bool((u[B] == -777).all())
    for lo, hi in ((0, 40), ((1 << 24) - 20, (1 << 24) + 20), ((1 << 25) - 40, B)):
        ry, ru, ey, eu = reference(x[lo:hi], f[lo:hi], {k: a[lo:hi] for k, a in v.items()}, "rms", "layer", True, 0.5, 2.0)
        within(y[lo:hi], ry, ey, dtype)
        within(u[lo:hi], ru, eu, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,N", [(5, 1000), (41, 1)])
def test_vectors_of_images_as_far_apart_as_they_may_be(B, N, dtype):
    """2^24 elements from image to image: a wave whose rows are of two images reaches both."""
    D, stride = 64, 1 << 24
    _say("residual_norm", B, N, "stride 2^24", dtype)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    t = lambda *s, std=1.0: torch.empty(*s, dtype=DT[dtype], device="cuda").normal_(0.0, std, generator=g)  # noqa: E731
    far = torch.full((B, stride), float("nan"), dtype=DT[dtype], device="cuda")
    far[:, :3 * D] = t(B, 3 * D, std=0.4)
    x, f, v = t(B, N, D), t(B, N, D), dict(gate=far[:, :D], mod_scale=far[:, D:2 * D], mod_shift=far[:, 2 * D:3 * D])
    cfg = rs.make_residual_norm_cfg(B, N, D, DT[dtype], rs.RS_NORM_RMS, rs.RS_NORM_LAYER, 1e-6, 1e-5, 0.5, 2.0, stride, stride)
    y, u = torch.empty_like(x), torch.empty_like(x)
    rs.rs_residual_norm_fwd(cfg, rs.make_residual_norm_weights(v), x, f, y, u)
    ry, ru, ey, eu = reference(x, f, v, "rms", "layer", True, 0.5, 2.0)
    within(y, ry, ey, dtype)
    within(u, ru, eu, dtype)
