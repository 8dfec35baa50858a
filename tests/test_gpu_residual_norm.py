"""The fused residual add with the norms, gate and modulation around it, against 64 bits."""
import sys

import numpy as np
import pytest
import torch

import paper_2508_00367_amd as rs
from i8_testlib import DT, U16, U32, f64, residual_norm

pytestmark = pytest.mark.gpu

KIND = {"none": rs.RS_NORM_NONE, "layer": rs.RS_NORM_LAYER, "rms": rs.RS_NORM_RMS}
VECTORS = ("post_g", "post_b", "gate", "pre_g", "pre_b", "mod_scale", "mod_shift")


def _say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def make(B, N, D, dtype, per_image, seed, offset=0.0):
    g = torch.Generator().manual_seed(seed)
    t = lambda *s, std=1.0, mean=0.0: (torch.randn(*s, generator=g) * std + mean).to(DT[dtype]).cuda()  # noqa: E731
    x = t(B, N, D, std=2.0, mean=offset)
    f = t(B, N, D, std=0.7, mean=offset)
    v = {n: t(D, std=0.2, mean=1.0 if n.endswith("_g") else 0.0) for n in VECTORS}
    stride = 0
    if per_image:
        stride = 3 * D + 8
        m = t(B, stride, std=0.4)
        v["gate"], v["mod_scale"], v["mod_shift"] = m[:, :D], m[:, D:2 * D], m[:, 2 * D:3 * D]
    return x, f, v, stride


def reference(x, f, v, post, pre, per_image, x_scale, f_scale, eps=(1e-6, 1e-5)):
    D = x.shape[-1]
    h = {n: None if t is None else (f64(t).reshape(-1, 1, D) if n in ("gate", "mod_scale", "mod_shift") else f64(t)) for n, t in v.items()}
    return residual_norm(f64(x), None if f is None else f64(f), post, pre, eps[0], eps[1], x_scale, f_scale, h)


def within(got, ref, err, dtype):
    tol = err * 1.01 + (U16 if dtype == "bf16" else U32) * (np.abs(ref) + err)
    worst = np.max(np.abs(f64(got).reshape(ref.shape) - ref) / np.maximum(tol, 1e-300))
    _say("  worst %.3f of the bound" % worst)
    assert worst <= 1.0


def check8(u_q, u_scale, u, eu, D):
    """The 8-bit rows stand for u: the scale is that of the largest magnitude, an integer is half a step off."""
    u, eu = u.reshape(-1, D), eu.reshape(-1, D)
    s = f64(u_scale)
    top = np.abs(u).max(1)
    assert np.all(np.abs(s - top / 127) <= eu.max(1) / 127 + 3 * U32 * s)
    q = u_q[:, :D].cpu().numpy().astype(np.float64)
    assert np.abs(q).max() <= 127 and np.all(np.abs(q).max(1) == 127)
    # x (1 / scale) is rounded three times before it goes to an integer
    assert np.all(np.abs(q * s[:, None] - u) <= s[:, None] * (0.5 + 3 * U32 * 127) + eu)


SIZES = [(1, 1, 8), (1, 1, 768), (2, 3, 24), (3, 5, 64), (1, 197, 192), (2, 50, 384), (1, 33, 520), (2, 9, 768), (3, 7, 1000), (1, 11, 1024),
         (2, 6, 1536), (1, 5, 2048), (1, 3, 2056), (2, 4, 4096), (1, 3, 5120), (1, 2, 8192), (1, 2, 8200), (1, 3, 16384)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("post,pre,per_image", [("none", "layer", False), ("layer", "layer", True), ("rms", "rms", True), ("layer", "none", False)])
@pytest.mark.parametrize("B,N,D", SIZES)
def test_residual_norm(B, N, D, post, pre, per_image, dtype):
    _say("residual_norm", B, N, D, post, pre, per_image, dtype)
    x, f, v, stride = make(B, N, D, dtype, per_image, seed=B + N + D)
    if post == "none":
        v["post_g"] = v["post_b"] = None
    if post == "rms":
        v["post_b"] = None
    if pre == "none":
        v["pre_g"] = v["pre_b"] = None
    cfg = rs.make_residual_norm_cfg(B, N, D, DT[dtype], KIND[post], KIND[pre], 1e-6, 1e-5, 0.75, 1.5, stride, stride)
    rows = B * N
    y, u = (torch.full((rows + 1, D), -777.0, dtype=DT[dtype], device="cuda") for _ in range(2))
    ldq = (D + 15) // 16 * 16 + 16
    u_q, u_scale = torch.full((rows + 1, ldq), 55, dtype=torch.int8, device="cuda"), torch.full((rows + 1,), -1.0, device="cuda")
    rs.rs_residual_norm_fwd(cfg, rs.make_residual_norm_weights(v), x, f, y[:rows], u[:rows], u_q[:rows, :D], u_scale[:rows])
    torch.cuda.synchronize()
    ry, ru, ey, eu = reference(x, f, v, post, pre, per_image, 0.75, 1.5)
    within(y[:rows], ry, ey, dtype)
    within(u[:rows], ru, eu, dtype)
    check8(u_q[:rows], u_scale[:rows], ru, eu, D)
    assert bool((y[rows:] == -777).all()) and bool((u[rows:] == -777).all()) and float(u_scale[rows]) == -1.0
    pad = (D + 15) // 16 * 16
    assert bool((u_q[rows] == 55).all()) and bool((u_q[:, pad:] == 55).all()) and bool((u_q[:rows, D:pad] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [192, 768, 4096])
def test_every_part_may_be_missing(D, dtype):
    """No branch, no vectors, one output at a time: the same bits as with all of them."""
    B, N = 2, 7
    x, f, v, _ = make(B, N, D, dtype, False, seed=D)
    none = rs.make_residual_norm_weights({})
    cfg = rs.make_residual_norm_cfg(B, N, D, DT[dtype], x_scale=1.0)
    new = lambda: torch.empty(B, N, D, dtype=DT[dtype], device="cuda")  # noqa: E731
    u = new()
    rs.rs_residual_norm_fwd(cfg, none, x, None, None, u)      # a LayerNorm
    _, ru, _, eu = reference(x, None, {}, "none", "layer", False, 1.0, 1.0, eps=(1e-6, 1e-6))
    within(u, ru, eu, dtype)
    y = new()
    rs.rs_residual_norm_fwd(cfg, none, x, f, y, None)         # a residual add
    ry, _, ey, _ = reference(x, f, {}, "none", "layer", False, 1.0, 1.0)
    within(y, ry, ey, dtype)
    w = rs.make_residual_norm_weights(v)
    cfg = rs.make_residual_norm_cfg(B, N, D, DT[dtype], rs.RS_NORM_LAYER, rs.RS_NORM_RMS)
    q = lambda: (torch.empty(B * N, D, dtype=torch.int8, device="cuda"), torch.empty(B * N, device="cuda"))  # noqa: E731
    ya, ua, (qa, sa) = new(), new(), q()
    rs.rs_residual_norm_fwd(cfg, w, x, f, ya, ua, qa, sa)
    yb, ub, (qb, sb) = new(), new(), q()
    rs.rs_residual_norm_fwd(cfg, w, x, f, yb, None)
    rs.rs_residual_norm_fwd(cfg, w, x, f, None, ub)
    rs.rs_residual_norm_fwd(cfg, w, x, f, None, None, qb, sb)
    assert torch.equal(ya, yb) and torch.equal(ua, ub) and torch.equal(qa, qb) and torch.equal(sa, sb)
    xc, fc = x.clone(), f.clone()                             # y in x's place, u in f's
    rs.rs_residual_norm_fwd(cfg, w, xc, fc, xc, fc)
    assert torch.equal(xc, ya) and torch.equal(fc, ua)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("post,pre", [("layer", "layer"), ("rms", "rms")])
def test_rows_far_from_zero_and_rows_of_zeros(post, pre, dtype):
    """A mean of 50 standard deviations, a constant row, rows of zeros, a channel 100 times the others."""
    B, N, D = 1, 6, 768
    x, f, v, _ = make(B, N, D, dtype, False, seed=8, offset=30.0)
    x[0, 1], f[0, 1] = 3.0, 2.0
    x[0, 2], f[0, 2] = 0.0, 0.0
    f[0, 3] = 0.0
    x[0, 4, 5], f[0, 4, 7] = 300.0, -90.0
    v["post_b"] = None if post == "rms" else v["post_b"]
    cfg = rs.make_residual_norm_cfg(B, N, D, DT[dtype], KIND[post], KIND[pre], 1e-6, 1e-5, 1.0, 1.0)
    y, u = torch.empty_like(x), torch.empty_like(x)
    rs.rs_residual_norm_fwd(cfg, rs.make_residual_norm_weights(v), x, f, y, u)
    ry, ru, ey, eu = reference(x, f, v, post, pre, False, 1.0, 1.0)
    within(y, ry, ey, dtype)
    within(u, ru, eu, dtype)


def test_infinities_and_nan_stay_in_their_rows():
    B, N, D = 1, 9, 320
    x, f, v, _ = make(B, N, D, "bf16", False, seed=4)
    x[0, 2, 3], x[0, 4, 319], f[0, 6, 0] = float("nan"), float("inf"), float("-inf")
    cfg = rs.make_residual_norm_cfg(B, N, D, torch.bfloat16, rs.RS_NORM_LAYER, rs.RS_NORM_LAYER)
    y, u = torch.empty_like(x), torch.empty_like(x)
    u_q, u_s = torch.empty(N, D, dtype=torch.int8, device="cuda"), torch.empty(N, device="cuda")
    rs.rs_residual_norm_fwd(cfg, rs.make_residual_norm_weights(v), x, f, y, u, u_q, u_s)
    bad = torch.isnan(u[0]).any(1).cpu().tolist()
    assert bad == [i in (2, 4, 6) for i in range(N)]
    assert torch.isnan(u_s).cpu().tolist() == bad and bool((u_q[[2, 4, 6]] == 0).all())


def test_many_rows():
    """More rows than one pass of the grid; every image its own vectors; a tail row."""
    B, N, D = 5, 9973, 64
    x, f, v, stride = make(B, N, D, "bf16", True, seed=77)
    cfg = rs.make_residual_norm_cfg(B, N, D, torch.bfloat16, rs.RS_NORM_RMS, rs.RS_NORM_LAYER, 1e-6, 1e-5, 1.0, 1.0, stride, stride)
    v["post_b"] = None
    y, u = torch.empty_like(x), torch.empty_like(x)
    rs.rs_residual_norm_fwd(cfg, rs.make_residual_norm_weights(v), x, f, y, u)
    ry, ru, ey, eu = reference(x, f, v, "rms", "layer", True, 1.0, 1.0)
    within(y, ry, ey, "bf16")
    within(u, ru, eu, "bf16")


def test_captured_and_replayed():
    B, N, D = 2, 40, 768
    x, f, v, _ = make(B, N, D, "bf16", False, seed=1)
    cfg = rs.make_residual_norm_cfg(B, N, D, torch.bfloat16, rs.RS_NORM_LAYER, rs.RS_NORM_RMS)
    w = rs.make_residual_norm_weights(v)
    y, u = torch.empty_like(x), torch.empty_like(x)
    rs.rs_residual_norm_fwd(cfg, w, x, f, y, u)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rs.rs_residual_norm_fwd(cfg, w, x, f, y, u)
    for i in range(4):
        x.copy_(torch.randn(B, N, D, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        gy, gu = y.clone(), u.clone()
        ey, eu = torch.empty_like(x), torch.empty_like(x)
        rs.rs_residual_norm_fwd(cfg, w, x, f, ey, eu)
        torch.cuda.synchronize()
        assert torch.equal(gy, ey) and torch.equal(gu, eu), i


def test_offsets_past_32_bits():
    """2.25e9 elements a tensor, 8-bit rows far apart; the rows on both sides of element 2^31 and the last ones."""
    N, D = 1100000, 2048
    x = torch.empty(1, N, D, dtype=torch.bfloat16, device="cuda").normal_()
    f = torch.empty_like(x).normal_()
    v = {n: t for n, t in make(1, 1, D, "bf16", False, 5)[2].items()}
    cfg = rs.make_residual_norm_cfg(1, N, D, torch.bfloat16, rs.RS_NORM_LAYER, rs.RS_NORM_RMS, 1e-6, 1e-5, 1.0, 1.0)
    y, u_q, u_s = torch.empty_like(x), torch.empty(N, D + 16, dtype=torch.int8, device="cuda"), torch.empty(N, device="cuda")
    rs.rs_residual_norm_fwd(cfg, rs.make_residual_norm_weights(v), x, f, y, None, u_q[:, :D], u_s)
    for rows in (slice(0, 4), slice(1048574, 1048580), slice(N - 4, N)):
        ry, ru, ey, eu = reference(x[:, rows], f[:, rows], v, "layer", "rms", False, 1.0, 1.0)
        within(y[:, rows], ry, ey, "bf16")
        check8(u_q[rows], u_s[rows], ru, eu, D)


@pytest.mark.parametrize("D", [64, 256, 264, 512, 520, 1024, 2048, 2056])
@pytest.mark.parametrize("rows", [1, 3, 1023, 1025, 2047, 2050, 4095, 4099])
def test_every_number_of_lanes(rows, D):
    """Rows on more lanes where there are few of them: the sizes on both sides of each step, every image its own vectors, one row each."""
    x, f, v, stride = make(rows, 1, D, "bf16", True, seed=rows + D)
    cfg = rs.make_residual_norm_cfg(rows, 1, D, torch.bfloat16, rs.RS_NORM_LAYER, rs.RS_NORM_LAYER, 1e-6, 1e-5, 0.5, 2.0, stride, stride)
    y, u = torch.empty_like(x), torch.empty_like(x)
    u_q, u_s = torch.empty(rows, (D + 15) // 16 * 16, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    rs.rs_residual_norm_fwd(cfg, rs.make_residual_norm_weights(v), x, f, y, u, u_q[:, :D], u_s)
    ry, ru, ey, eu = reference(x, f, v, "layer", "layer", True, 0.5, 2.0)
    within(y, ry, ey, "bf16")
    within(u, ru, eu, "bf16")
    check8(u_q, u_s, ru, eu, D)


def test_vectors_that_do_not_fit_the_configuration_are_refused():
    B, N, D = 3, 4, 64
    x, f, v, stride = make(B, N, D, "bf16", True, seed=2)
    y = torch.empty_like(x)
    ok = dict(post=rs.RS_NORM_LAYER, pre=rs.RS_NORM_NONE, gate_stride=stride, mod_stride=stride)
    v["pre_g"] = v["pre_b"] = None
    call = lambda v, **kw: rs.rs_residual_norm_fwd(rs.make_residual_norm_cfg(B, N, D, torch.bfloat16, **{**ok, **kw}),  # noqa: E731
                                                   rs.make_residual_norm_weights(v), x, f, y, None)
    call(v)
    for bad in (dict(v, gate=v["gate"][:2]), dict(v, gate=v["gate"][:, :56]), dict(v, post_g=v["post_g"][:32]), dict(v, gate=v["gate"][0]),
                {n: None if t is None else t.float() for n, t in v.items()}):
        with pytest.raises(AssertionError):
            call(bad)
    with pytest.raises(AssertionError):
        call(v, gate_stride=0)
