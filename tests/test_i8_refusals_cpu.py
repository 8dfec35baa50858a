"""What the 8-bit linear layers and the fused residual / norm step refuse, before anything is launched; host side only."""
import ctypes

import pytest
import torch

import paper_2508_00367_amd as rs
from paper_2508_00367_amd import binding

P = [0x10000000 * (i + 1) for i in range(24)]   # far apart, aligned, never dereferenced
BAD, NO = rs.RS_ERR_INVALID_ARG, rs.RS_ERR_UNSUPPORTED
BIG = 1 << 44                                   # a place that nothing else is near


def test_struct_layouts_match_header():
    assert ctypes.sizeof(binding.RsResidualNormWeights) == 7 * 8
    assert ctypes.sizeof(binding.RsResidualNormCfg) == 10 * 4 + 2 * 8


def _refused(status, want, what):
    assert status == want, (what, status, rs.rs_last_error())
    assert rs.rs_last_error() != ""


@pytest.mark.parametrize("kw,want", [
    (dict(x=None), BAD), (dict(q=None), BAD), (dict(scale=None), BAD), (dict(M=-1), BAD), (dict(M=1 << 31), BAD), (dict(K=0), BAD),
    (dict(K=131072, ldx=131072, ldq=131072), NO), (dict(ldx=95), BAD), (dict(ldq=80), BAD), (dict(ldq=100), BAD), (dict(ldx=1 << 30), NO),
    (dict(ldq=1 << 30), NO), (dict(dtype=2), BAD), (dict(dtype=-1), BAD), (dict(x=P[0] + 8), BAD), (dict(q=P[1] + 4), BAD), (dict(scale=P[2] + 2), BAD),
    (dict(q=P[0] + 16), BAD), (dict(scale=P[0] + 32), BAD), (dict(scale=P[1] + 4), BAD)])
def test_quantize_rows_refuses(kw, want):
    a = dict(x=P[0], M=10, K=96, ldx=96, dtype=rs.RS_BF16, q=P[1], ldq=96, scale=P[2])
    a.update(kw)
    _refused(rs.lib().rs_quantize_rows(a["x"], a["M"], a["K"], a["ldx"], a["dtype"], a["q"], a["ldq"], a["scale"], None), want, kw)


@pytest.mark.parametrize("kw,want", [
    (dict(w=None), BAD), (dict(q=None), BAD), (dict(scale=None), BAD), (dict(K=0), BAD), (dict(N=0), BAD), (dict(N=-3), BAD),
    (dict(K=131072), NO), (dict(N=(1 << 20) + 1), NO), (dict(dtype=5), BAD), (dict(w=P[0] + 2), BAD), (dict(q=P[1] + 1), BAD),
    (dict(scale=P[2] + 1), BAD), (dict(q=P[0]), BAD), (dict(scale=P[0] + 16), BAD)])
def test_quantize_columns_refuses(kw, want):
    a = dict(w=P[0], K=64, N=48, dtype=rs.RS_F32, q=P[1], scale=P[2])
    a.update(kw)
    _refused(rs.lib().rs_quantize_columns(a["w"], a["K"], a["N"], a["dtype"], a["q"], a["scale"], None), want, kw)


def test_pack_refuses_and_sizes():
    L = rs.lib()
    for args, want in [((None, P[1], 64, 64), BAD), ((P[0], None, 64, 64), BAD), ((P[0], P[1], 0, 64), BAD), ((P[0], P[1], 64, -1), BAD),
                       ((P[0], P[1], 131072, 64), NO), ((P[0] + 3, P[1], 64, 64), BAD), ((P[0], P[1] + 8, 64, 64), BAD), ((P[0], P[0] + 64, 64, 64), BAD)]:
        _refused(L.rs_pack_linear_i8(*args, None), want, args)
    assert rs.rs_packed_linear_i8_size(0, 64) == rs.rs_packed_linear_i8_size(64, 0) == rs.rs_packed_linear_i8_size(131072, 64) == 0
    assert rs.rs_packed_linear_i8_size(64, (1 << 20) + 1) == 0
    for K, N in [(1, 1), (64, 64), (588, 1000), (131071, 1 << 20)]:
        assert rs.rs_packed_linear_i8_size(K, N) >= K * N


@pytest.mark.parametrize("kw,want", [
    (dict(a=None), BAD), (dict(a_scale=None), BAD), (dict(w=None), BAD), (dict(w_scale=None), BAD), (dict(out=None), BAD),
    (dict(res=None, epi=rs.RS_EPI_BIAS_RES), BAD), (dict(M=-1), BAD), (dict(M=1 << 31), BAD), (dict(N=0), BAD), (dict(K=0), BAD), (dict(K=-64), BAD),
    (dict(K=131072, lda=131072), NO), (dict(N=(1 << 20) + 1), NO), (dict(lda=80), BAD), (dict(lda=100), BAD), (dict(lda=(1 << 21) + 16), NO),
    (dict(epi=3), BAD), (dict(epi=-1), BAD), (dict(dtype=2), BAD), (dict(a=P[0] + 8), BAD), (dict(a_scale=P[1] + 2), BAD), (dict(w=P[2] + 4), BAD),
    (dict(w_scale=P[3] + 4), BAD), (dict(bias=P[4] + 2), BAD), (dict(res=P[5] + 8, epi=rs.RS_EPI_BIAS_RES), BAD), (dict(out=P[6] + 4), BAD),
    (dict(out=P[0] + 16), BAD), (dict(out=P[1]), BAD), (dict(out=P[2] + 64), BAD), (dict(out=P[3]), BAD), (dict(out=P[4]), BAD),
    (dict(out=P[5] + 16, epi=rs.RS_EPI_BIAS_RES), BAD)])
def test_linear_i8_refuses(kw, want):
    a = dict(a=P[0], lda=96, a_scale=P[1], w=P[2], w_scale=P[3], bias=P[4], res=P[5], out=P[6], M=10, N=64, K=96, epi=rs.RS_EPI_BIAS,
             dtype=rs.RS_BF16)
    a.update(kw)
    _refused(rs.lib().rs_linear_i8_fwd(*[a[k] for k in ("a", "lda", "a_scale", "w", "w_scale", "bias", "res", "out", "M", "N", "K", "epi", "dtype")],
                                       None), want, kw)


_CFG = dict(B=2, N=5, D=64, dtype=rs.RS_BF16, post=rs.RS_NORM_LAYER, pre=rs.RS_NORM_RMS)
_W = dict(post_g=P[10], post_b=P[11], gate=P[12], pre_g=P[13], pre_b=P[14], mod_scale=P[15], mod_shift=P[16])


@pytest.mark.parametrize("c,v,kw,want", [
    (dict(dtype=3), {}, {}, BAD), (dict(post=3), {}, {}, BAD), (dict(pre=-1), {}, {}, BAD), (dict(B=-1), {}, {}, BAD), (dict(N=-1), {}, {}, BAD),
    (dict(D=0), {}, {}, BAD), (dict(D=60), {}, {}, NO), (dict(D=16392), {}, {}, NO), (dict(B=1 << 16, N=1 << 15), {}, {}, NO),
    (dict(post_eps=0.0), {}, {}, BAD), (dict(pre_eps=-1.0), {}, {}, BAD), (dict(pre_eps=float("nan")), {}, {}, BAD),
    (dict(gate_stride=-64), {}, {}, BAD), (dict(mod_stride=60), {}, {}, BAD), (dict(gate_stride=1 << 30), {}, {}, NO), (dict(mod_stride=1 << 30), {}, {}, NO),
    (dict(post=rs.RS_NORM_NONE), {}, {}, BAD), (dict(pre=rs.RS_NORM_NONE), {}, {}, BAD), (dict(), {}, dict(f=None), BAD),
    (dict(post=rs.RS_NORM_NONE), dict(post_g=None, post_b=None), dict(f=None), BAD),                 # a gate without a branch
    (dict(), {}, dict(u_q=None), BAD), (dict(), {}, dict(u_scale=None), BAD), (dict(), {}, dict(y=None, u=None, u_q=None, u_scale=None), BAD),
    (dict(), {}, dict(ldq=48), BAD), (dict(), {}, dict(ldq=72), BAD), (dict(), {}, dict(ldq=1 << 30), NO), (dict(), {}, dict(x=None), BAD),
    (dict(), {}, dict(x=P[0] + 8), BAD), (dict(), {}, dict(f=P[1] + 2), BAD), (dict(), {}, dict(y=P[2] + 4), BAD), (dict(), {}, dict(u=P[3] + 8), BAD),
    (dict(), {}, dict(u_q=P[4] + 4), BAD), (dict(), {}, dict(u_scale=P[5] + 2), BAD), (dict(), dict(gate=P[12] + 2), {}, BAD), (dict(), dict(mod_shift=P[16] + 8), {}, BAD),
    (dict(), {}, dict(y=P[1]), BAD), (dict(), {}, dict(u=P[0]), BAD), (dict(), {}, dict(y=P[0] + 16), BAD), (dict(), {}, dict(u=P[1] + 16), BAD),
    (dict(), {}, dict(u=P[2]), BAD), (dict(), {}, dict(u_q=P[0]), BAD), (dict(), {}, dict(u_q=P[3] + 16), BAD), (dict(), {}, dict(u_scale=P[4] + 8), BAD),
    (dict(), {}, dict(u_scale=P[13] + 4), BAD), (dict(mod_stride=4096), {}, dict(y=P[15] + 2 * 4096 + 16), BAD), (dict(gate_stride=4096), {}, dict(u=P[12] + 2 * 4096), BAD)])
def test_residual_norm_refuses(c, v, kw, want):
    cfg = rs.make_residual_norm_cfg(**{k: n for k, n in {**_CFG, **c}.items()})
    w = binding.RsResidualNormWeights()
    for name, p in {**_W, **v}.items():
        setattr(w, name, p)
    a = dict(x=P[0], f=P[1], y=P[2], u=P[3], u_q=P[4], ldq=64, u_scale=P[5])
    a.update(kw)
    _refused(rs.lib().rs_residual_norm_fwd(ctypes.byref(cfg), ctypes.byref(w), *[a[k] for k in ("x", "f", "y", "u", "u_q", "ldq", "u_scale")], None),
             want, (c, v, kw))


def test_null_structs_and_empty_calls():
    L = rs.lib()
    cfg, w = rs.make_residual_norm_cfg(**_CFG), binding.RsResidualNormWeights()
    _refused(L.rs_residual_norm_fwd(None, ctypes.byref(w), P[0], P[1], P[2], P[3], None, 0, None, None), BAD, "cfg")
    _refused(L.rs_residual_norm_fwd(ctypes.byref(cfg), None, P[0], P[1], P[2], P[3], None, 0, None, None), BAD, "weights")
    for empty in (dict(B=0), dict(N=0)):
        cfg = rs.make_residual_norm_cfg(**{**_CFG, **empty})
        assert L.rs_residual_norm_fwd(ctypes.byref(cfg), ctypes.byref(w), None, P[1], P[2], P[3], None, 0, None, None) == rs.RS_OK
    assert L.rs_quantize_rows(None, 0, 96, 96, rs.RS_BF16, None, 96, None, None) == rs.RS_OK
    assert L.rs_linear_i8_fwd(None, 96, None, None, None, None, None, None, 0, 64, 96, rs.RS_EPI_BIAS, rs.RS_BF16, None) == rs.RS_OK


def test_the_binding_refuses_tensors_that_are_not_on_the_gpu():
    f, q, s = torch.zeros(4, 16), torch.zeros(4, 16, dtype=torch.int8), torch.zeros(4)
    cfg = rs.make_residual_norm_cfg(1, 4, 16, rs.RS_F32)
    for call in (lambda: rs.rs_quantize_rows(f, q, s), lambda: rs.rs_quantize_columns(f, q, torch.zeros(16)),
                 lambda: rs.rs_pack_linear_i8(q, torch.zeros(1 << 14, dtype=torch.uint8)),
                 lambda: rs.rs_linear_i8_fwd(q, s, torch.zeros(1 << 14, dtype=torch.uint8), s, None, None, torch.zeros(4, 4)),
                 lambda: rs.rs_residual_norm_fwd(cfg, rs.make_residual_norm_weights({}), f, None, None, f.clone()),
                 lambda: rs.make_residual_norm_weights(dict(pre_g=torch.ones(16)))):
        with pytest.raises(AssertionError, match="device"):
            call()
