"""The 8-bit operators together, as a block uses them: EncoderBlockI8, each step against 64 bits on what the step before left."""
import sys

import numpy as np
import pytest
import torch

import oracle
import paper_2508_00367_amd as rs
import synth_inputs as si
from i8_testlib import DT, U16, U32, f64, linear_bound, linear_i8, quantize, residual_norm
from rs_testlib import TOL, host_round, norm_err, to_dev

pytestmark = pytest.mark.gpu


def _say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def _block(B, N, D, H, Dm, dtype, post, seed=0):
    w = {k: to_dev(host_round(v, dtype), dtype) for k, v in si.block_weights(seed, 0, D, Dm).items()}
    if post != rs.RS_NORM_NONE:
        for i in (1, 2):
            w["post%d_g" % i] = to_dev(host_round(1 + si.generic(seed, 40 + i, (D,), std=0.1), dtype), dtype)
            w["gate%d" % i] = to_dev(host_round(si.generic(seed, 50 + i, (D,), std=0.5), dtype), dtype)
        w["ln1_b"] = None
    x = to_dev(host_round(si.tokens(seed, B, N, D, spread=0.4), dtype), dtype)
    return w, x


def _near(got, ref, err, dtype):
    tol = 1.01 * err + (U16 if dtype == "bf16" else U32) * (np.abs(ref) + err)
    assert np.all(np.abs(f64(got).reshape(ref.shape) - ref) <= np.maximum(tol, 1e-300))


def _same_8bit(q, scale, u, eu, D):
    s = f64(scale)[:, None]
    u, eu = u.reshape(-1, D), eu.reshape(-1, D)
    assert np.all(np.abs(q.cpu().numpy().astype(np.float64) * s - u) <= s * (0.5 + 3 * U32 * 127) + eu)


@pytest.mark.parametrize("B,N,D,H,Dm,P,K", [(2, 197, 192, 3, 768, 1, 140), (1, 50, 64, 1, 200, 0, 50), (3, 65, 128, 2, 520, 2, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("norm,post", [("layer", "none"), ("rms", "rms")])
def test_each_step_of_a_block(B, N, D, H, Dm, P, K, dtype, norm, post):
    _say("block", B, N, D, H, Dm, P, K, dtype, norm, post)
    kind = {"none": rs.RS_NORM_NONE, "layer": rs.RS_NORM_LAYER, "rms": rs.RS_NORM_RMS}
    w, x = _block(B, N, D, H, Dm, dtype, kind[post])
    blk = rs.EncoderBlockI8(B, N, D, H, Dm, w, P, K, kind[norm], kind[post], x_scale=0.9, f_scale=1.1)
    h = {k: None if v is None else f64(v) for k, v in w.items()}
    g = lambda k: None if h.get(k) is None else h[k]  # noqa: E731
    M, seen = B * N, {}
    names = ("rs_residual_norm_fwd", "rs_linear_i8_fwd", "rs_quantize_rows")
    keep, order = {n: getattr(rs.binding, n) for n in names}, []

    def spy(name):
        def call(*a):
            keep[name](*a)
            torch.cuda.synchronize()
            i = len(order)
            order.append(name)
            seen[i] = {k: t.clone() for k, t in (("q", blk.q), ("qs", blk.q_scale), ("hq", blk.hq), ("hs", blk.h_scale), ("branch", blk.branch))}
        return call

    import paper_2508_00367_amd.runner as runner
    try:
        for n in names:
            setattr(runner.rs, n, spy(n))
        y, kept, scores = blk.step(x)
    finally:
        for n in names:
            setattr(runner.rs, n, keep[n])
    torch.cuda.synchronize()
    assert order == [names[0], names[1], names[2], names[1], names[0], names[1], names[2], names[1], names[0]]

    def layer(a, a_s, name, epi, out):
        wq, ws = quantize(w["w_" + name].float().cpu().numpy(), 0)
        ref, size = linear_i8(a.cpu().numpy(), f64(a_s), wq, ws, h["b_" + name], None, epi)
        assert np.all(np.abs(f64(out).reshape(ref.shape) - ref) <= linear_bound(ref, size, epi, dtype)), name

    _, u, _, eu = residual_norm(f64(x), None, "none", norm, 1e-6, 1e-6, 1.0, 1.0, dict(pre_g=g("ln1_g"), pre_b=g("ln1_b") if norm == "layer" else None))
    _same_8bit(seen[0]["q"], seen[0]["qs"], u, eu, D)
    layer(seen[0]["q"], seen[0]["qs"], "qkv", "bias", blk.qkv)
    qkv = f64(blk.qkv)
    att = oracle.attention(qkv[:, :, 0], qkv[:, :, 1], qkv[:, :, 2], 0.125)
    assert norm_err(f64(blk.att).reshape(att.shape), att) < TOL[dtype]
    q, s = quantize(blk.att.float().cpu().numpy().reshape(M, D), 1)
    assert np.array_equal(seen[2]["q"].cpu().numpy(), q) and np.array_equal(seen[2]["qs"].cpu().numpy(), s)
    layer(seen[2]["q"], seen[2]["qs"], "proj", "bias", seen[3]["branch"])
    x1, u, e1, eu = residual_norm(f64(x), f64(seen[3]["branch"]).reshape(B, N, D), post, norm, 1e-6, 1e-6, 0.9, 1.1, dict(
        post_g=g("post1_g"), gate=g("gate1"), pre_g=g("ln2_g"), pre_b=g("ln2_b")))
    _near(blk.x1, x1, e1, dtype)
    _same_8bit(seen[4]["q"], seen[4]["qs"], u, eu, D)
    layer(seen[4]["q"], seen[4]["qs"], "fc1", "gelu", blk.hid)
    q, s = quantize(blk.hid.float().cpu().numpy(), 1)
    assert np.array_equal(blk.hq.cpu().numpy(), q) and np.array_equal(blk.h_scale.cpu().numpy(), s)
    layer(blk.hq, blk.h_scale, "fc2", "bias", blk.branch)
    f2 = f64(blk.branch).reshape(B, N, D)
    xhat, _, e2, _ = residual_norm(f64(blk.x1), f2, post, "none", 1e-6, 1e-6, 0.9, 1.1, dict(post_g=g("post2_g"), gate=g("gate2")))
    _near(blk.xhat, xhat, e2, dtype)
    sc = f64(scores)
    assert norm_err(sc, np.sqrt(((f2 - f64(blk.x1)) ** 2).sum(-1))) < 1e-5
    assert np.array_equal(kept.cpu().numpy(), oracle.topk(sc, P, K))
    assert np.array_equal(f64(y), oracle.gather(f64(blk.xhat), kept.cpu().numpy()))


def test_near_the_block_in_full_precision():
    """The 8-bit block against the fp64 oracle's block: every operand of the four products is off by at most half of 1/127 of its row's or
    column's largest value, 0.29 of a step rms; rows of unit normals reach 3.5 of their standard deviation, so that is 0.8 % of an
    operand, and 1.1 % of a product of two, for a branch of two layers (and softmax or GELU, of slope 1.13 at most, between them) 1.8 %.
    Twice that, relative in the 2-norm, for the two branches and the residual stream that carries the first into the second."""
    B, N, D, H, Dm = 2, 197, 384, 6, 1536
    w, x = _block(B, N, D, H, Dm, "bf16", rs.RS_NORM_NONE)
    blk = rs.EncoderBlockI8(B, N, D, H, Dm, w, 1, 196)
    blk.step(x)
    torch.cuda.synchronize()
    ref = oracle.block(f64(x).astype(np.float32), {k: f64(v).astype(np.float32) for k, v in w.items()}, H)
    got = f64(blk.xhat)
    off = np.linalg.norm(got - ref["xhat"]) / np.linalg.norm(ref["xhat"])
    _say("xhat off by %.4f" % off)
    assert off < 0.036


def test_captured_and_replayed():
    B, N, D, H, Dm = 2, 65, 128, 2, 512
    w, x = _block(B, N, D, H, Dm, "bf16", rs.RS_NORM_NONE)
    blk, eager = (rs.EncoderBlockI8(B, N, D, H, Dm, w, 1, 40) for _ in range(2))
    blk.step(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        blk.step(x)
    for i in range(4):
        x.copy_(torch.randn(B, N, D, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (blk.y, blk.kept, blk.scores)]
        want = eager.step(x)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
