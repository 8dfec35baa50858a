"""8-bit linear layers on the GPU: quantization of rows and columns bit for bit, products against 64 bits, ragged sizes."""
import sys

import numpy as np
import pytest
import torch

import paper_2508_00367_amd as rs
from i8_testlib import DT, f64, linear_bound, linear_i8, quantize

pytestmark = pytest.mark.gpu

EPI = {"bias": rs.RS_EPI_BIAS, "gelu": rs.RS_EPI_BIAS_GELU, "res": rs.RS_EPI_BIAS_RES}


def _say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def rows8(M, K, extra=0, fill=0):
    """int8 rows a multiple of 16 bytes apart, `extra` x 16 bytes of room behind them; every byte `fill`."""
    return torch.full((M, (K + 15) // 16 * 16 + 16 * extra), fill, dtype=torch.int8, device="cuda")


def packed(w):
    p = torch.full((rs.rs_packed_linear_i8_size(*w.shape) + 64,), 77, dtype=torch.uint8, device="cuda")
    rs.rs_pack_linear_i8(w, p)
    assert bool((p[-64:] == 77).all())  # nothing behind the size the library asks for
    return p


def run_linear(a, a_scale, w, w_scale, bias, res, dtype, epi, stream=None):
    """The output, from a buffer whose rows before and behind it must stay as they were."""
    M, N = a.shape[0], w.shape[1]
    guard = (1024 // N + 8) // 8 * 8       # rows; the output starts 16-byte aligned
    buf = torch.full((M + 2 * guard, N), -777.0, dtype=DT[dtype], device="cuda")
    pw = packed(w)
    torch.cuda.synchronize()
    rs.rs_linear_i8_fwd(a, a_scale, pw, w_scale, bias, res, buf[guard:guard + M], EPI[epi], stream)
    torch.cuda.synchronize()
    assert bool((buf[:guard] == -777).all()) and bool((buf[guard + M:] == -777).all())
    return buf[guard:guard + M]


def make(M, K, N, dtype, epi, seed, extra=0, lo=-128, hi=128):
    g = torch.Generator().manual_seed(seed)
    a = rows8(M, K, extra, fill=113)       # whatever lies behind column K
    a[:, :K] = torch.randint(lo, hi, (M, K), generator=g).to(torch.int8).cuda()
    w = torch.randint(lo, hi, (K, N), generator=g).to(torch.int8).cuda()
    a_scale = (torch.rand(M, generator=g) * 0.02 + 1e-3).cuda()
    w_scale = (torch.rand(N, generator=g) * 0.02 / K ** 0.5 + 1e-4).cuda()
    bias = torch.randn(N, generator=g).to(DT[dtype]).cuda()
    res = torch.randn(M, N, generator=g).to(DT[dtype]).cuda() if epi == "res" else None
    return a[:, :K], a_scale, w, w_scale, bias, res


def check(out, a, a_scale, w, w_scale, bias, res, dtype, epi):
    ref, size = linear_i8(a.cpu().numpy(), f64(a_scale), w.cpu().numpy(), f64(w_scale), None if bias is None else f64(bias),
                          None if res is None else f64(res), epi)
    tol = linear_bound(ref, size, epi, dtype)
    worst = np.max(np.abs(f64(out) - ref) / tol)
    _say("  worst %.3f of the bound" % worst)
    assert worst <= 1.0


SHAPES = [(1, 1, 1), (2, 17, 5), (1, 768, 2304), (5, 64, 64), (17, 16, 1000), (31, 128, 64), (33, 129, 65), (64, 127, 192),
          (65, 100, 63), (127, 588, 257), (129, 640, 128), (197, 768, 768), (256, 256, 256), (300, 131, 520), (513, 1024, 320),
          (1003, 588, 1000)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("epi", ["bias", "gelu", "res"])
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_linear_i8(M, K, N, epi, dtype):
    _say("linear_i8", M, K, N, epi, dtype)
    t = make(M, K, N, dtype, epi, seed=M + K + N, extra=(M + N) % 3)
    check(run_linear(*t, dtype, epi), *t, dtype, epi)


# One size for each kernel, rows of whole 16-byte pieces and others: tests/test_i8_choice_cpu.py has which is which.
EVERY_KERNEL = [(40, 300, 200), (197, 768, 2304), (197, 770, 1155), (788, 768, 768), (900, 200, 1001), (788, 4096, 1024), (1576, 768, 2304),
                (1700, 1300, 2051), (1576, 1024, 4096), (2500, 1100, 3001), (3000, 2048, 4096), (3000, 2100, 4001)]


@pytest.mark.parametrize("epi,dtype", [("bias", "bf16"), ("gelu", "bf16"), ("res", "bf16"), ("res", "f32"), ("gelu", "f32")])
@pytest.mark.parametrize("M,K,N", EVERY_KERNEL)
def test_every_kernel(M, K, N, epi, dtype):
    """Against 64 bits in the outer rows and columns and a sample of the others, where a tile's edges are."""
    _say("every kernel", M, K, N, epi, dtype)
    a, a_s, w, w_s, bias, res = make(M, K, N, dtype, epi, seed=M + N)
    out = run_linear(a, a_s, w, w_s, bias, res, dtype, epi)
    rows = sorted(set(range(70)) | set(range(M - 140, M)) | set(range(0, M, 37))) if M > 400 else list(range(M))
    check(out[rows], a[rows], a_s[rows], w, w_s, bias, None if res is None else res[rows], dtype, epi)
    cols = sorted(set(range(min(N, 70))) | set(range(max(N - 70, 0), N)))
    check(out[:, cols], a, a_s, w[:, cols], w_s[cols], bias[cols], None if res is None else res[:, cols], dtype, epi)


@pytest.mark.parametrize("K", [1, 127, 128, 129, 640, 1024, 1025, 2048, 3200, 5000, 9000])
@pytest.mark.parametrize("M,N", [(33, 70), (300, 1100), (1100, 3000), (2900, 4000)])
def test_every_length_of_the_inner_axis(M, N, K):
    """Rings and peeled tails of every kernel, from one slice to many; exact sums, so every row is the same where the rows are."""
    _say("inner axis", M, K, N)
    a, a_s, w, w_s, bias, _ = make(M, K, N, "f32", "bias", seed=K)
    a[1:], a_s[1:] = a[:1].clone(), a_s[:1].clone()
    out = run_linear(a, a_s, w, w_s, bias, None, "f32", "bias")
    check(out[:1], a[:1], a_s[:1], w, w_s, bias, None, "f32", "bias")
    assert bool((out == out[:1]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_bias_no_rows_and_out_is_res(dtype):
    a, a_s, w, w_s, bias, res = make(70, 96, 136, dtype, "res", 5)
    check(run_linear(a, a_s, w, w_s, None, None, dtype, "bias"), a, a_s, w, w_s, None, None, dtype, "bias")
    pw = packed(w)
    rs.rs_linear_i8_fwd(a[:0], a_s[:0], pw, w_s, bias, None, torch.empty(0, 136, dtype=DT[dtype], device="cuda"))
    inout = res.clone()
    rs.rs_linear_i8_fwd(a, a_s, pw, w_s, bias, inout, inout, rs.RS_EPI_BIAS_RES)
    check(inout, a, a_s, w, w_s, bias, res, dtype, "res")


def test_sums_at_the_edge_of_32_bits():
    """K = 131071 products of -128 and -128: 2147467264, under 2^31; and the alternating sum."""
    K = 131071
    a, w = rows8(3, K), torch.full((K, 4), -128, dtype=torch.int8, device="cuda")
    a[:, :K] = -128
    a[1, :K] = 127
    a[2, 1:K:2] = 127
    ones = torch.ones(4, device="cuda")
    out = run_linear(a[:, :K], ones[:3], w, ones, None, None, "f32", "bias")
    ref = (a[:, :K].long().cpu() @ w.long().cpu()).double().numpy()
    assert np.array_equal(f64(out), ref.astype(np.float32).astype(np.float64))


def test_scales_of_any_kind():
    """A NaN scale makes its row NaN and leaves the others; zero scales leave the bias."""
    a, a_s, w, w_s, bias, _ = make(40, 64, 72, "f32", "bias", 9)
    a_s[3], a_s[39], a_s[17] = float("nan"), float("nan"), 0.0
    out = run_linear(a, a_s, w, w_s, bias, None, "f32", "bias")
    nan = torch.isnan(out)
    assert bool(nan[[3, 39]].all()) and int(nan.sum()) == 2 * 72
    assert torch.equal(out[17], bias)
    keep = [i for i in range(40) if i not in (3, 39)]
    check(out[keep], a[keep], a_s[keep], w, w_s, bias, None, "f32", "bias")


def test_scale_views_and_row_ranges():
    """Any rows of a larger batch: a scale pointer that is only 4-byte aligned."""
    a, a_s, w, w_s, bias, _ = make(300, 80, 96, "bf16", "bias", 11)
    whole = run_linear(a, a_s, w, w_s, bias, None, "bf16", "bias")
    part = run_linear(a[37:250], a_s[37:250], w, w_s, bias, None, "bf16", "bias")
    assert torch.equal(part, whole[37:250])


# ---- quantization -----------------------------------------------------------------------------------------------------
QSHAPES = [(1, 1), (1, 768), (3, 7), (197, 768), (64, 588), (33, 1000), (5, 4096), (2, 4100), (3, 16384), (2, 40001), (300, 192),
           (1000, 64), (1, 131071)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K", QSHAPES)
def test_quantize_rows(M, K, dtype):
    _say("quantize_rows", M, K, dtype)
    g = torch.Generator().manual_seed(M * 7 + K)
    for pitch in (K, K + 8, K + 13):
        wide = (torch.randn(M, pitch, generator=g) * torch.exp(torch.randn(M, 1, generator=g))).to(DT[dtype]).cuda()
        x = wide[:, :K]
        q, scale = rows8(M, K, extra=1, fill=55), torch.full((M + 2,), -1.0, device="cuda")
        rs.rs_quantize_rows(x, q[:, :K], scale[1:M + 1])
        torch.cuda.synchronize()
        rq, rscale = quantize(x.float().cpu().numpy(), 1)
        assert np.array_equal(q[:, :K].cpu().numpy(), rq)
        assert np.array_equal(scale[1:M + 1].cpu().numpy(), rscale)
        assert float(scale[0]) == float(scale[-1]) == -1.0
        pad = (K + 15) // 16 * 16
        assert bool((q[:, K:pad] == 0).all()) and bool((q[:, pad:] == 55).all())


@pytest.mark.parametrize("K", [40, 64, 1024, 5000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_special_rows(K, dtype):
    """Zeros, one value only, the smallest numbers, halves that go to even, the largest numbers, infinities and NaN."""
    x = torch.zeros(12, K)
    x[1, K // 2] = -3.5
    x[2] = 2.0 ** -149 if dtype == "f32" else 2.0 ** -133
    x[3] = 1e-37
    x[4, 0], x[4, 1:20] = 127.0, torch.arange(19) - 8.5
    x[5] = torch.finfo(DT[dtype]).max
    x[6, 3] = float("inf")
    x[7, K - 1] = float("-inf")
    x[8, K - 2] = float("nan")
    x[9, 0], x[9, 1] = float("nan"), float("inf")
    x[10] = torch.linspace(-1, 1, K)
    x[11] = -0.0
    x = x.to(DT[dtype]).cuda()
    q, scale = rows8(12, K), torch.empty(12, device="cuda")
    rs.rs_quantize_rows(x, q[:, :K], scale)
    rq, rscale = quantize(x.float().cpu().numpy(), 1)
    assert np.array_equal(q[:, :K].cpu().numpy(), rq)
    assert np.array_equal(scale.cpu().numpy(), rscale, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K,N", [(1, 1), (5, 3), (33, 31), (64, 64), (588, 1000), (768, 2304), (1025, 33)])
def test_quantize_columns(K, N, dtype):
    g = torch.Generator().manual_seed(K + N)
    w = (torch.randn(K, N, generator=g) * torch.exp(torch.randn(N, generator=g)))
    w[:, N // 2] = 0
    w[K // 2, 0] = float("nan")
    w = w.to(DT[dtype]).cuda()
    q, scale = torch.empty(K, N, dtype=torch.int8, device="cuda"), torch.full((N + 1,), -1.0, device="cuda")
    rs.rs_quantize_columns(w, q, scale[:N])
    rq, rscale = quantize(w.float().cpu().numpy(), 0)
    assert np.array_equal(q.cpu().numpy(), rq)
    assert np.array_equal(scale[:N].cpu().numpy(), rscale, equal_nan=True) and float(scale[N]) == -1.0


# ---- as they are used -------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layer_from_rows_of_the_type(dtype):
    """quantize columns -> pack, quantize rows -> product: the bits of the plain form's integers, on a stream of its own."""
    M, K, N = 197, 768, 1152
    g = torch.Generator().manual_seed(3)
    x = torch.randn(M, K, generator=g).to(DT[dtype]).cuda()
    wf = (torch.randn(K, N, generator=g) * 0.02).to(DT[dtype]).cuda()
    bias = torch.randn(N, generator=g).to(DT[dtype]).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        w, w_s = torch.empty(K, N, dtype=torch.int8, device="cuda"), torch.empty(N, device="cuda")
        rs.rs_quantize_columns(wf, w, w_s)
        a, a_s = rows8(M, K), torch.empty(M, device="cuda")
        rs.rs_quantize_rows(x, a, a_s)
        pw = torch.empty(rs.rs_packed_linear_i8_size(K, N), dtype=torch.uint8, device="cuda")
        rs.rs_pack_linear_i8(w, pw)
        out = torch.empty(M, N, dtype=DT[dtype], device="cuda")
        rs.rs_linear_i8_fwd(a, a_s, pw, w_s, bias, None, out, rs.RS_EPI_BIAS_GELU)
    side.synchronize()
    aq, as_ = quantize(x.float().cpu().numpy(), 1)
    wq, ws = quantize(wf.float().cpu().numpy(), 0)
    ref, size = linear_i8(aq, as_, wq, ws, f64(bias), None, "gelu")
    assert np.all(np.abs(f64(out) - ref) <= linear_bound(ref, size, "gelu", dtype))


def test_captured_and_replayed():
    """A graph of quantization and product, replayed on new inputs between eager calls, gives the eager call's bits."""
    M, K, N = 50, 200, 328
    _, _, w, w_s, bias, _ = make(M, K, N, "bf16", "bias", 21)
    pw = packed(w)
    x = torch.randn(M, K, device="cuda").bfloat16()
    a, a_s, out = rows8(M, K)[:, :K], torch.empty(M, device="cuda"), torch.empty(M, N, dtype=torch.bfloat16, device="cuda")

    def call(out):
        rs.rs_quantize_rows(x, a, a_s)
        rs.rs_linear_i8_fwd(a, a_s, pw, w_s, bias, None, out)

    call(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for i in range(4):
        x.copy_(torch.randn(M, K, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        eager = torch.empty_like(out)
        call(eager)
        torch.cuda.synchronize()
        assert torch.equal(got, eager), i


def test_offsets_past_32_bits():
    """Outputs of 2.4e9 elements; activations whose rows lie 2 MiB apart over 2.3 GB; the last rows and columns against 64 bits."""
    M, K, N = 60000, 16, 40000
    a, a_s, w, w_s, bias, _ = make(M, K, N, "bf16", "bias", 31)
    out = torch.full((M, N), -777.0, dtype=torch.bfloat16, device="cuda")
    rs.rs_linear_i8_fwd(a, a_s, packed(w), w_s, bias, None, out)
    for rows in (slice(0, 3), slice(53686, 53690), slice(M - 3, M)):   # element 2^31 lies in row 53687
        check(out[rows], a[rows], a_s[rows], w, w_s, bias, None, "bf16", "bias")
    del out
    far = torch.full((1100, 1 << 21), 55, dtype=torch.int8, device="cuda")
    a2, a2_s, w2, w2_s, b2, _ = make(1100, 64, 96, "f32", "bias", 32)
    far[:, :64] = a2
    check(run_linear(far[:, :64], a2_s, w2, w2_s, b2, None, "f32", "bias"), a2, a2_s, w2, w2_s, b2, None, "f32", "bias")


def test_quantize_rows_past_32_bits():
    M, K = 1100000, 2048
    x = torch.empty(M, K, dtype=torch.bfloat16, device="cuda")
    x.normal_()
    q, scale = torch.full((M + 1, K), 55, dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    rs.rs_quantize_rows(x, q[:M], scale)
    for rows in (slice(0, 4), slice(1048574, 1048580), slice(M - 4, M)):
        rq, rscale = quantize(x[rows].float().cpu().numpy(), 1)
        assert np.array_equal(q[rows].cpu().numpy(), rq) and np.array_equal(scale[rows].cpu().numpy(), rscale)
    assert bool((q[M] == 55).all())


def test_two_streams_at_once():
    """No workspace, nothing shared: two calls that overlap in time give what each gives alone."""
    t = [make(900, 1024, 1000, "bf16", "gelu", s) for s in (41, 42)]
    alone = [run_linear(*x, "bf16", "gelu") for x in t]
    pws = [packed(x[2]) for x in t]
    outs = [torch.empty_like(o) for o in alone]
    streams = [torch.cuda.Stream() for _ in t]
    torch.cuda.synchronize()
    for _ in range(10):
        for x, pw, o, s in zip(t, pws, outs, streams):
            rs.rs_linear_i8_fwd(x[0], x[1], pw, x[3], x[4], None, o, rs.RS_EPI_BIAS_GELU, s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(alone, outs))


def test_rows_that_have_no_room_for_their_last_bytes_are_refused():
    """A row of 100 bytes is written up to byte 112: not into what lies behind it."""
    x, scale = torch.randn(3, 100, device="cuda"), torch.empty(3, device="cuda")
    tight = torch.full((5, 100), 55, dtype=torch.int8, device="cuda")
    for rows in (3, 1):
        with pytest.raises((rs.RsError, AssertionError)):
            rs.rs_quantize_rows(x[:rows], tight[:rows], scale[:rows])
    last = torch.full((2 * 112 + 100,), 55, dtype=torch.int8, device="cuda").as_strided((3, 100), (112, 1))
    with pytest.raises(AssertionError, match="room"):
        rs.rs_quantize_rows(x, last, scale)
    pw = packed(torch.ones(100, 8, dtype=torch.int8, device="cuda"))
    with pytest.raises(AssertionError, match="room"):
        rs.rs_linear_i8_fwd(last, scale, pw, torch.ones(8, device="cuda"), None, None, torch.empty(3, 8, device="cuda"))
    torch.cuda.synchronize()
    assert bool((tight == 55).all()) and bool((last == 55).all())
    one = torch.empty(112, dtype=torch.int8, device="cuda")       # a single row: any stride will do where it is whole
    rs.rs_quantize_rows(torch.randn(1, 112, device="cuda"), one.as_strided((1, 112), (1, 1)), scale[:1])
