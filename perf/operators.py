"""The 8-bit linear layers and the fused residual / normalisation step: what is measured of them.

A case is a dict of plain values.  `prepare` makes what a program holds before the call (inputs on the GPU from a seed,
packed weights, output buffers), `run` is one pass, through the framework's entry points where `own` is true and in
elementary torch operations otherwise, `work` is what a pass cannot do without and `exact` the result in 64 bits.

Operators (`op`)
  quantize  rows to 8-bit integers with one scale a row
  linear    out = epilogue((a_q w_q) a_scale w_scale + bias); `quant`: the rows arrive in `dtype` and are quantized first
  norm      y = x_scale x + f_scale gate Norm(f),  u = Norm(y) (1 + mod_scale) + mod_shift; `N8` > 0: u leaves as 8-bit rows
            and goes through a linear layer of N8 outputs
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}
_TINY = 1.1754943508222875e-38  # the smallest normal number in 32 bits: no scale is below it


def _linear(name, M, K, N, epi, dtype, quant):
    return dict(name=name, op="linear", M=M, K=K, N=N, epi=epi, dtype=dtype, quant=quant)


def _norm(name, B, T, D, post, pre, modulated, dtype, N8=0):
    return dict(name=name, op="norm", B=B, T=T, D=D, post=post, pre=pre, modulated=modulated, dtype=dtype, N8=N8)


def listed():
    return [
        # One token through a QKV layer whose rows are in 8 bits already: the smallest call, where latency counts.
        _linear("linear_one_token", 1, 768, 2304, "bias", "bf16", False),
        # One image through the output projection of a base model, from the attention's bf16 output.
        _linear("linear_one_image", 197, 768, 768, "res", "bf16", True),
        # Flattened 14 x 14 x 3 patches to a ragged head in single precision: no size is a multiple of the tiles.
        _linear("linear_ragged", 1003, 588, 1000, "gelu", "f32", True),
        # Second layer of the MLP on eight clips of 1569 tokens: a long inner axis, the residual added.
        _linear("linear_clips_fc2", 12552, 4096, 1024, "res", "bf16", False),
        # First layer of the MLP of a large model on four clips of 4097 tokens, with GELU.
        _linear("linear_clips_fc1", 16388, 1024, 4096, "gelu", "bf16", False),
        # QKV of a base model at batch 256: a short inner axis, mostly output.
        _linear("linear_batch_qkv", 50432, 768, 2304, "bias", "bf16", True),
        # The largest: a wide layer on 32768 tokens.
        _linear("linear_wide", 32768, 4096, 4096, "bias", "bf16", True),
        # Rows of one image, and the hidden activations of four long clips.
        dict(name="quantize_one_image", op="quantize", M=197, K=768, dtype="bf16"),
        dict(name="quantize_clips", op="quantize", M=16388, K=4096, dtype="bf16"),
        # One token, residual scale (a vector) and the next block's LayerNorm: latency.
        _norm("norm_one_token", 1, 1, 768, "none", "layer", False, "bf16"),
        # Four long clips, RMS norms on both sides, gate, scale and shift of their own for each clip, single precision.
        _norm("norm_clips_modulated", 4, 4097, 1024, "rms", "rms", True, "f32"),
        # Batch 256 of a base model into the 8-bit QKV layer of the next block.
        _norm("norm_batch_8bit", 256, 197, 768, "layer", "layer", False, "bf16", N8=2304),
    ]


_MOST = 32768 * 4096 * 4096  # multiply-adds of the largest listed case


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi, odd):
    """A size of the range; most are multiples of 64, as models have them, every fourth is as it falls (`odd`) or a multiple of 8."""
    v = _log(rng, lo, hi)
    if rng.random() < 0.25:
        return max(lo, v if odd else v // 8 * 8)
    return max(64, v // 64 * 64)


def draw(rng):
    op = rng.choice(["linear", "linear", "norm", "quantize"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "linear":
        K, N = _width(rng, 48, 8192, True), _width(rng, 48, 8192, True)
        return dict(op=op, M=_log(rng, 1, min(65536, _MOST // (K * N))), K=K, N=N, epi=rng.choice(["bias", "gelu", "res"]),
                    dtype=dtype, quant=rng.random() < 0.5)
    if op == "quantize":
        return dict(op=op, M=_log(rng, 1, 65536), K=_width(rng, 48, 4096, True), dtype=dtype)
    B, D = _log(rng, 1, 256), _width(rng, 64, 4096, False)
    T = _log(rng, 1, max(1, min(4097, (1 << 26) // (B * D))))
    N8 = _width(rng, 64, 4096, False) if dtype == "bf16" and rng.random() < 0.4 else 0  # 8-bit blocks keep their rows in bf16
    return dict(op=op, B=B, T=T, D=D, post=rng.choice(["none", "layer", "rms"]), pre=rng.choice(["layer", "rms"]),
                modulated=rng.random() < 0.5, dtype=dtype, N8=N8)


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _normal(g, *shape, std=1.0, mean=0.0):
    return torch.randn(*shape, generator=g, device="cuda").mul_(std).add_(mean)


def _tokens(g, rows, width):
    """Rows as an encoder's residual stream has them: magnitudes of their own, a few channels far above the others."""
    x = _normal(g, rows, width)
    x *= torch.exp(_normal(g, rows, 1, std=0.5))
    x *= torch.exp(_normal(g, width, std=0.3))
    return x


def _to_8bit(x, dim):
    """(integers, scales) of the rows (dim 1) or columns (dim 0) of x, in 32 bits."""
    x = x.float()
    scale = (x.abs().amax(dim, keepdim=True) * (1.0 / 127.0)).clamp_min(_TINY)
    return torch.round(x * torch.reciprocal(scale)).to(torch.int8), scale.squeeze(dim)


def _weights(g, K, N, dtype, s):
    w = _normal(g, K, N, std=0.02)
    w *= torch.exp(_normal(g, N, std=0.3))
    s["w"], s["w_scale"] = _to_8bit(w, 0)
    s["bias"] = _normal(g, N, std=0.1).to(_TYPES[dtype])
    if own:
        import paper_2508_00367_amd as rs
        s["packed"] = torch.empty(rs.rs_packed_linear_i8_size(K, N), dtype=torch.uint8, device="cuda")
        rs.rs_pack_linear_i8(s["w"], s["packed"])


def _rows8(M, K):
    """Room for 8-bit rows: 16-byte rows."""
    return torch.empty(M, -(-K // 16) * 16, dtype=torch.int8, device="cuda")[:, :K]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    dt = _TYPES[case["dtype"]]
    s = dict(case=case)
    if case["op"] == "norm":
        B, T, D = case["B"], case["T"], case["D"]
        rows = B * T
        s["x"] = (3 * _tokens(g, rows, D)).to(dt)
        s["f"] = _tokens(g, rows, D).to(dt)
        vec = lambda std, mean: _normal(g, D, std=std, mean=mean).to(dt)  # noqa: E731
        s["post_g"], s["post_b"] = vec(0.1, 1.0), vec(0.1, 0.0)
        s["pre_g"], s["pre_b"] = vec(0.1, 1.0), vec(0.1, 0.0)
        if case["modulated"]:  # the three vectors of an image lie in one row of a [B, 3 D] tensor, as a modulation layer leaves them
            m = _normal(g, B, 3 * D, std=0.3).to(dt)
            s["gate"], s["mod_scale"], s["mod_shift"] = m[:, :D], m[:, D:2 * D], m[:, 2 * D:]
        else:
            s["gate"], s["mod_scale"], s["mod_shift"] = vec(0.2, 0.5), None, None
        s["y"] = torch.empty(rows, D, dtype=dt, device="cuda")
        if case["N8"]:
            _weights(g, D, case["N8"], case["dtype"], s)
            s["u_q"], s["u_scale"] = _rows8(rows, D), torch.empty(rows, device="cuda")
            s["out"] = torch.empty(rows, case["N8"], dtype=dt, device="cuda")
        else:
            s["u"] = torch.empty(rows, D, dtype=dt, device="cuda")
        if own:
            _prepare_norm(s)
        return s
    M, K = case["M"], case["K"]
    s["x"] = _tokens(g, M, K).to(dt)
    s["q"], s["q_scale"] = _rows8(M, K), torch.empty(M, device="cuda")
    if case["op"] == "quantize":
        return s
    N = case["N"]
    if not case["quant"]:
        q, s["q_scale"] = _to_8bit(s.pop("x"), 1)
        s["q"].copy_(q)
    _weights(g, K, N, case["dtype"], s)
    s["res"] = _tokens(g, M, N).to(dt) if case["epi"] == "res" else None
    s["out"] = torch.empty(M, N, dtype=dt, device="cuda")
    return s


_X_SCALE, _F_SCALE, _EPS = 0.9, 1.25, 1e-6


# ---- the framework's calls ------------------------------------------------------------------------------------------
def _prepare_norm(s):
    import paper_2508_00367_amd as rs
    c = s["case"]
    kind = {"none": rs.RS_NORM_NONE, "layer": rs.RS_NORM_LAYER, "rms": rs.RS_NORM_RMS}
    stride = 3 * c["D"] if c["modulated"] else 0
    s["cfg"] = rs.make_residual_norm_cfg(c["B"], c["T"], c["D"], _TYPES[c["dtype"]], post=kind[c["post"]], pre=kind[c["pre"]],
                                         post_eps=_EPS, pre_eps=_EPS, x_scale=_X_SCALE, f_scale=_F_SCALE,
                                         gate_stride=stride, mod_stride=stride)
    rms_b = {"post_b": None if c["post"] == "rms" else s["post_b"], "pre_b": None if c["pre"] == "rms" else s["pre_b"]}
    if c["post"] == "none":
        rms_b["post_b"] = None
    s["vectors"] = rs.make_residual_norm_weights(dict(s, **rms_b, post_g=None if c["post"] == "none" else s["post_g"]))


def _run_own(s):
    import paper_2508_00367_amd as rs
    c = s["case"]
    if c["op"] == "quantize":
        rs.rs_quantize_rows(s["x"], s["q"], s["q_scale"])
        return s["q"], s["q_scale"]
    if c["op"] == "linear":
        if c["quant"]:
            rs.rs_quantize_rows(s["x"], s["q"], s["q_scale"])
        epi = {"bias": rs.RS_EPI_BIAS, "gelu": rs.RS_EPI_BIAS_GELU, "res": rs.RS_EPI_BIAS_RES}[c["epi"]]
        rs.rs_linear_i8_fwd(s["q"], s["q_scale"], s["packed"], s["w_scale"], s["bias"], s["res"], s["out"], epi)
        return s["out"]
    if c["N8"]:
        rs.rs_residual_norm_fwd(s["cfg"], s["vectors"], s["x"], s["f"], s["y"], None, s["u_q"], s["u_scale"])
        rs.rs_linear_i8_fwd(s["u_q"], s["u_scale"], s["packed"], s["w_scale"], s["bias"], None, s["out"], rs.RS_EPI_BIAS)
        return s["y"], s["out"]
    rs.rs_residual_norm_fwd(s["cfg"], s["vectors"], s["x"], s["f"], s["y"], s["u"])
    return s["y"], s["u"]


# ---- plain form -----------------------------------------------------------------------------------------------------
def _plain_product(q, q_scale, s, epi, res):
    out = (q.float() @ s["w"].float()) * (q_scale[:, None] * s["w_scale"][None, :]) + s["bias"].float()
    if epi == "gelu":
        out = 0.5 * out * (1.0 + torch.erf(out * math.sqrt(0.5)))
    if epi == "res":
        out = out + res.float()
    return out.to(s["bias"].dtype)


def _plain_norm(v, kind, g, b):
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    v = v * torch.rsqrt((v * v).mean(1, keepdim=True) + _EPS) * g.float()
    return v + b.float() if kind == "layer" else v


def _per_image(v, c):
    """A vector for all, or one for each image, against rows [B * T, D]."""
    v = v.float()
    return v.repeat_interleave(c["T"], 0) if v.dim() == 2 else v


def run(s):
    if own:
        return _run_own(s)
    c = s["case"]
    if c["op"] == "quantize":
        return _to_8bit(s["x"], 1)
    if c["op"] == "linear":
        q, scale = _to_8bit(s["x"], 1) if c["quant"] else (s["q"], s["q_scale"])
        return _plain_product(q, scale, s, c["epi"], s["res"])
    p = _plain_norm(s["f"].float(), c["post"], s["post_g"], s["post_b"])
    y = _X_SCALE * s["x"].float() + _F_SCALE * (_per_image(s["gate"], c) * p)
    u = _plain_norm(y, c["pre"], s["pre_g"], s["pre_b"])
    if c["modulated"]:
        u = u * (1.0 + _per_image(s["mod_scale"], c)) + _per_image(s["mod_shift"], c)
    if c["N8"]:
        q, scale = _to_8bit(u, 1)
        return y.to(s["x"].dtype), _plain_product(q, scale, s, "bias", None)
    return y.to(s["x"].dtype), u.to(s["x"].dtype)


# ---- 64 bits --------------------------------------------------------------------------------------------------------
def _exact_8bit(x):
    """Scale and integers are defined by roundings to 32 bits (a value next to a border goes one way only by them): each step in 64
    bits, rounded once."""
    once = lambda v: v.float().double()  # noqa: E731
    scale = once(x.abs().max(1).values * once(torch.tensor(1.0 / 127.0))).clamp(min=_TINY)
    return once(once(x) * once(1.0 / scale).unsqueeze(1)).round(), scale


def _exact_product(q, scale, s, epi, res):
    out = torch.nn.functional.linear(q, s["w"].double().t().contiguous())
    out = torch.addcmul(s["bias"].double().expand_as(out), out * scale.unsqueeze(1), s["w_scale"].double().expand_as(out))
    if epi == "gelu":
        out = torch.nn.functional.gelu(out)
    return out + res.double() if epi == "res" else out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantize":
        return None, _exact_8bit(s["x"].double())[1]
    if case["op"] == "linear":
        q, scale = _exact_8bit(s["x"].double()) if case["quant"] else (s["q"].double(), s["q_scale"].double())
        return _exact_product(q, scale, s, case["epi"], s["res"])

    def norm(v, kind, g, b):
        if kind == "layer":
            return torch.nn.functional.layer_norm(v, v.shape[-1:], g.double(), b.double(), _EPS)
        return v / (v.square().sum(-1, keepdim=True) / v.shape[-1] + _EPS).sqrt() * g.double() if kind == "rms" else v

    B, T, D = case["B"], case["T"], case["D"]
    wide = lambda v: v.double().view(-1, 1, D)  # noqa: E731
    f = norm(s["f"].double().view(B, T, D), case["post"], s["post_g"], s["post_b"])
    y = s["x"].double().view(B, T, D) * _X_SCALE + f * wide(s["gate"].contiguous()) * _F_SCALE
    u = norm(y, case["pre"], s["pre_g"], s["pre_b"])
    if case["modulated"]:
        u = u + u * wide(s["mod_scale"].contiguous()) + wide(s["mod_shift"].contiguous())
    y, u = y.view(-1, D), u.reshape(-1, D)
    return (y, _exact_product(*_exact_8bit(u), s, "bias", None)) if case["N8"] else (y, u)


def work(case):
    e = _BYTES[case["dtype"]]
    if case["op"] == "quantize":
        M, K = case["M"], case["K"]
        return {"bytes": M * K * (e + 1) + 4 * M, "flops": 0}
    if case["op"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        rows = M * K * e if case["quant"] else M * (K + 4)
        return {"bytes": rows + K * N + N * (4 + e) + M * N * e * (2 if case["epi"] == "res" else 1), "flops": 2 * M * K * N}
    rows, D, N8 = case["B"] * case["T"], case["D"], case["N8"]
    vectors = (2 + 2 * (case["post"] != "none") + (3 * case["B"] if case["modulated"] else 1)) * D * e
    if N8:
        return {"bytes": 3 * rows * D * e + vectors + D * N8 + N8 * (4 + e) + rows * N8 * e, "flops": 2 * rows * D * N8}
    return {"bytes": 4 * rows * D * e + vectors, "flops": 12 * rows * D}
