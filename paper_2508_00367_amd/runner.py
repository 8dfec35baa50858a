"""Launch sequences: a whole encoder stack (EncoderStack) and a block whose linear layers run in 8 bits (EncoderBlockI8).

EncoderStack: block after block through rs_block_fwd, ping-ponging two
activation buffers, optionally with the batch cut into parts that run on HIP streams of their own.

Argument marshalling and buffer management only: every step of the computation runs inside the
HIP library.  bench.py times `EncoderStack.step`, and the full-depth parity tests run the very same
object (same configurations, buffers and streams) with a `capture` callback between blocks.
"""
from __future__ import annotations

import torch

from . import binding as rs
from .schedule import keep_counts

_OPS = {"mlp": rs.RS_SHIFT_MLP, "attn": rs.RS_SHIFT_ATTN, "block": rs.RS_SHIFT_BLOCK}


class EncoderStack:
    """`wl`: a workload description (B, N, D, H, Dm, blocks, prune, optional n_prefix / op);
    `x0`: device tensor [B, N, D] (bf16); `block_weights[l]`: dict name -> device tensor.

    streams = S > 1 cuts the batch into S nearly equal parts, each with its own workspace, buffers
    and HIP stream: images are independent, the kernels are the same and so are the results."""

    def __init__(self, wl: dict, x0: torch.Tensor, block_weights: list, streams: int = 1, unpruned: bool = False):
        self.B, self.N, self.D, self.H, self.Dm, self.L = wl["B"], wl["N"], wl["D"], wl["H"], wl["Dm"], wl["blocks"]
        self.P = wl.get("n_prefix", 1)
        self.op = _OPS[wl.get("op", "mlp")]
        self.sched = keep_counts(self.N, self.P, self.L, None if unpruned else wl["prune"])
        self.x0 = x0
        self.dtype = x0.dtype
        dev = x0.device
        assert x0.shape == (self.B, self.N, self.D) and len(block_weights) == self.L
        self._keep_alive = []
        self.weights = []
        cfg0 = rs.make_cfg(self.B, self.N, self.D, self.H, self.Dm, self.P, self.N - self.P, self.dtype)
        for w in block_weights:                      # one-off re-layout, outside any timed region
            packed = torch.empty(max(rs.rs_packed_weights_size(cfg0), 16), dtype=torch.uint8, device=dev)
            rs.rs_pack_weights(cfg0, rs.make_weights(w), packed)
            self._keep_alive.append((w, packed))
            self.weights.append(rs.make_weights(w, packed))
        self.gemm_variant = 0            # tile-variant switch of the bf16 GEMMs (0 = chosen by shape)
        # hand row statistics from block to block (same results either way; the fp32 blocks make no use of them)
        self.chain = self.dtype == torch.bfloat16
        self.set_streams(streams)

    def tune(self, candidates=((1, 0), (2, 0), (2, 1)), steps: int = 8, rounds: int = 2):
        """Times a few launch configurations (streams, GEMM tile variant) and keeps the fastest.
        Every configuration computes the same bits (images are independent, the tile variants add
        products and shift sums in one fixed order), so this is a choice of speed only: parts on
        several streams overlap well when every kernel is of one kind (the persistent 256 x 256 GEMM
        everywhere), a single stream gains most from the shape-dependent mix of kernels.
        Returns {(streams, variant): seconds per step}."""
        import time
        seen = {}
        for _ in range(rounds):                      # every candidate `rounds` times, the best time counts
            for S, v in candidates:
                if S > self.B:
                    continue
                self.set_streams(S)
                self.gemm_variant = v
                for _ in range(2):
                    self.step()
                torch.cuda.synchronize()
                t0 = time.perf_counter()
                for _ in range(steps):
                    self.step()
                torch.cuda.synchronize()
                key = (len(self.parts), v)
                seen[key] = min(seen.get(key, 1e30), (time.perf_counter() - t0) / steps)
        (S, v) = min(seen, key=seen.get)
        self.set_streams(S)
        self.gemm_variant = v
        return seen

    def set_streams(self, streams: int) -> None:
        S = max(1, min(int(streams), self.B))
        dev = self.x0.device
        self.parts, first = [], 0
        for i in range(S):
            Bp = self.B // S + (1 if i < self.B % S else 0)
            cfgs = [rs.make_cfg(Bp, n_in, self.D, self.H, self.Dm, self.P, n_keep, self.dtype, op=self.op)
                    for n_in, n_keep in self.sched]
            self.parts.append(dict(
                first=first, B=Bp, x=self.x0[first:first + Bp], cfgs=cfgs,
                ws=torch.empty(max(rs.rs_block_workspace_size(c) for c in cfgs), dtype=torch.uint8, device=dev),
                bufs=[torch.empty((Bp, self.N, self.D), device=dev, dtype=self.dtype) for _ in range(2)],
                kept=torch.empty((Bp, self.N), device=dev, dtype=torch.int32),
                stats=torch.empty((Bp * self.N, 2), device=dev, dtype=torch.float32),
                stream=torch.cuda.Stream() if S > 1 else None))
            first += Bp

    def step(self, capture=None, scores=None):
        """One forward of the stack.  Parts with a stream of their own are enqueued there, a single
        part on the current stream (the capture stream while a HIP graph is recorded).
        capture(l, part, src, dst) is called after block l of a part has been enqueued;
        scores: optional per-part list of float32 [Bp, N] tensors the blocks write their scores to.
        Returns the per-part output tensors (views of the ping-pong buffers, [Bp, K_last, D])."""
        rs.rs_tune_gemm_variant(self.gemm_variant)     # process-wide switch: set on every step
        src = [p["x"] for p in self.parts]
        for l in range(self.L):
            for i, p in enumerate(self.parts):
                stream = p["stream"] if p["stream"] is not None else torch.cuda.current_stream()
                dst = p["bufs"][l & 1]
                # every block but the last leaves the row statistics of its output for the next
                # block's first LayerNorm (written by the gather as it copies the surviving rows)
                rs.rs_block_fwd_chained(p["cfgs"][l], self.weights[l], src[i], p["stats"] if l > 0 and self.chain else None,
                                        dst, p["stats"] if l + 1 < self.L and self.chain else None, p["kept"],
                                        None if scores is None else scores[i], p["ws"], stream)
                if capture is not None:
                    capture(l, p, src[i], dst)
                src[i] = dst
        K = self.P + self.sched[-1][1]
        return [s.view(-1)[:p["B"] * K * self.D].view(p["B"], K, self.D) for s, p in zip(src, self.parts)]


class EncoderBlockI8:
    """One encoder block whose four linear layers run in 8-bit integers, with token pruning behind it: the calls of the library in
    their order, and the buffers between them.  Weights are quantized and packed once, here; activations on their way: the two norms
    in front of the branches write 8-bit rows themselves, the attention's output and the hidden activations are quantized by a call.

        x1   = x_scale x  + f_scale gate1 . Norm_post1(SA(Norm_1(x)))
        xhat = x_scale x1 + f_scale gate2 . Norm_post2(MLP(Norm_2(x1)))
        scores = D(MLP branch, x1);  y = the n_prefix first and the n_keep highest-scoring rows of xhat

    `w`: name -> device tensor: the twelve tensors of rs_block_weights (biases, ln*_g and ln*_b may be missing) and, for encoders that
    have them, post1_g, post1_b, gate1, post2_g, post2_b, gate2, all [D].  `norm`, `post`: RS_NORM_* in front of the
    branches and behind them.  One object serves one stream at a time, the one it was made on or one that has waited for that."""

    def __init__(self, B: int, N: int, D: int, H: int, Dm: int, w: dict, n_prefix: int, n_keep: int, norm=rs.RS_NORM_LAYER,
                 post=rs.RS_NORM_NONE, eps: float = 1e-6, x_scale: float = 1.0, f_scale: float = 1.0, dist=rs.RS_DIST_L2):
        assert D == 64 * H, "heads are 64 wide"
        self.B, self.N, self.D, self.H, self.Dm, self.P, self.n_keep, self.dist = B, N, D, H, Dm, n_prefix, n_keep, dist
        dt, dev = w["w_qkv"].dtype, w["w_qkv"].device
        self.layers = {k: self._pack(w["w_" + k], w.get("b_" + k)) for k in ("qkv", "proj", "fc1", "fc2")}
        cfg = lambda post, pre: rs.make_residual_norm_cfg(B, N, D, dt, post, pre, eps, eps, x_scale, f_scale)  # noqa: E731
        # in front of the attention: no branch yet, x as it is
        self.first = (rs.make_residual_norm_cfg(B, N, D, dt, rs.RS_NORM_NONE, norm, eps, eps),
                      rs.make_residual_norm_weights(dict(pre_g=w.get("ln1_g"), pre_b=w.get("ln1_b"))))
        self.between = (cfg(post, norm), rs.make_residual_norm_weights(dict(
            post_g=w.get("post1_g"), post_b=w.get("post1_b"), gate=w.get("gate1"), pre_g=w.get("ln2_g"), pre_b=w.get("ln2_b"))))
        self.last = (cfg(post, rs.RS_NORM_NONE), rs.make_residual_norm_weights(dict(
            post_g=w.get("post2_g"), post_b=w.get("post2_b"), gate=w.get("gate2"))))
        M = B * N
        new = lambda *s, dtype=dt: torch.empty(*s, dtype=dtype, device=dev)  # noqa: E731
        self.q, self.q_scale = new(M, D, dtype=torch.int8), new(M, dtype=torch.float32)
        self.hq, self.h_scale = new(M, (Dm + 15) // 16 * 16, dtype=torch.int8)[:, :Dm], new(M, dtype=torch.float32)
        self.qkv, self.att, self.hid = new(B, N, 3, H, 64), new(B, N, H, 64), new(M, Dm)
        self.branch, self.x1, self.xhat = new(M, D), new(B, N, D), new(B, N, D)
        self.scores = new(B, N, dtype=torch.float32)
        self.kept = new(B, n_prefix + n_keep, dtype=torch.int32)
        self.y = new(B, n_prefix + n_keep, D)
        self.ws = new(max(rs.rs_shift_topk_workspace_size(B, N, D, dt), 16), dtype=torch.uint8)

    @staticmethod
    def _pack(w: torch.Tensor, bias):
        K, N = w.shape
        q, scale = torch.empty_like(w, dtype=torch.int8), torch.empty(N, dtype=torch.float32, device=w.device)
        rs.rs_quantize_columns(w, q, scale)
        packed = torch.empty(rs.rs_packed_linear_i8_size(K, N), dtype=torch.uint8, device=w.device)
        rs.rs_pack_linear_i8(q, packed)
        return packed, scale, bias

    def _linear(self, name: str, a, a_scale, out, epi=rs.RS_EPI_BIAS) -> None:
        packed, scale, bias = self.layers[name]
        rs.rs_linear_i8_fwd(a, a_scale, packed, scale, bias, None, out, epi)

    def step(self, x: torch.Tensor):
        """x [B, N, D] -> (y [B, n_prefix + n_keep, D], kept_idx, scores [B, N]): buffers of this object, valid until the next step."""
        B, N, D, M = self.B, self.N, self.D, self.B * self.N
        rs.rs_residual_norm_fwd(*self.first, x, None, None, None, self.q, self.q_scale)
        self._linear("qkv", self.q, self.q_scale, self.qkv.view(M, 3 * D))
        rs.rs_attention_fwd(self.qkv[:, :, 0], self.qkv[:, :, 1], self.qkv[:, :, 2], self.att, 0.125)
        rs.rs_quantize_rows(self.att.view(M, D), self.q, self.q_scale)
        self._linear("proj", self.q, self.q_scale, self.branch)
        rs.rs_residual_norm_fwd(*self.between, x, self.branch, self.x1, None, self.q, self.q_scale)
        self._linear("fc1", self.q, self.q_scale, self.hid, rs.RS_EPI_BIAS_GELU)
        rs.rs_quantize_rows(self.hid, self.hq, self.h_scale)
        self._linear("fc2", self.hq, self.h_scale, self.branch)
        rs.rs_residual_norm_fwd(*self.last, self.x1, self.branch, self.xhat, None)
        rs.rs_shift_topk(self.branch.view(B, N, D), self.x1, self.xhat, self.P, self.n_keep, self.scores, self.kept, self.y,
                         self.dist, self.ws)
        return self.y, self.kept, self.scores
