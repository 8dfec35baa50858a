"""A row through rs_residual_norm_fwd is the same bits in a batch of any size, though rows are given more lanes where there are few."""
import sys

import pytest
import torch

import paper_2508_00367_amd as rs
from i8_testlib import DT
from test_gpu_residual_norm import KIND, make

pytestmark = pytest.mark.gpu


def _run(x, f, v, post, pre, dtype):
    B, N, D = x.shape
    cfg = rs.make_residual_norm_cfg(B, N, D, DT[dtype], KIND[post], KIND[pre], 1e-6, 1e-5, 0.75, 1.5)
    y, u = torch.empty_like(x), torch.empty_like(x)
    q, s = torch.empty(N, (D + 15) // 16 * 16, dtype=torch.int8, device="cuda"), torch.empty(N, device="cuda")
    rs.rs_residual_norm_fwd(cfg, rs.make_residual_norm_weights(v), x, f, y, u, q[:, :D], s)
    return y[0], u[0], q, s


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("post,pre", [("layer", "layer"), ("rms", "rms")])
@pytest.mark.parametrize("D", [8, 64, 120, 128, 136, 192, 256, 264, 384, 512, 520, 768, 776, 1000, 1024, 1032, 1536, 2048, 2056, 4096])
def test_a_row_is_the_same_in_any_batch(D, post, pre, dtype):
    """On both sides of every number of rows at which the lanes change (16, 8 and 4 rows a compute unit)."""
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    most = 16 * cus + 1
    print("batches", D, post, dtype, flush=True)
    x, f, v, _ = make(1, most, D, dtype, False, seed=D, offset=0.5)
    if post == "rms":
        v["post_b"] = v["pre_b"] = None
    want = _run(x, f, v, post, pre, dtype)
    for rows in (1, 7, 4 * cus, 4 * cus + 1, 8 * cus, 8 * cus + 1, 16 * cus):
        got = _run(x[:, most - rows:].clone(), f[:, most - rows:].clone(), v, post, pre, dtype)
        for name, g, w in zip(("y", "u", "q", "scale"), got, want):
            assert torch.equal(g, w[most - rows:]), (name, rows)
