"""Cross attention of sequences without a live key: OUT is 0 and LSE -inf in
every row, whatever the queries hold, and beside them the rows of the other
sequences are theirs."""
import math

import pytest
import torch

from test_gpu_cross import exact, make

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32

# one token, whole and in ranges of keys; few rows; 128-row workgroups, whole and in ranges; a head's keys in LDS;
# tasks, whole and in ranges
SHAPES = [(1, 200, 2, 128), (1, 5000, 2, 64), (20, 333, 4, 128), (200, 333, 2, 128), (70, 3000, 2, 64),
          (4500, 200, 24, 128), (3000, 640, 24, 64), (2500, 900, 12, 128), (700, 3000, 4, 128), (500, 5000, 4, 64)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["lens", "mask"])
@pytest.mark.parametrize("Lq,S,H,D", SHAPES)
def test_queries_that_are_not_numbers(gpu_lib, Lq, S, H, D, kind, dtype):
    from paper_2607_15650_amd.cross import CrossAttention
    B, lens = 3, [0, S - 3, 0]
    q, k, v = make(B, Lq, S, H, H, D, dtype, seed=Lq + S)
    t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    live = torch.arange(S, device="cuda") < t[:, None]
    clean = q.clone()
    # in both sequences without keys and in the other one
    for b in range(B):
        q[b, 0, 0, 3] = math.nan
        q[b, Lq // 2, H - 1, 0] = math.inf
        q[b, Lq - 1, H // 2] = -math.inf
    out, lse = CrossAttention(D ** -0.5)(q, k, v, **({"kv_lens": t} if kind == "lens" else {"key_mask": live}))
    for b in (0, 2):
        assert not out[b].isnan().any() and not out[b].any()
        assert torch.isneginf(lse[b]).all()
    eo, el = exact(clean[1:2], k[1:2], v[1:2], D ** -0.5, live[1:2], "cuda")
    rows = torch.isfinite(q[1].double().sum(-1)).cpu()                 # [Lq, H]
    vm = float(v[1][live[1]].abs().max())
    tol = (2.0 ** -7 + 2.0 ** -17) * vm if dtype == BF16 else 1e-5 * vm
    d = (out[1].double().cpu() - eo[0]).abs()[rows]
    assert d.numel() == 0 or float(d.max()) <= tol
    assert bool(out[1].cpu()[~rows].isnan().all(-1).all())
    e = (lse[1].double().cpu() - el[0]).abs()[rows.T]
    assert e.numel() == 0 or bool((e <= 1e-5 * (1 + el[0][rows.T].abs())).all())
