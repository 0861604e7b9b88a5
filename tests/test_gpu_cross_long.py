"""Cross attention to the most keys it takes: one key and value, repeated by a
stride of 0."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("less", [0, 12345])
def test_most_keys(gpu_lib, less):
    """The partial states' ranges end at the last key: OUT is the value, LSE the
    score and the log of the number."""
    from paper_2607_15650_amd import api
    S, D = (1 << 31) - (1 << 20), 64
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    q, k, v = (torch.randn(1, 1, 1, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    lens = torch.tensor([S - less], dtype=torch.int32, device="cuda")
    n = api.cross_attn_workspace_bytes(q.dtype, 1, 1, 1, D, 1, S)
    # thousands of ranges, each with a partial state of D + 1 floats
    assert n >= 1000 * 4 * (D + 1)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(1, 1, 1, device="cuda")
    api.cross_attn(q, k.expand(1, S, 1, D), v.expand(1, S, 1, D), 0.125, out, lse, lens if less else None, None, ws)
    s = float((q.double() * k.double()).sum()) * 0.125
    # probabilities of 1 but for the rounding of the maximum; the row sums of 2^31 in float32, in partial sums of some
    # thousand terms: 2^-24 of each, LSE by its own rounding
    assert abs(float(lse) - (s + math.log(S - less))) <= 1e-4
    # one probability's rounding, and the output's
    assert float(((out - v).double().abs() - (2.0 ** -7 + 2.0 ** -14) * v.double().abs()).max()) <= 0
