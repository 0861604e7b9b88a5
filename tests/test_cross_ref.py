"""The element-wise tolerance of the cross attention, without a GPU: what a bf16
kernel rounds stays inside it, a wrong tile of V does not."""
import pytest
import torch

from cross_ref import reference, tolerance

BF16 = torch.bfloat16


@pytest.mark.parametrize("Lq,S,D", [(64, 6000, 128), (64, 5000, 64), (33, 333, 128)])
def test_a_wrong_tile_is_seen(Lq, S, D):
    g = torch.Generator().manual_seed(S)
    q, k, v = (torch.randn(1, n, 1, D, generator=g).to(BF16) for n in (Lq, S, S))
    live = torch.ones(1, S, dtype=torch.bool)
    want, _, apart = reference(q, k, v, D ** -0.5, live)
    tol = tolerance(BF16, want, apart, float(v.abs().max()))
    # probabilities and output rounded as the kernels round them
    s = (q[0, :, 0].float() @ k[0, :, 0].float().T) * D ** -0.5
    p = torch.exp(s - s[:, :32].max(dim=1, keepdim=True).values)
    out = (p.to(BF16).float() @ v[0, :, 0].float() / p.sum(1, keepdim=True)).to(BF16)
    assert bool(((out.double() - want[0, :, 0]).abs() <= tol[0, :, 0]).all())
    # 32 keys' values left out, and moved by one key
    at = S // 64 * 32
    for tile in (torch.zeros(32, D, dtype=BF16), v[0, at:at + 32, 0].roll(1, 0)):
        w = v.clone()
        w[0, at:at + 32, 0] = tile
        wrong, _, _ = reference(q, k, w, D ** -0.5, live)
        assert float(((wrong - want).abs() > 2 * tol).double().mean()) > 0.001
