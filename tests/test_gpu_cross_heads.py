"""Cross attention of few rows and many heads or sequences, masked and not."""
import pytest
import torch

from cross_ref import reference, tolerance

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def sampled(B, Lq, S, H, D, masked, at, seed=0):
    """One call of keys and values that all sequences share, against 64 bits at the
    sequences `at`; the queries repeat every 8 sequences, the masks do not."""
    from paper_2607_15650_amd.cross import CrossAttention
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    base = torch.randn(8, Lq, H, D, generator=g, device="cuda").to(BF16)
    q = base.repeat((B + 7) // 8, 1, 1, 1)[:B]
    k, v = (torch.randn(1, S, H, D, generator=g, device="cuda").to(BF16).expand(B, S, H, D) for _ in range(2))
    mask = (torch.rand(B, S, generator=g, device="cuda") < 0.5) if masked else None
    if masked:
        mask[at[1]] = False
    out, lse = CrossAttention(D ** -0.5)(q, k, v, key_mask=mask)
    i = torch.tensor(at, device="cuda")
    n = len(at)
    live = mask[i] if masked else torch.ones(n, S, dtype=torch.bool, device="cuda")
    want, el, apart = reference(q[i], k[:n], v[:n], D ** -0.5, live, "cuda")
    over = (out[i].double().cpu() - want).abs() - tolerance(BF16, want, apart, float(v[0].abs().max()))
    assert float(over.max()) <= 0
    none = torch.isneginf(el)
    got = lse[i].double().cpu()
    assert torch.equal(torch.isneginf(got), none)
    assert bool(((got - el)[~none].abs() <= 1e-5 * (1 + el[~none].abs())).all())


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("B,Lq,S,H,D", [(700, 40, 200, 16, 64), (300, 130, 77, 16, 128), (64, 513, 320, 8, 128),
                                        (40, 1025, 600, 8, 64), (40, 2049, 300, 8, 64)])
def test_few_rows_of_many_heads(gpu_lib, B, Lq, S, H, D, masked):
    sampled(B, Lq, S, H, D, masked, [0, 1, B // 2, B - 1], seed=Lq)


@pytest.mark.parametrize("masked", [False, True])
def test_more_sequences_than_a_grid_is_high(gpu_lib, masked):
    """Beyond 65,535 sequences a masked call lists its keys where it would move them
    together (its workspace says which)."""
    from paper_2607_15650_amd import api
    Lq, S, D = 256, 700, 128

    def need(B, masked):
        return api.cross_attn_workspace_bytes(BF16, B, 1, 1, D, Lq, S, masked)

    most, packed = 65535, 2 * 65535 * S * D * 2
    assert need(most, True) >= packed and need(most + 1, True) < packed // 16 and need(most, False) == 0
    sampled(most + 9, Lq, S, 1, D, masked, [0, 1, most - 1, most, most + 8], seed=5)
