"""Cross attention against 64 bits, element by element: within the rounding of the
probabilities and of the output (cross_ref.tolerance), which a wrong row of V
passes at any number of keys (test_cross_ref.py shows it)."""
import pytest
import torch

from cross_ref import reference, tolerance
from test_gpu_cross import SHAPES, make, poison

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def check(got, q, k, v, live):
    out, lse = (x.double().cpu() for x in got)
    top = float(v[live].abs().max()) if bool(live.any()) else 0.0
    v = torch.where(live[:, :, None, None], v, 0)
    want, el, apart = reference(q, k, v, q.shape[-1] ** -0.5, live, "cuda")
    over = (out - want).abs() - tolerance(q.dtype, want, apart, top)
    assert float(over.max()) <= 0, float(over.max())
    none = torch.isneginf(el)
    assert torch.equal(torch.isneginf(lse), none)
    assert bool(((lse - el)[~none].abs() <= 1e-5 * (1 + el[~none].abs())).all())


# those of test_gpu_cross.py, and more: many rows over few and many keys, key ranges, thousands of keys
MORE = [(2, 4500, 77, 24, 24, 128), (1, 6000, 200, 36, 36, 64), (2, 3000, 640, 40, 20, 64), (2, 2100, 333, 12, 12, 128),
        (3, 1000, 1100, 24, 8, 64), (3, 700, 2050, 20, 20, 128), (2, 300, 6000, 6, 2, 128), (2, 500, 5000, 8, 8, 64),
        (2, 1, 16384, 6, 2, 128)]


@pytest.mark.parametrize("kind", ["all", "lens", "mask"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,Lq,S,H,Hk,D", SHAPES + MORE)
def test_elements(gpu_lib, B, Lq, S, H, Hk, D, dtype, kind):
    from paper_2607_15650_amd.cross import CrossAttention
    q, k, v = make(B, Lq, S, H, Hk, D, dtype, seed=Lq + S, packed=kind == "lens")
    live, kw = torch.ones(B, S, dtype=torch.bool, device="cuda"), {}
    if kind == "lens":
        lens = torch.tensor([S, S // 2 + 1, 0][:B], dtype=torch.int32, device="cuda")
        live, kw = torch.arange(S, device="cuda") < lens[:, None], {"kv_lens": lens}
    elif kind == "mask":
        g = torch.Generator(device="cuda")
        g.manual_seed(S)
        live = torch.rand(B, S, generator=g, device="cuda") < 0.6
        kw = {"key_mask": live}
    k, v = poison(k, v, live)
    check(CrossAttention(D ** -0.5)(q, k, v, **kw), q, k, v, live)


@pytest.mark.parametrize("kind", ["all", "mask"])
@pytest.mark.parametrize("B,Lq,S,H,Hk,D", [(1, 1, 77, 12, 12, 128), (2, 1, 4099, 8, 2, 64), (1, 1, 16384, 6, 2, 128),
                                           (2, 8, 700, 8, 2, 64), (1, 32, 3000, 4, 4, 128)])
def test_few_rows_round_once(gpu_lib, B, Lq, S, H, Hk, D, kind):
    """Up to 32 rows of a key/value head: the probabilities are two bf16 planes, so
    what is left is the output's rounding (2^-8), that of the second plane (2^-16 of
    a probability) and float32's (2^-16 of the probabilities at scores of order 10,
    2^-18 of the largest value for the sums)."""
    from paper_2607_15650_amd.cross import CrossAttention
    q, k, v = make(B, Lq, S, H, Hk, D, BF16, seed=Lq + S)
    live, kw = torch.ones(B, S, dtype=torch.bool, device="cuda"), {}
    if kind == "mask":
        live = torch.arange(S, device="cuda").expand(B, S) % 3 != 1
        kw = {"key_mask": live.contiguous()}
    out, _ = CrossAttention(D ** -0.5)(q, k, v, **kw)
    want, _, apart = reference(q, k, v, D ** -0.5, live, "cuda")
    tol = 2.0 ** -8 * want.abs() + 2.0 ** -15 * apart + 2.0 ** -18 * float(v.abs().max())
    over = (out.double().cpu() - want).abs() - tol
    assert float(over.max()) <= 0, float(over.max())
