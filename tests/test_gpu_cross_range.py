"""Cross attention at the ends of the value range, in every kernel of it, against
64 bits: finite inputs whose attention is finite give finite results."""
import math

import pytest
import torch

from cross_ref import reference, tolerance

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32

# one token, whole and in ranges of keys; few rows; 128-row workgroups, whole and in ranges; a head's keys in LDS;
# tasks, whole and in ranges.  In float32 the forms of 32, 128 and 256 rows.
FORMS = [(BF16, 1, 200, 2, 128), (BF16, 1, 5000, 2, 64), (BF16, 20, 333, 4, 64), (BF16, 200, 333, 2, 128),
         (BF16, 200, 333, 2, 64), (BF16, 70, 3000, 2, 64), (BF16, 4500, 200, 48, 128), (BF16, 6000, 200, 36, 64),
         (BF16, 2500, 900, 24, 128), (BF16, 3000, 900, 24, 64), (BF16, 700, 3000, 8, 128), (BF16, 500, 5000, 8, 64),
         (F32, 1, 200, 2, 128), (F32, 3, 5000, 2, 64), (F32, 1047, 333, 12, 128), (F32, 2500, 130, 24, 128),
         (F32, 1500, 97, 24, 64)]


def masked(kind, S):
    """Which keys are live, and the argument that says so."""
    live = torch.ones(1, S, dtype=torch.bool, device="cuda")
    if kind == "mask":
        live[:, 1::7] = False
        return live, {"key_mask": live}
    return live, {}


def check(got, q, k, v, scale, live, lse_tol=0.0):
    out, lse = (x.double().cpu() for x in got)
    want, el, apart = reference(q, k, v, scale, live, "cuda")
    assert torch.isfinite(want).all() and torch.isfinite(el).all()
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    top = float(v.double().abs().max())
    over = (out - want).abs() - tolerance(q.dtype, want, apart, top)
    assert float(over.max()) <= 0, float(over.max()) / top
    assert bool(((lse - el).abs() <= 1e-5 * (1 + el.abs()) + lse_tol * el.abs()).all())


@pytest.mark.parametrize("kind", ["all", "mask"])
@pytest.mark.parametrize("dtype,Lq,S,H,D", FORMS)
def test_large_values(gpu_lib, dtype, Lq, S, H, D, kind):
    """Values of 2^100 under a score far above those of the first keys, in some
    rows and not in others."""
    from paper_2607_15650_amd.cross import CrossAttention
    g = torch.Generator(device="cuda")
    g.manual_seed(S)
    q = torch.zeros(1, Lq, H, D, device="cuda")
    q[..., 0] = torch.where(torch.arange(Lq, device="cuda") % 3 == 1, 0.0, 1.0)[None, :, None]
    k = torch.zeros(1, S, H, D, device="cuda")
    k[:, S * 3 // 4 // 7 * 7, :, 0] = 38.0
    k[:, S // 2 // 7 * 7, :, 0] = 37.0
    v = (torch.rand(1, S, H, D, generator=g, device="cuda") + 0.5) * 2.0 ** 100
    q, k, v = q.to(dtype), k.to(dtype), v.to(dtype)
    live, kw = masked(kind, S)
    check(CrossAttention(math.log(2.0))(q, k, v, **kw), q, k, v, math.log(2.0), live)


@pytest.mark.parametrize("kind", ["all", "mask"])
@pytest.mark.parametrize("dtype,Lq,S,H,D", FORMS)
def test_values_near_the_largest(gpu_lib, dtype, Lq, S, H, D, kind):
    """Means of values of 3e38, of one sign and of both."""
    from paper_2607_15650_amd.cross import CrossAttention
    g = torch.Generator(device="cuda")
    g.manual_seed(S)
    q = torch.randn(1, Lq, H, D, generator=g, device="cuda").to(dtype)
    k = (torch.randn(1, S, H, D, generator=g, device="cuda") * 0.1).to(dtype)
    v = torch.full((1, S, H, D), 3e38, device="cuda")
    v[..., 1::2] *= torch.where(torch.rand(1, S, H, D // 2, generator=g, device="cuda") < 0.5, -1.0, 1.0)
    v = v.to(dtype)
    live, kw = masked(kind, S)
    check(CrossAttention(D ** -0.5)(q, k, v, **kw), q, k, v, D ** -0.5, live)
