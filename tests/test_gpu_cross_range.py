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


def gap(q, k, scale, live):
    """Of every row: how far the largest score lies above the next, and what
    float32 may be off by in them: 2^-24 of sum |q k| scale for each of D products
    and sums, at most."""
    top, off = [], []
    for h in range(q.shape[2]):
        a, b = q[0, :, h].double(), k[0, live[0], h].double().T.contiguous()
        t = (a @ b * scale).topk(2, dim=1).values
        top.append((t[:, 0] - t[:, 1]).cpu())
        off.append((a.abs() @ b.abs()).max(dim=1).values.cpu() * scale * 2.0 ** -24 * q.shape[3])
    return torch.stack(top), torch.stack(off)


@pytest.mark.parametrize("kind", ["all", "mask"])
@pytest.mark.parametrize("dtype,Lq,S,H,D", FORMS)
def test_large_scores(gpu_lib, dtype, Lq, S, H, D, kind):
    """Scores of 1e8 ... 1e30, in rows beside ordinary ones: the largest takes all."""
    from paper_2607_15650_amd.cross import CrossAttention
    g = torch.Generator(device="cuda")
    g.manual_seed(S + 1)
    k = torch.randn(1, S, H, D, generator=g, device="cuda") * 1e4
    q = torch.randn(1, Lq, H, D, generator=g, device="cuda")
    power = torch.randint(4, 27, (1, Lq, H, 1), generator=g, device="cuda").float()
    power[:, ::5] = -4.0
    q, k = (q * 10.0 ** power).to(dtype), k.to(dtype)
    v = torch.randn(1, S, H, D, generator=g, device="cuda").to(dtype)
    live, kw = masked(kind, S)
    scale = 1.1 * D ** -0.5
    out, lse = (x.double().cpu() for x in CrossAttention(scale)(q, k, v, **kw))
    want, el, apart = reference(q, k, v, scale, live, "cuda")
    assert torch.isfinite(lse).all() and torch.isfinite(out).all()
    # scores off by `off` each, and the float32 scale and its product with log2(e)
    d, off = gap(q, k, scale, live)
    assert bool(((lse - el).abs()[0] <= 1e-5 * (1 + el.abs()[0]) + off + 2.0 ** -21 * el.abs()[0]).all())
    ordinary = (power[0, :, :, 0] < 0).cpu()
    over = ((out - want).abs() - tolerance(dtype, want, apart, float(v.double().abs().max())))[0].amax(-1)
    assert float(over[ordinary].max()) <= 0
    # the largest stays it by 30 at least, and takes all: its value, one product and one rounding
    clear = (d > 2 * off + 30).T & ~ordinary
    assert int(clear.sum()) * 2 >= int((~ordinary).sum())
    one = (out - want).abs()[0] - 2.0 ** (-8 if dtype == BF16 else -22) * want.abs()[0] - 2.0 ** -40
    assert float(one.amax(-1)[clear].max()) <= 0 if bool(clear.any()) else True


# shared heads, sequences of different lengths, and keys in LDS to the last byte of it (listed in the workspace)
@pytest.mark.parametrize("kind", ["lens", "mask"])
@pytest.mark.parametrize("dtype,B,Lq,S,H,Hk,D", [
    (BF16, 2, 1, 3000, 12, 2, 128), (BF16, 3, 7, 100, 8, 4, 64), (BF16, 2, 70, 500, 6, 2, 128), (BF16, 2, 40, 4000, 6, 2, 64),
    (BF16, 2, 2000, 320, 24, 8, 128), (BF16, 2, 4500, 640, 24, 24, 64), (BF16, 2, 1000, 900, 24, 8, 128),
    (BF16, 2, 300, 3000, 12, 4, 64), (F32, 2, 300, 333, 12, 4, 128), (F32, 2, 2, 3000, 12, 4, 64)])
def test_large_scores_and_values(gpu_lib, dtype, B, Lq, S, H, Hk, D, kind):
    """Scores of 1e3 ... 1e30 whose largest is the next one's double at least, over
    values of 1e38: in each row the value of one key, in float32 its product with
    a few plane errors."""
    from paper_2607_15650_amd.cross import CrossAttention
    g = torch.Generator(device="cuda")
    g.manual_seed(S + 1)
    q = torch.zeros(B, Lq, H, D, device="cuda")
    q[..., 5] = 10.0 ** torch.randint(3, 31, (B, Lq, H), generator=g, device="cuda").float()
    q[:, ::2, :, 5] *= -1
    # every key but two between -1/4 and 1/4; the largest is 1, the smallest -1
    k = torch.zeros(B, S, Hk, D, device="cuda")
    k[..., 5] = (torch.rand(B, S, Hk, generator=g, device="cuda") - 0.5) / 2
    lens = torch.tensor([S - 5, S // 2, S][:B], dtype=torch.int32, device="cuda")
    live = torch.arange(S, device="cuda") < lens[:, None]
    if kind == "mask":
        live = live & (torch.arange(S, device="cuda") % 5 != 3)
    for b in range(B):
        at = live[b].nonzero().flatten()
        k[b, at[-2], :, 5], k[b, at[len(at) // 3], :, 5] = 1.0, -1.0
    v = (torch.rand(B, S, Hk, D, generator=g, device="cuda") * 4 - 2) * 1e38
    q, k, v = q.to(dtype), k.to(dtype), v.to(dtype)
    out, lse = (x.double().cpu() for x in CrossAttention(1.3)(
        q, k, v, **({"kv_lens": lens} if kind == "lens" else {"key_mask": live})))
    want, el, _ = reference(q, k, v, 1.3, live, "cuda")
    # scores are one product; the next key's probability is below exp(-1.3 * 1e3 * 3 / 4)
    assert torch.isfinite(out).all()
    assert float(((out - want).abs() - 2.0 ** (-8 if dtype == BF16 else -22) * want.abs()).max()) <= 2e38 * 2.0 ** -22
    assert float(((lse - el).abs() - 2.0 ** -21 * el.abs()).max()) <= 0


@pytest.mark.parametrize("dtype,Lq,S,H,D", FORMS)
def test_an_infinite_value_of_a_repeated_key(gpu_lib, dtype, Lq, S, H, D):
    """One key and value for all places (a stride of 0): what lies past the last
    place of a tile is nothing, not the value again with a weight of 0."""
    from paper_2607_15650_amd.cross import CrossAttention
    g = torch.Generator(device="cuda")
    g.manual_seed(S)
    q, k, v = (torch.randn(1, n, H, D, generator=g, device="cuda").to(dtype) for n in (Lq, 1, 1))
    v[..., 3], v[..., 9] = math.inf, -math.inf
    out, lse = CrossAttention(D ** -0.5)(q, k.expand(1, S, H, D), v.expand(1, S, H, D))
    assert bool((out[..., 3] == math.inf).all()) and bool((out[..., 9] == -math.inf).all())
    rest = torch.ones(D, dtype=torch.bool, device="cuda")
    rest[3] = rest[9] = False
    # equal probabilities, of one rounding: the value, and the output's rounding
    d = (out - v)[..., rest].double().abs() - (2.0 ** (-7 if dtype == BF16 else -20)) * v[..., rest].double().abs()
    assert float(d.max()) <= 2.0 ** -18
    s = (q.double() * k.double()).sum(-1) * D ** -0.5 + math.log(S)
    assert float((lse.double() - s.transpose(1, 2)).abs().max()) <= 1e-4
