"""Cross attention (ditango_cross_attn) against attention in 64 bits.

Tolerances.  bf16: the probabilities and the output are rounded to bf16, each
by at most 2^-8 of its value, so |out - exact| <= 2^-8 sum p|v| / sum p + 2^-8
|exact| + float32 accumulation, taken as 2^-18 of max|v|; bounded below by
(2^-7 + 2^-17) max|v| over the live keys of the head.  float32: products off by
2^-24 |x y| each (three planes) plus accumulation: scores off by at most
2^-23 * 8 * |q||k| scale (8 for the sums' growth) move a probability by that
much, twice over (numerator and row sum); the test's scores are of order 5, so
2^-23 * 8 * 5 * 2 < 1e-5 of max|v|.  LSE: off by as much as the scores, and by
the float32 rounding of its value and of exp2/log2 (2^-21 of a score of order
32): 1e-5 * (1 + |lse|).
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def exact(q, k, v, scale, live, device="cpu"):
    """q [B, L, H, D], k, v [B, S, Hk, D], live bool [B, S] -> OUT, LSE in 64 bits."""
    q, k, v = (x.double().to(device) for x in (q, k, v))
    B, L, H, D = q.shape
    G = H // k.shape[2]
    out = torch.zeros(B, L, H, D, dtype=torch.float64, device=device)
    lse = torch.full((B, H, L), -math.inf, dtype=torch.float64, device=device)
    for b in range(B):
        at = live[b].to(device).nonzero().flatten()
        if at.numel() == 0:
            continue
        for h in range(H):
            s = q[b, :, h] @ k[b, at, h // G].T.contiguous() * scale
            lse[b, h] = torch.logsumexp(s, 1)
            out[b, :, h] = torch.softmax(s, 1) @ v[b, at, h // G]
    return out.cpu(), lse.cpu()


def check(got, q, k, v, scale, live, device="cpu"):
    out, lse = (x.double().cpu() for x in got)
    eo, el = exact(q, k, v, scale, live, device)
    lv = v.double().cpu()[live.cpu()]
    vm = float(lv.abs().max()) if lv.numel() else 0.0
    tol = (2.0 ** -7 + 2.0 ** -17) * vm if q.dtype == BF16 else 1e-5 * vm
    assert torch.isfinite(out).all()
    err = float((out - eo).abs().max())
    assert err <= tol, (err, tol)
    none = torch.isneginf(el)
    assert torch.equal(torch.isneginf(lse), none)
    d = (lse - el)[~none].abs()
    assert d.numel() == 0 or bool((d <= 1e-5 * (1 + el[~none].abs())).all()), float(d.max())


def make(B, Lq, S, H, Hk, D, dtype, seed=0, packed=False):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)   # noqa: E731
    q = r(B, Lq, H, D)
    if packed:
        kv = r(B, S, 2 * Hk, D)
        return q, kv[:, :, :Hk], kv[:, :, Hk:]
    return q, r(B, S, Hk, D), r(B, S, Hk, D)


def poison(k, v, live):
    """NaN, infinities and the types' lowest values where no key is live."""
    bad = torch.tensor([math.nan, math.inf, -math.inf, torch.finfo(k.dtype).min], device="cuda").to(k.dtype)
    fill = bad[torch.arange(k.shape[1], device="cuda") % 4][None, :, None, None]
    at = ~live[:, :, None, None]
    return torch.where(at, fill, k), torch.where(at, fill, v)


# B, q_len, kv_len, H, Hk, D: one token to a block, one key to thousands, tile edges, shared heads
SHAPES = [
    (1, 1, 1, 1, 1, 128), (1, 1, 77, 12, 12, 128), (2, 1, 4099, 8, 2, 64), (3, 1, 1000, 6, 1, 128),
    (1, 2, 63, 4, 4, 64), (2, 17, 64, 8, 4, 128), (1, 33, 65, 3, 3, 64), (1, 127, 128, 5, 5, 128),
    (2, 128, 129, 4, 1, 64), (1, 129, 31, 2, 2, 128), (1, 300, 512, 6, 3, 128), (1, 515, 333, 4, 4, 64),
    (1, 1000, 700, 2, 2, 128), (2, 257, 1500, 3, 1, 64), (1, 70, 3000, 2, 2, 128), (1, 5, 9000, 16, 2, 64),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(gpu_lib, shape, dtype):
    from paper_2607_15650_amd.cross import CrossAttention
    B, Lq, S, H, Hk, D = shape
    q, k, v = make(B, Lq, S, H, Hk, D, dtype, seed=Lq + S)
    scale = D ** -0.5
    check(CrossAttention(scale)(q, k, v), q, k, v, scale, torch.ones(B, S, dtype=torch.bool, device="cuda"))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Lq,S", [(1, 200), (1, 5000), (40, 200), (300, 700), (600, 130)])
def test_lengths(gpu_lib, dtype, D, Lq, S):
    """Prefixes from nothing to all, out of range ones clamped; what lies behind is never used."""
    from paper_2607_15650_amd.cross import CrossAttention
    lens = [0, 1, S, 64, S // 2 + 1, -5, S + 9]
    B, H, Hk = len(lens), 4, 2
    q, k, v = make(B, Lq, S, H, Hk, D, dtype, seed=3, packed=True)
    live = torch.tensor([[c < n for c in range(S)] for n in lens], device="cuda")
    k, v = poison(k, v, live)
    t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    check(CrossAttention(D ** -0.5)(q, k, v, kv_lens=t), q, k, v, D ** -0.5, live)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Lq,S", [(1, 100), (1, 5000), (20, 333), (300, 333), (400, 2100)])
@pytest.mark.parametrize("kind", [torch.bool, torch.uint8])
def test_masks(gpu_lib, dtype, D, Lq, S, kind):
    """Random masks, one key, the last key, none, and a mask together with lengths."""
    from paper_2607_15650_amd.cross import CrossAttention
    B, H, Hk = 5, 4, 4
    q, k, v = make(B, Lq, S, H, Hk, D, dtype, seed=5)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    mask = torch.rand((B, S), generator=g, device="cuda") < 0.5
    mask[1] = False
    mask[1, 7] = True
    mask[2] = False
    mask[2, S - 1] = True
    mask[3] = False
    given = mask if kind == torch.bool else mask.to(torch.uint8) * 3
    op = CrossAttention(D ** -0.5)
    kp, vp = poison(k, v, mask)
    check(op(q, kp, vp, key_mask=given), q, kp, vp, D ** -0.5, mask)
    lens = torch.tensor([S // 2, S, S - 1, S, 0], dtype=torch.int32, device="cuda")
    both = mask & (torch.arange(S, device="cuda") < lens[:, None])
    kp, vp = poison(k, v, both)
    check(op(q, kp, vp, kv_lens=lens, key_mask=given), q, kp, vp, D ** -0.5, both)


# many rows: few keys (kept in LDS), more (streamed), many (tasks one after another, whole or in key ranges)
@pytest.mark.parametrize("kind", ["all", "lens", "mask"])
@pytest.mark.parametrize("B,Lq,S,H,Hk,D", [
    (2, 4500, 77, 24, 24, 128), (3, 2600, 320, 30, 10, 128), (1, 6000, 200, 36, 36, 64), (2, 3000, 640, 40, 20, 64),
    (2, 2100, 333, 12, 12, 128), (2, 900, 513, 24, 24, 128), (3, 1000, 1100, 24, 8, 64), (3, 700, 2050, 20, 20, 128),
    (2, 300, 6000, 6, 2, 128), (2, 500, 5000, 8, 8, 64),
])
def test_many_rows(gpu_lib, B, Lq, S, H, Hk, D, kind):
    from paper_2607_15650_amd.cross import CrossAttention
    q, k, v = make(B, Lq, S, H, Hk, D, BF16, seed=Lq, packed=kind == "lens")
    live = torch.ones(B, S, dtype=torch.bool, device="cuda")
    kw = {}
    if kind == "lens":
        lens = torch.tensor([S // 2 + 1, 0, S][:B], dtype=torch.int32, device="cuda")
        live, kw = torch.arange(S, device="cuda") < lens[:, None], {"kv_lens": lens}
    elif kind == "mask":
        live = torch.rand(B, S, device="cuda") < 0.6
        live[0] = False
        live[0, S // 3] = True
        kw = {"key_mask": live}
    k, v = poison(k, v, live)
    check(CrossAttention(D ** -0.5)(q, k, v, **kw), q, k, v, D ** -0.5, live, "cuda")


@pytest.mark.parametrize("kind", ["all", "lens", "mask"])
@pytest.mark.parametrize("B,Lq,S,H,Hk,D", [(2, 1047, 333, 12, 12, 128), (2, 2500, 130, 24, 12, 128), (2, 1500, 97, 24, 24, 64)])
def test_many_rows_f32(gpu_lib, B, Lq, S, H, Hk, D, kind):
    from paper_2607_15650_amd.cross import CrossAttention
    q, k, v = make(B, Lq, S, H, Hk, D, F32, seed=Lq, packed=True)
    live = torch.ones(B, S, dtype=torch.bool, device="cuda")
    kw = {}
    if kind == "lens":
        lens = torch.tensor([S - 32, 0], dtype=torch.int32, device="cuda")
        live, kw = torch.arange(S, device="cuda") < lens[:, None], {"kv_lens": lens}
    elif kind == "mask":
        live = torch.rand(B, S, device="cuda") < 0.6
        kw = {"key_mask": live}
    k, v = poison(k, v, live)
    q[0, 7] *= 1e-36                       # values that the planes do not hold
    check(CrossAttention(D ** -0.5)(q, k, v, **kw), q, k, v, D ** -0.5, live, "cuda")


@pytest.mark.parametrize("B,Lq,S,H,D", [(1, 9000, 100, 24, 128), (1, 13000, 300, 16, 64), (1, 2500, 900, 12, 128),
                                        (1, 700, 3000, 8, 128), (1, 700, 3000, 8, 64), (1, 200, 400, 4, 128)])
def test_many_rows_of_rising_scores(gpu_lib, B, Lq, S, H, D):
    """The maximum of the first keys does not hold for the later ones, in some rows: they are raised or run again."""
    from paper_2607_15650_amd.cross import CrossAttention
    q, k, v = make(B, Lq, S, H, H, D, BF16, seed=11)
    q[:, ::3] = q[:, ::3].abs()
    ramp = (torch.arange(S, device="cuda").float() * (64 / S))[None, :, None, None].expand(B, S, H, D)
    k = ramp.to(BF16).contiguous()
    live = torch.ones(B, S, dtype=torch.bool, device="cuda")
    out, lse = CrossAttention(0.125)(q, k, v)
    eo, el = exact(q, k, v, 0.125, live, "cuda")
    # scores up to 64 * sum|q| / 8 < 64 * 128 / 8 = 1024: off by 2^-24 * 1024 * 8 (growth of the sums) < 5e-4
    assert float((lse.double().cpu() - el).abs().max()) <= 5e-4
    assert float((out.double().cpu() - eo).abs().max()) <= (2 ** -7 + 1e-3) * float(v.abs().max())
    # and a row whose scores are not numbers stays alone
    q[0, 5, 1, 3] = float("nan")
    again = CrossAttention(0.125)(q, k, v)
    same = torch.ones(Lq, dtype=torch.bool, device="cuda")
    same[5] = False
    assert torch.isnan(again[0][0, 5, 1]).all() and torch.isnan(again[1][0, 1, 5])
    assert float((again[0][:, same].double().cpu() - eo[:, same.cpu()]).abs().max()) <= (2 ** -7 + 1e-3) * float(v.abs().max())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq", [1, 200])
def test_no_keys(gpu_lib, dtype, Lq):
    from paper_2607_15650_amd.cross import CrossAttention
    q, k, v = make(2, Lq, 0, 4, 2, 64, dtype)
    for mask in (None, torch.zeros(2, 0, dtype=torch.bool, device="cuda")):
        out, lse = CrossAttention(0.125)(q, k, v, key_mask=mask)
        assert not out.any() and torch.isneginf(lse).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq", [1, 150])
def test_strides(gpu_lib, dtype, Lq):
    """Head-major and packed layouts, a sequence shared by the batch, and rows that are copied first."""
    from paper_2607_15650_amd.cross import CrossAttention
    B, S, H, Hk, D = 3, 140, 4, 2, 64
    q, k, v = make(B, Lq, S, H, Hk, D, dtype, seed=8)
    op, scale = CrossAttention(D ** -0.5), D ** -0.5
    live = torch.ones(B, S, dtype=torch.bool, device="cuda")
    major = lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)   # noqa: E731
    check(op(major(q), major(k), major(v)), q, k, v, scale, live)
    wide = torch.randn(B, S, Hk, D + 8, device="cuda").to(dtype)
    check(op(q, wide[..., :D], wide[..., 8:]), q, wide[..., :D], wide[..., 8:], scale, live)
    one = k[:1].expand(B, -1, -1, -1)
    check(op(q, one, v), q, one, v, scale, live)
    odd = torch.randn(B, S, Hk, D + 1, device="cuda").to(dtype)
    check(op(q, odd[..., 1:], odd[..., :D]), q, odd[..., 1:], odd[..., :D], scale, live)
    flat = torch.randn(B * Lq * H * D + 1, device="cuda").to(dtype)
    q1 = flat[1:].view(B, Lq, H, D)
    check(op(q1, k, v), q1, k, v, scale, live)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq", [1, 200])
def test_scores_of_any_size(gpu_lib, dtype, Lq):
    """Scores that rise far along the keys (the running maximum is raised again
    and again), and ones of thousands, where one key takes all."""
    from paper_2607_15650_amd.cross import CrossAttention
    B, S, H, D = 1, 700, 2, 64
    q, k, v = make(B, Lq, S, H, H, D, dtype, seed=2)
    live = torch.ones(B, S, dtype=torch.bool, device="cuda")
    q = q.abs()
    ramp = (torch.arange(S, device="cuda").float() / 8)[None, :, None, None].expand(B, S, H, D).to(dtype).contiguous()
    # scores of up to 87 * sum|q| * scale = 560: float32 holds them to 2^-24 * 560 * growth of the sums (8), which
    # moves neighbours (scores 0.8 apart at least) by 5e-4 of their weight: LSE by 5e-4, OUT by 1e-3 max|v|
    out, lse = CrossAttention(0.125)(q, ramp, v)
    eo, el = exact(q, ramp, v, 0.125, live)
    vm = float(v.abs().max())
    assert float((lse.double().cpu() - el).abs().max()) <= 5e-4
    assert float((out.double().cpu() - eo).abs().max()) <= ((2 ** -7 + 1e-3) if dtype == BF16 else 1e-3) * vm
    down = ramp.flip(1).contiguous()
    out, lse = CrossAttention(0.125)(q, down, v)
    eo, el = exact(q, down, v, 0.125, live)
    assert float((lse.double().cpu() - el).abs().max()) <= 5e-4
    assert float((out.double().cpu() - eo).abs().max()) <= ((2 ** -7 + 1e-3) if dtype == BF16 else 1e-3) * vm


# the kernels for a token, for few rows, for a head's keys in LDS and for many rows and keys
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Lq,S,H", [(1, 200, 2), (1, 5000, 2), (200, 333, 2), (4500, 200, 48), (2500, 900, 24)])
def test_scores_of_minus_infinity(gpu_lib, dtype, D, Lq, S, H):
    """Keys whose every score is -inf, the first of all among them, weigh nothing beside others."""
    from paper_2607_15650_amd.cross import CrossAttention
    q, k, v = make(1, Lq, S, H, H, D, dtype, seed=8)
    q[..., 0] = q[..., 0].abs() + 0.125
    live = torch.ones(1, S, dtype=torch.bool, device="cuda")
    live[:, :170] = False
    live[:, 180:190] = False
    k[..., 0] = torch.where(live[:, :, None], k[..., 0], -math.inf)
    # (exponents far below the others' too: nothing else may stand for the maximum)
    q[..., 1] = q[..., 1].abs() + 0.125
    k[..., 1] = -200.0
    out, lse = CrossAttention(D ** -0.5)(q, k, v)
    eo, el = exact(q, k, v, D ** -0.5, live, "cuda")
    vm = float(v.abs().max())
    # scores of up to 100, off by 2^-24 * 8 of that
    assert float((lse.double().cpu() - el).abs().max()) <= 1e-4
    assert float((out.double().cpu() - eo).abs().max()) <= ((2 ** -7 + 2e-4) if dtype == BF16 else 2e-4) * vm


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq,H,far", [(1, 2, False), (150, 2, False), (150, 2, True), (4500, 48, False)])
@pytest.mark.parametrize("masked", [False, True])
def test_rows_far_apart(gpu_lib, dtype, Lq, H, far, masked):
    """Offsets past 2^31 elements: keys and values, and the queries, as columns of wide rows."""
    from paper_2607_15650_amd import api
    S, D, wide = 270, 64, 1 << 23

    def column(n, at, wide):
        x = torch.as_strided(buf, (1, n, H, D), (0, wide, D, 1), at)
        x.copy_(torch.randn(x.shape, device="cuda"))
        return x

    buf = torch.empty(S * wide, dtype=dtype, device="cuda")
    k, v = column(S, 0, wide), column(S, H * D, wide)
    if far:
        q = column(Lq, 2 * H * D, wide)
    else:
        q = torch.randn(1, Lq, H, D, device="cuda").to(dtype)
    mask = (torch.rand(1, S, device="cuda") < 0.6) if masked else None
    live = mask if masked else torch.ones(1, S, dtype=torch.bool, device="cuda")
    ws = torch.empty(api.cross_attn_workspace_bytes(dtype, 1, H, H, D, Lq, S, masked), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty(1, Lq, H, D, dtype=dtype, device="cuda"), torch.empty(1, H, Lq, device="cuda")
    api.cross_attn(q, k, v, 0.125, out, lse, None, mask, ws)
    check((out, lse), q, k, v, 0.125, live, "cuda")


@pytest.mark.parametrize("masked", [False, True])
def test_many_sequences(gpu_lib, masked):
    """More sequences than a grid's second dimension holds; more threads than a launch has are refused."""
    from paper_2607_15650_amd import _lib, api
    from paper_2607_15650_amd.cross import CrossAttention
    B, Lq, S, D = 66000, 40, 600, 64
    q, (k, v) = torch.randn(B, Lq, 1, D, device="cuda").to(BF16), torch.randn(2, 1, S, 1, D, device="cuda").to(BF16)
    mask = (torch.rand(B, S, device="cuda") < 0.5) if masked else None
    out, lse = CrossAttention(0.125)(q, k.expand(B, S, 1, D), v.expand(B, S, 1, D), key_mask=mask)
    at = torch.tensor([0, 1, 65534, 65535, 65536, B - 1], device="cuda")
    live = mask[at] if masked else torch.ones(6, S, dtype=torch.bool, device="cuda")
    check((out[at], lse[at]), q[at], k.expand(6, S, 1, D), v.expand(6, S, 1, D), 0.125, live)
    B = 1 << 24
    q = torch.zeros(1, 1, 1, D, dtype=BF16, device="cuda").expand(B, 1, 1, D)
    with pytest.raises(_lib.DitangoError):
        api.cross_attn(q, q, q, 0.125, torch.empty(B, 1, 1, D, dtype=BF16, device="cuda"))


def test_composes_with_other_states(gpu_lib):
    """A state like the partitions': the halves of the keys, composed, are the whole."""
    from paper_2607_15650_amd import api
    B, Lq, S, H, D = 2, 200, 300, 4, 128
    q, k, v = make(B, Lq, S, H, H, D, BF16, seed=4)
    outs = torch.empty(2, B, Lq, H, D, device="cuda", dtype=BF16)
    lses = torch.empty(2, B, H, Lq, device="cuda")
    api.cross_attn(q, k[:, :130], v[:, :130], 0.09, outs[0], lses[0])
    api.cross_attn(q, k[:, 130:], v[:, 130:], 0.09, outs[1], lses[1])
    out, lse = torch.empty_like(outs[0]), torch.empty_like(lses[0])
    api.merge_states(outs, lses, out, lse)
    live = torch.ones(B, S, dtype=torch.bool, device="cuda")
    eo, el = exact(q, k, v, 0.09, live)
    assert float((lse.double().cpu() - el).abs().max()) <= 1e-5 * (1 + float(el.abs().max()))
    # two roundings of the states and one of the composition
    assert float((out.double().cpu() - eo).abs().max()) <= 3 * 2 ** -8 * float(v.abs().max())


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("Lq", [1, 300])
def test_without_workspace_or_lse(gpu_lib, masked, Lq):
    """Without the workspace of the split the same rows come from one range; a second run gives the same bits."""
    from paper_2607_15650_amd import api
    B, S, H, D = 2, 2000, 4, 128
    q, k, v = make(B, Lq, S, H, H, D, BF16, seed=6)
    mask = None
    if masked:
        mask = torch.rand(B, S, device="cuda") < 0.7
    live = mask if masked else torch.ones(B, S, dtype=torch.bool, device="cuda")
    n = api.cross_attn_workspace_bytes(BF16, B, H, H, D, Lq, S, masked)
    ws = torch.full((n + 256,), 255, dtype=torch.uint8, device="cuda")
    outs = []
    for _ in range(2):
        out, lse = torch.empty_like(q), torch.empty(B, H, Lq, device="cuda")
        api.cross_attn(q, k, v, 0.1, out, lse, None, mask, ws[:n])
        outs.append((out, lse))
        check((out, lse), q, k, v, 0.1, live)
        assert bool((ws[n:] == 255).all())
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    out = torch.empty_like(q)
    api.cross_attn(q, k, v, 0.1, out, None, None, mask, ws[:n])
    assert torch.equal(out, outs[0][0])
    if not masked:
        out, lse = torch.empty_like(q), torch.empty(B, H, Lq, device="cuda")
        api.cross_attn(q, k, v, 0.1, out, lse)
        check((out, lse), q, k, v, 0.1, live)


def test_refusals(gpu_lib):
    from paper_2607_15650_amd import api, _lib
    q, k, v = make(2, 3, 5, 4, 2, 64, BF16)
    out, lse = torch.empty_like(q), torch.empty(2, 4, 3, device="cuda")
    ok = dict(q=q, k=k, v=v, scale=0.1, out=out, lse=lse)
    bad = [
        dict(k=k[:, :4]), dict(k=k[:1], v=v[:1]), dict(k=k.float()), dict(out=out.float()), dict(out=out[:, :2]),
        dict(lse=lse[:, :2]), dict(lse=lse.double()), dict(kv_lens=torch.zeros(2, dtype=torch.int64, device="cuda")),
        dict(kv_lens=torch.zeros(3, dtype=torch.int32, device="cuda")),
        dict(key_mask=torch.ones(2, 4, dtype=torch.bool, device="cuda")),
        dict(key_mask=torch.ones(2, 5, device="cuda")), dict(key_mask=torch.ones(2, 5, dtype=torch.bool, device="cuda")),
        dict(q=q.cpu()), dict(q=q.transpose(2, 3)), dict(q=q[:, :, :3], out=out[:, :, :3].contiguous()),
    ]
    for kw in bad:
        with pytest.raises((ValueError, TypeError)):
            api.cross_attn(**{**ok, **kw})
    with pytest.raises(TypeError):
        api.cross_attn(q.half(), k.half(), v.half(), 0.1, out.half())
    with pytest.raises(_lib.DitangoError):
        api.cross_attn(**{**ok, "scale": -1.0})
    odd = torch.zeros(2, 5, 2, 65, dtype=BF16, device="cuda")
    with pytest.raises(_lib.DitangoError):
        api.cross_attn(**{**ok, "k": odd[..., 1:], "v": odd[..., :64]})


def test_streams_and_graphs(gpu_lib):
    """On a stream of its own, and captured: every replay reads the buffers' contents of that time."""
    from paper_2607_15650_amd import api
    B, Lq, S, H, Hk, D = 2, 1, 3000, 8, 2, 128
    for masked, lq in ((False, 1), (True, 1), (True, 300)):
        q, k, v = make(B, lq, S, H, Hk, D, BF16, seed=9)
        lens = torch.tensor([S, 500], dtype=torch.int32, device="cuda")
        mask = (torch.rand(B, S, device="cuda") < 0.5) if masked else None
        ws = torch.empty(api.cross_attn_workspace_bytes(BF16, B, H, Hk, D, lq, S, masked), dtype=torch.uint8, device="cuda")
        out, lse = torch.empty_like(q), torch.empty(B, H, lq, device="cuda")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            api.cross_attn(q, k, v, 0.09, out, lse, lens, mask, ws)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            api.cross_attn(q, k, v, 0.09, out, lse, lens, mask, ws)
        for i in range(3):
            q.copy_(torch.randn_like(q, dtype=torch.float32))
            lens.copy_(torch.tensor([S - 100 * i, 7 * i], dtype=torch.int32))
            if masked:
                mask.copy_(torch.rand(B, S, device="cuda") < 0.3)
            ws.fill_(255)
            out.fill_(float("nan"))
            graph.replay()
            got = out.clone(), lse.clone()
            api.cross_attn(q, k, v, 0.09, out, lse, lens, mask, ws)
            torch.cuda.synchronize()
            assert torch.equal(out, got[0]) and torch.equal(lse, got[1])
            live = torch.arange(S, device="cuda") < lens[:, None]
            if masked:
                live = live & mask
            check(got, q, k, v, 0.09, live)
