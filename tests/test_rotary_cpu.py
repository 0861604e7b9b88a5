"""The rotary frequencies against worked values, the latent grid's positions,
and what the rotary and cross attention entry points refuse, without a GPU:
every C call here fails its checks before anything is launched."""
import ctypes
import math

import pytest
import torch

from paper_2607_15650_amd.rotary import Rotary, axis_frequencies, grid_positions

FAKE = 0x10000


@pytest.fixture(scope="module")
def L():
    from paper_2607_15650_amd import _lib
    return _lib.lib()


def test_frequencies():
    f, factor = axis_frequencies(4, 100.0)
    assert f == [1.0, 0.1] and factor == 1.0
    f, _ = axis_frequencies(4, 100.0, {"kind": "linear", "factor": 4})
    assert f == [0.25, 0.025]
    # ntk: the first pair keeps its frequency, the last is divided by the factor
    base = axis_frequencies(128)[0]
    f, factor = axis_frequencies(128, scaling={"kind": "ntk", "factor": 8.0})
    assert f[0] == 1.0 and f[-1] == pytest.approx(base[-1] / 8, rel=1e-12) and factor == 1.0
    assert all(a <= b for a, b in zip(f, base))
    # yarn: pairs of more than beta turns are kept, of less than alpha divided
    f, factor = axis_frequencies(128, scaling={"kind": "yarn", "factor": 4.0, "original": 8192, "alpha": 1, "beta": 32})
    turns = [8192 * x / (2 * math.pi) for x in base]
    for got, b, r in zip(f, base, turns):
        g = min(1.0, max(0.0, (r - 1) / 31))
        assert got == pytest.approx(b * g + b / 4 * (1 - g), rel=1e-12)
    assert f[0] == base[0] and f[-1] == base[-1] / 4
    assert factor == pytest.approx(1 + 0.1 * math.log(4), rel=1e-15)


def test_frequency_refusals():
    for dim in (0, 3, -2):
        with pytest.raises(ValueError):
            axis_frequencies(dim)
    for sc in ({"kind": "other", "factor": 2}, {"kind": "linear", "factor": 0.5}, {"kind": "linear", "factor": math.nan},
               {"kind": "yarn", "factor": 2, "original": 0}, {"kind": "yarn", "factor": 2, "original": 9, "beta": 1}):
        with pytest.raises(ValueError):
            axis_frequencies(8, scaling=sc)
    with pytest.raises(ValueError):
        axis_frequencies(2, scaling={"kind": "ntk", "factor": 2})
    for kw in ({"layout": "other"}, {"norm": "other"}, {"axes": [64, 66]}, {"axes": []}, {"axes": [63]}):
        with pytest.raises(ValueError):
            Rotary(128, **kw)


def test_grid_positions():
    p = grid_positions(2, 3, 4, device="cpu")
    assert p.dtype == torch.int32 and tuple(p.shape) == (1, 24, 3)
    assert p[0].tolist() == [[t, h, w] for t in range(2) for h in range(3) for w in range(4)]
    assert torch.equal(grid_positions(2, 3, 4, 7, 9, device="cpu"), p[:, 7:16])
    with pytest.raises(ValueError):
        grid_positions(2, 3, 4, 20, 5, device="cpu")


def cross(L, q=FAKE, k=FAKE, v=FAKE, dt=1, B=2, H=4, Hk=2, D=64, q_len=3, kv_len=5, qs=None, ks=None, vs=None,
          lens=None, mask=None, scale=0.1, out=FAKE + 4096, lse=FAKE, ws=None, n=0):
    I3 = ctypes.c_int64 * 3
    qs = qs or (q_len * H * D, H * D, D)
    ks = ks or (kv_len * Hk * D, Hk * D, D)
    vs = vs or ks
    return L.ditango_cross_attn(q, I3(*qs), k, I3(*ks), v, I3(*vs), dt, B, H, Hk, D, q_len, kv_len, lens, mask, scale,
                                out, lse, ws, n, None)


def test_cross_refusals(L):
    assert cross(L, q=None) == 1
    assert cross(L, k=None) == 1
    assert cross(L, v=None) == 1
    assert cross(L, out=None) == 1
    assert cross(L, dt=2) == 1
    assert cross(L, B=0) == 1
    assert cross(L, H=0) == 1
    assert cross(L, Hk=0) == 1
    assert cross(L, Hk=3) == 1                 # heads not a multiple
    assert cross(L, q_len=0) == 1
    assert cross(L, kv_len=-1) == 1
    assert cross(L, D=96) == 2
    assert cross(L, q_len=1 << 30) == 2        # rows beyond 32 bits
    assert cross(L, kv_len=0x7fffffff) == 2
    for s in (0.0, -1.0, float("nan"), float("inf")):
        assert cross(L, scale=s) == 1
    assert cross(L, qs=(-768, 256, 64)) == 1
    # 16-byte rows
    assert cross(L, q=FAKE + 2) == 2
    assert cross(L, k=FAKE + 8) == 2
    assert cross(L, v=FAKE + 4) == 2
    assert cross(L, out=FAKE + 8) == 2
    assert cross(L, ks=(640, 132, 64)) == 2
    assert cross(L, vs=(640, 128, 60)) == 2
    assert cross(L, ks=(1 << 40, 1 << 24, 64)) == 2
    # the output at an input's place
    for kw in (dict(k=FAKE + 256, v=FAKE + 512), dict(q=FAKE + 256, v=FAKE + 512), dict(q=FAKE + 256, k=FAKE + 512)):
        assert cross(L, out=FAKE, **kw) == 1
    # a mask needs a workspace, 256-byte aligned and large enough
    assert cross(L, mask=FAKE) == 1
    assert cross(L, mask=FAKE, ws=FAKE, n=100) == 1
    assert cross(L, ws=FAKE + 16, n=1 << 20) == 1
    assert L.ditango_cross_attn_workspace_bytes(1, 0, 4, 4, 64, 3, 5, 0) == 0
    assert L.ditango_cross_attn_workspace_bytes(1, 1, 4, 3, 64, 3, 5, 0) == 0
    assert L.ditango_cross_attn_workspace_bytes(1, 1, 4, 4, 80, 3, 5, 0) == 0


def rotary(L, n=1, dt=1, B=2, S=3, D=64, pos=FAKE, pos_b=1, axes=1, pairs=32, layout=0, factor=1.0, norm=0, eps=1e-6,
           x=FAKE, y=FAKE, w=FAKE, heads=2, xs=None, ys=None, freq=None, axis=None):
    from paper_2607_15650_amd import _lib
    arr = (_lib.RotaryTensor * 2)()
    for a in arr:
        a.x, a.y, a.weight, a.heads = x, y, w, heads
        a.x_strides[:] = xs or (S * heads * D, heads * D, D)
        a.y_strides[:] = ys or (S * heads * D, heads * D, D)
    f = (ctypes.c_double * 64)(*(freq or [1.0] * 64))
    ax = (ctypes.c_uint8 * 64)(*(axis or [0] * 64))
    return L.ditango_rotary(arr, n, dt, B, S, D, pos, pos_b, axes, f, ax, 2 * pairs, layout, factor, norm, eps, None)


def test_rotary_refusals(L):
    assert rotary(L, n=0) == 1
    assert rotary(L, n=3) == 1
    assert rotary(L, dt=2) == 1
    assert rotary(L, B=0) == 1
    assert rotary(L, S=0) == 1
    assert rotary(L, D=96) == 2
    assert rotary(L, pos=None) == 1
    assert rotary(L, pos_b=3) == 1
    assert rotary(L, axes=0) == 1
    assert rotary(L, axes=9) == 1
    assert rotary(L, axis=[0, 1] + [0] * 62) == 1
    assert rotary(L, freq=[math.inf] + [0.0] * 63) == 1
    assert rotary(L, freq=[math.nan] + [0.0] * 63) == 1
    assert rotary(L, pairs=0) == 1
    assert rotary(L, pairs=33) == 1
    assert rotary(L, layout=2) == 1
    assert rotary(L, norm=3) == 1
    assert rotary(L, factor=math.nan) == 1
    assert rotary(L, norm=1, eps=-1.0) == 1
    assert rotary(L, norm=2, eps=math.nan) == 1
    assert rotary(L, norm=1, w=None) == 1
    assert rotary(L, x=None) == 1
    assert rotary(L, y=None) == 1
    assert rotary(L, heads=0) == 1
    assert rotary(L, heads=1025) == 2
    assert rotary(L, xs=(-384, 128, 64)) == 1
    assert rotary(L, xs=(768, 256, 64)) == 1   # in place with other strides
    assert rotary(L, B=1 << 16, S=1 << 16) == 2
    # outputs whose rows overlap: repeated, closer than a row, interleaved heads; two tensors at one place
    other = ctypes.create_string_buffer(16)
    for ys in ((768, 128, 0), (0, 128, 64), (768, 64, 64), (768, 128, 32), (64, 128, 64)):
        assert rotary(L, B=2, heads=2, y=ctypes.addressof(other), ys=ys) == 1
    assert rotary(L, n=2) == 1
    # 2^32 threads: a launch has fewer
    assert rotary(L, S=1 << 30, heads=1) == 2
