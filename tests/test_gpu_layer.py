"""Rotary positions, selective self attention and cross attention together, as a
DiT layer runs them over denoising steps: the engines with `rotary` against the
same engines on tensors rotated beforehand (bit for bit: the same kernels on the
same rows), and the chain against attention in 64 bits on those tensors."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
B, S, H, D, P = 2, 700, 4, 64, 5
OFFS = [0, 150, 290, 290, 520, 700]          # one partition without tokens


def inputs(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").to(BF16)   # noqa: E731
    qkv = r(B, S, 3 * H, D)
    return (*(qkv[:, :, i * H:(i + 1) * H] for i in range(2)), qkv[:, :, 2 * H:].contiguous(),
            (1 + 0.1 * r(D).float()).to(BF16), (1 + 0.1 * r(D).float()).to(BF16))


def positions():
    from paper_2607_15650_amd.rotary import grid_positions
    return grid_positions(10, 7, 10)


def rotary(norm="head"):
    from paper_2607_15650_amd.rotary import Rotary
    return Rotary(D, axes=[24, 20, 20], norm=norm)


def test_engines_rotate_what_they_read(gpu_lib):
    from paper_2607_15650_amd.ase import ErrorModelSelectiveAttention
    from paper_2607_15650_amd.groups import GroupedSelectiveAttention, base_groups
    from paper_2607_15650_amd.step import SelectiveAttention
    op, pos, scale = rotary(), positions(), D ** -0.5
    args = (B, H, D, OFFS, scale)
    one, two = SelectiveAttention(*args, rotary=op), SelectiveAttention(*args)
    gargs = (B, H, D, OFFS, 1, 2, scale)
    g1, g2 = GroupedSelectiveAttention(*gargs, rotary=op), GroupedSelectiveAttention(*gargs)
    eargs = (B, H, D, OFFS, 3, 1, scale, 0.5, 0.4)
    e1, e2 = (ErrorModelSelectiveAttention(*eargs, evaluate=True, rotary=r) for r in (op, None))
    groups = base_groups(P, 1, 2)
    for t in range(3):
        q, k, v, wq, wk = inputs(t)
        qr, kr = op(q, k, pos, wq, wk)
        for qb in (1, 3):
            select = [1] * P if t == 0 else [int(j in (qb, 4 * (t - 1))) for j in range(P)]
            got = one.step(t, qb, q, k, v, select, pos, wq, wk)
            want = two.step(t, qb, qr, kr, v, select)
            assert all(torch.equal(a, b) for a, b in zip(got, want))
        compute = groups if t == 0 else groups[:t]
        got, want = g1.step(t, q, k, v, compute, pos, wq, wk), g2.step(t, qr, kr, v, compute)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        a, b = e1.step(t, q, k, v, pos, wq, wk), e2.step(t, qr, kr, v)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        assert a[2]["compute"] == b[2]["compute"] and a[2].get("measured") == b[2].get("measured")


def attention64(q, k, v, scale, live=None):
    """[B, L, H, D] x [B, S, H, D]: OUT in 64 bits."""
    out = torch.zeros(q.shape, dtype=torch.float64)
    q, k, v = (x.double().cpu() for x in (q, k, v))
    for b in range(q.shape[0]):
        at = torch.arange(k.shape[1]) if live is None else live[b].cpu().nonzero().flatten()
        for h in range(q.shape[2]):
            s = q[b, :, h] @ k[b, at, h].T * scale
            out[b, :, h] = torch.softmax(s, 1) @ v[b, at, h]
    return out


@pytest.mark.parametrize("graph", [False, True])
def test_layer(gpu_lib, graph):
    """Two blocks of a layer over one step: rotate, attend to the sequence, then to the prompt; captured too."""
    from paper_2607_15650_amd.cross import CrossAttention
    from paper_2607_15650_amd.step import SelectiveAttention
    op, pos, scale = rotary("row"), positions(), D ** -0.5
    q, k, v, _, _ = inputs(5)
    wq, wk = (torch.linspace(0.5, 1.5, H * D, device="cuda").to(BF16) for _ in range(2))
    text_k, text_v = (torch.randn(B, 77, H, D, device="cuda").to(BF16) for _ in range(2))
    lens = torch.tensor([77, 20], dtype=torch.int32, device="cuda")
    engine, cross = SelectiveAttention(B, H, D, OFFS, scale, rotary=op), CrossAttention(scale)

    def layer():
        got = []
        for qb in (0, 4):
            x, _, _ = engine.step(0, qb, q, k, v, [1] * P, pos, wq, wk)
            # (the block's output is the next projection's input; here the query itself)
            y, _ = cross(x, text_k, text_v, kv_lens=lens)
            got.append((x, y))
        return got

    if graph:
        layer()
        torch.cuda.synchronize()
        rec = torch.cuda.CUDAGraph()
        with torch.cuda.graph(rec):
            got = layer()
        for i in range(3):
            q.copy_(torch.randn(q.shape, device="cuda"))
            lens.copy_(torch.tensor([77 - i, 20 + i], dtype=torch.int32))
            rec.replay()
            again = [(x.clone(), y.clone()) for x, y in got]
            want = layer()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for p, r in zip(again, want) for a, b in zip(p, r))
    else:
        got = layer()
    live = torch.arange(77, device="cuda") < lens[:, None]
    qr, kr = op(q[:, :OFFS[1]].contiguous(), None, pos[:, :OFFS[1]].contiguous(), wq), op(k, None, pos, wk)
    # the probabilities' and the output's rounding, and that of the states that are composed: 2^-8 each of at most
    # max|v|; float32 accumulation beside them
    tol = lambda t: (3 * 2.0 ** -8 + 2.0 ** -16) * float(t.abs().max())   # noqa: E731
    x, y = got[0]
    assert float((x.double().cpu() - attention64(qr, kr, v, scale)).abs().max()) <= tol(v)
    assert float((y.double().cpu() - attention64(x, text_k, text_v, scale, live)).abs().max()) <= tol(text_v)


def test_a_captured_step_keeps_its_buffers(gpu_lib):
    """Steps of larger query blocks, after the capture of a smaller one's, leave its replays as they were."""
    from paper_2607_15650_amd.step import SelectiveAttention
    pos, scale = positions(), D ** -0.5
    q, k, v, wq, wk = inputs(7)
    engine, other = (SelectiveAttention(B, H, D, OFFS, scale, rotary=rotary()) for _ in range(2))
    engine.step(0, 1, q, k, v, [1] * P, pos, wq, wk)           # 140 rows, of at most 230
    torch.cuda.synchronize()
    rec = torch.cuda.CUDAGraph()
    with torch.cuda.graph(rec):
        got = engine.step(0, 1, q, k, v, [1] * P, pos, wq, wk)
    for i in range(3):
        engine.step(0, 3, q, k, v, [1] * P, pos, wq, wk)
        fill = [torch.full((B, 230, H, D), math.nan, dtype=BF16, device="cuda") for _ in range(8)]
        q.copy_(torch.randn(q.shape, device="cuda"))
        rec.replay()
        want = other.step(0, 1, q, k, v, [1] * P, pos, wq, wk)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and bool(torch.isnan(torch.stack(fill)).all())


def test_refusals(gpu_lib):
    from paper_2607_15650_amd.step import SelectiveAttention
    q, k, v, wq, wk = inputs(1)
    pos = positions()
    plain, turned = SelectiveAttention(B, H, D, OFFS, 0.1), SelectiveAttention(B, H, D, OFFS, 0.1, rotary=rotary())
    with pytest.raises(ValueError):
        plain.step(0, 0, q.contiguous(), k.contiguous(), v, [1] * P, pos)
    with pytest.raises(ValueError):
        turned.step(0, 0, q, k, v, [1] * P)
    with pytest.raises(ValueError):
        turned.step(0, 0, q, k, v, [1] * P, pos[:, :5], wq, wk)
    with pytest.raises(ValueError):
        turned.step(0, 0, q, k, v, [1] * P, pos)               # the norm needs its weights
