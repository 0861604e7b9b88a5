"""Host side of the cross attention's and the rotary inputs' classes, without a
GPU: what they hand over and copy, and the buffers they keep (the calls are
recorded, nothing is computed)."""
import pytest
import torch

from paper_2607_15650_amd import api
from paper_2607_15650_amd.cross import CrossAttention

BF16 = torch.bfloat16


@pytest.fixture
def calls(monkeypatch):
    """Arguments of every cross_attn call; each wants the workspace that `need` says."""
    log, need = [], {"bytes": 0}
    monkeypatch.setattr(api, "cross_attn", lambda *a: log.append(a))
    monkeypatch.setattr(api, "cross_attn_workspace_bytes", lambda *a: need["bytes"])
    return log, need


def test_rows_that_cannot_be_read_in_place_are_copied(calls):
    log, _ = calls
    buf = torch.arange(1 << 25, dtype=torch.int32).to(BF16)

    def rows(stride, heads=64, at=0):
        return torch.as_strided(buf, (1, 2, 2, 64), (0, stride, heads, 1), at)

    def handed(**kw):
        x = {**dict(q=rows(256), k=rows(256), v=rows(256)), **kw}
        CrossAttention(0.125)(**x)
        got = dict(zip("qkv", log[-1][:3]))
        assert all(torch.equal(got[n], x[n]) for n in "qkv")
        return {n for n in "qkv" if got[n].data_ptr() == x[n].data_ptr() and got[n].stride() == x[n].stride()}

    far = 1 << 24
    assert handed() == {"q", "k", "v"}
    # keys and values below 2^24 elements apart stay, queries at any distance
    assert handed(q=rows(far), k=rows(far - 8), v=rows(far - 8)) == {"q", "k", "v"}
    assert handed(k=rows(far)) == {"q", "v"}
    assert handed(v=rows(far + 8)) == {"q", "k"}
    for bad in (rows(257), rows(256, heads=68), rows(256, at=1)):
        for n in "qkv":
            assert handed(**{n: bad}) == set("qkv") - {n}


def test_each_device_has_its_workspace(calls):
    """Calls on two devices in turn keep one buffer each, however many they are; a
    larger call keeps the smaller one's for graphs that hold it."""
    log, need = calls
    need["bytes"] = 1000
    op = CrossAttention(0.125)
    x = torch.zeros(1, 2, 2, 64, dtype=BF16)
    y = x.to("meta")
    for _ in range(4):
        for t in (x, y):
            op(t, t, t)
    used = [a[-1] for a in log]
    assert all(w.device == a[0].device and w.numel() == 1000 for w, a in zip(used, log))
    assert all(w is used[i % 2] for i, w in enumerate(used)) and not op._kept
    need["bytes"] = 1500
    z = torch.zeros(1, 3, 2, 64, dtype=BF16)
    op(z, x, x)
    assert log[-1][-1].numel() >= 1500 and len(op._kept) == 1 and op._kept[0] is used[0]


def test_rotated_inputs_keep_a_buffer_of_each_type():
    """Steps in bf16 and float32 in turn (states in float32 take both) use two
    pairs of buffers, however many they are, and a larger batch keeps what it
    replaces, within what it uses."""
    from paper_2607_15650_amd.rotary import RotatedInputs
    seen = []

    def rotary(x, k, pos, qw=None, kw=None, q_out=None, k_out=None):
        seen.append(q_out.data_ptr())

    r = RotatedInputs(rotary, [0, 4, 12])
    pos = torch.zeros(1, 12, 1, dtype=torch.int32)

    def step(dtype, B=1):
        x = torch.zeros(B, 12, 2, 64, dtype=dtype)
        q = r.begin(0, x, x, pos, None, None)
        k = r.keys([1, 1])
        assert q.shape == (B, 4, 2, 64) and k.shape == x.shape and q.dtype == k.dtype == dtype
        return q.data_ptr(), k.data_ptr()

    first = [step(d) for d in (BF16, torch.float32)]
    assert [step(d) for _ in range(3) for d in (BF16, torch.float32)] == first * 3 and not r._kept
    for B in range(2, 12):
        step(BF16, B)
    in_use = sum(b.numel() * b.element_size() for b in r._buffers.values())
    assert 0 < sum(b.numel() * b.element_size() for b in r._kept) <= in_use
    assert {b.data_ptr() for b in r._kept} >= set(first[0])


def test_a_replaced_attention_workspace_stays_allocated(monkeypatch):
    """A step that was captured holds the address of the workspace of its time."""
    from paper_2607_15650_amd.workspace import AttnWorkspace
    monkeypatch.setattr(api, "attn_workspace_bytes", lambda dtype, B, H, D, q_len, offsets, select: 256 * q_len)
    ws = AttnWorkspace("cpu")
    get = lambda n: ws.get(BF16, 1, 1, 64, n, [0, 1], [1])   # noqa: E731
    small = get(1)
    at = small.data_ptr()
    assert get(1) is small
    del small
    held = [get(n) for n in range(2, 40)]
    assert any(b.data_ptr() == at and b.numel() == 256 for b in ws._kept)
    assert all(b.numel() >= 256 * n for n, b in zip(range(2, 40), held))
    assert sum(b.numel() for b in ws._kept) <= ws.buf.numel()
