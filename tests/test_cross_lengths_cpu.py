"""The number of keys that the cross attention takes, without a GPU."""
from test_rotary_cpu import L, cross   # noqa: F401

MOST = (1 << 31) - (1 << 20)


def test_most_keys(L):   # noqa: F811
    """More than 2^31 - 2^20 are refused for their number; the others are not
    (what stops those here is that there is no device to run on, or a mask
    without a workspace)."""
    far = dict(ks=(0, 0, 64), vs=(0, 0, 64))
    for n in (MOST + 1, (1 << 31) - 1025, (1 << 31) - 1):
        assert cross(L, kv_len=n, **far) == 2
        assert L.ditango_cross_attn_workspace_bytes(1, 2, 4, 2, 64, 3, n, 0) == 0
    for n in (MOST, MOST - 1, 1 << 30):
        assert cross(L, kv_len=n, mask=0x10000, **far) == 1
