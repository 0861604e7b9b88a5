"""float32 self attention at the ends of the value range (it shares its loop with the
float32 cross attention), in its forms of 32, 128 and 256 rows."""
import math

import pytest
import torch

from test_gpu_f32 import SHAPES, reference, run

pytestmark = pytest.mark.gpu


def offsets(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


@pytest.mark.parametrize("D,H,q_len,lens", SHAPES)
def test_large_scores(gpu_lib, D, H, q_len, lens):
    """Scores of 1e3 ... 1e30, the largest of a partition two from the next: its value
    alone, through the planes' products (2^-22), and LSE its score."""
    offs = offsets(lens)
    g = torch.Generator().manual_seed(D + H)
    q, k = torch.zeros(1, q_len, H, D), torch.zeros(1, offs[-1], H, D)
    q[..., 7] = 10.0 ** torch.randint(3, 31, (1, q_len, H), generator=g).float()
    q[:, ::2, :, 7] *= -1
    k[..., 7] = (torch.rand(1, offs[-1], H, generator=g) - 0.5) / 2
    for a, e in zip(offs, offs[1:]):
        if e - a > 1:
            k[:, a + (e - a) // 3, :, 7], k[:, e - 1, :, 7] = 1.0, -1.0
    v = torch.randn(1, offs[-1], H, D, generator=g)
    out, lse = run(q, k, v, offs, 1.3)
    outs, lses = reference(q, k, v, offs, 1.3)
    for j, n in enumerate(lens):
        if n:
            assert float((out[j] - outs[j]).abs().max()) <= 2.0 ** -22 * float(v.abs().max())
            assert float(((lse[j] - lses[j]).abs() - 2.0 ** -21 * lses[j].abs()).max()) <= 0


@pytest.mark.parametrize("D,H,q_len,lens", SHAPES)
def test_values_near_the_largest(gpu_lib, D, H, q_len, lens):
    offs = offsets(lens)
    g = torch.Generator().manual_seed(D + H)
    q, k = (torch.randn(1, n, H, D, generator=g) for n in (q_len, offs[-1]))
    v = torch.full((1, offs[-1], H, D), 3e38)
    v[..., ::2] *= torch.where(torch.rand(1, offs[-1], H, D // 2, generator=g) < 0.5, -1.0, 1.0)
    out, lse = run(q, k, v, offs, 1 / math.sqrt(D))
    outs, lses = reference(q, k, v, offs, 1 / math.sqrt(D))
    for j, n in enumerate(lens):
        if n:
            # probabilities off by 1e-5 together, as at values of order 1
            assert bool(torch.isfinite(out[j]).all()) and float((out[j] - outs[j]).abs().max()) <= 1e-5 * 3e38
            assert float((lse[j] - lses[j]).abs().max()) <= 1e-5
