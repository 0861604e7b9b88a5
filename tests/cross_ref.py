"""Cross attention in 64 bits, and how far bf16 and float32 results may be from
it, element by element."""
import math

import torch


def reference(q, k, v, scale, live, device="cpu"):
    """q [B, L, H, D], k, v [B, S, Hk, D], live bool [B, S] -> OUT, LSE and sum
    p |v| (what the rounding of the probabilities goes by) in 64 bits, on the CPU."""
    q, k, v = (x.double().to(device) for x in (q, k, v))
    B, L, H, D = q.shape
    G = H // k.shape[2]
    out, apart = (torch.zeros(B, L, H, D, dtype=torch.float64, device=device) for _ in range(2))
    lse = torch.full((B, H, L), -math.inf, dtype=torch.float64, device=device)
    for b in range(B):
        at = live[b].to(device).nonzero().flatten()
        if at.numel() == 0:
            continue
        for h in range(H):
            vb = v[b, at, h // G].contiguous()
            s = q[b, :, h] @ k[b, at, h // G].T.contiguous() * scale
            lse[b, h] = torch.logsumexp(s, 1)
            p = torch.softmax(s, 1)
            out[b, :, h] = p @ vb
            apart[b, :, h] = p @ vb.abs()
    return out.cpu(), lse.cpu(), apart.cpu()


def tolerance(dtype, want, apart, top):
    """Of OUT against ``want``, with ``apart`` = sum p |v| and ``top`` = max |v|.

    bf16: the probabilities are rounded, by at most 2^-8 each, and the output by
    2^-8; beside them float32: scores off by 2^-24 a product and sum of a tile's
    few, which at scores of order 10 moves a probability by less than 2^-15, and
    the sums of the products, under 2^-18 of the largest value.
    float32: scores of order 5 off by 2^-23 * 8 move a probability by 1e-5, numerator
    and row sum together."""
    if dtype == torch.bfloat16:
        return (2.0 ** -8 + 2.0 ** -14) * apart + 2.0 ** -8 * want.abs() + 2.0 ** -18 * top
    return 1e-5 * apart + 2.0 ** -22 * top
