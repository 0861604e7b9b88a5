"""The operators around the selective self attention of a video-DiT layer, as
cases that can be timed and compared: the rotary positions (with the
root-mean-square norm) that make its queries and keys, and the cross attention
to an encoder's states that follows it.

Plain forms: elementary torch operations in 32 bits, rounded once at the end;
angles in 64 bits.  Inputs are what a projection leaves: unit-variance noise
with a smooth component along the sequence, norm weights around one.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}
_EPS = 1e-6


def _cross(name, dtype, B, H, Hk, Lq, Lk, D, live, short, packed=False):
    return {"name": name, "kind": "cross", "dtype": dtype, "B": B, "H": H, "Hk": Hk, "Lq": Lq, "Lk": Lk, "D": D,
            "live": live, "short": short, "packed": packed}


def _rotary(name, dtype, B, S, H, Hk, D, R, layout, norm, scaling, grid, first, packed=False):
    return {"name": name, "kind": "rotary", "dtype": dtype, "B": B, "S": S, "H": H, "Hk": Hk, "D": D, "R": R,
            "layout": layout, "norm": norm, "scaling": scaling, "grid": grid, "first": first, "packed": packed}


def listed():
    return [
        # one token against a short prompt: launch latency
        _cross("cross_token", "bf16", 1, 12, 12, 1, 77, 128, "all", 77),
        # one token of each of eight sequences against long encoder states
        # (a reference clip), heads shared by three, ragged lengths
        _cross("cross_token_long", "bf16", 8, 24, 8, 1, 16384, 128, "lens", 1000),
        # the flagship step's query block against a 512-token prompt, 40 heads
        _cross("cross_video", "bf16", 1, 40, 40, 9450, 512, 128, "all", 512),
        # conditional and unconditional branch in one batch, prompts of 512
        # and 77 tokens, keys and values from one packed projection
        _cross("cross_cfg_lens", "bf16", 2, 12, 12, 4095, 512, 128, "lens", 77, True),
        # head dim 64, 48 heads, 129 frames at 720p over 8 ranks, padded
        # prompt pieces of two encoders: a key mask with 256 of 333 live
        _cross("cross_d64_mask", "bf16", 1, 48, 48, 14850, 333, 64, "mask", 256),
        # a long block against long encoder states, heads shared by three
        _cross("cross_long_gqa", "bf16", 1, 24, 8, 8192, 4099, 128, "all", 4099),
        # float32 at an ordinary, odd size
        _cross("cross_f32", "f32", 1, 12, 12, 2047, 333, 128, "all", 333),
        # one token of each of eight sequences, far positions, half layout on
        # half of the head, scaled for long contexts: launch latency
        _rotary("rotary_token", "bf16", 8, 1, 24, 8, 128, 64, "half", "none", "yarn", False, 1000000),
        # the flagship step's query block and its own keys: 40 heads, frame,
        # row and column axes, norm over the whole row
        _rotary("rotary_video", "bf16", 1, 9450, 40, 40, 128, 128, "interleaved", "row", "none", True, 28350),
        # head dim 64, 48 heads, norm of each head, queries and keys read in
        # place from a packed projection
        _rotary("rotary_packed_d64", "bf16", 1, 14850, 48, 48, 64, 64, "half", "head", "none", True, 44550, True),
        # a batch of two long sequences, no norm, one axis
        _rotary("rotary_long", "bf16", 2, 16384, 24, 24, 128, 128, "half", "none", "ntk", False, 65536),
        # float32 at an ordinary, odd size
        _rotary("rotary_f32", "f32", 1, 4095, 12, 12, 128, 128, "interleaved", "head", "linear", False, 0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges; no dearer than the largest listed one."""
    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["cross", "cross", "rotary"])
        g = rng.choice([1, 1, 1, 2, 3, 4, 8])
        hk = _log(rng, 1, 48)
        c = {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "bf16", "f32"]), "B": rng.choice([1, 1, 2, 3, 8]),
             "H": g * hk, "Hk": hk, "D": rng.choice([64, 128]), "packed": rng.choice([True, False])}
        if c["H"] > 64:
            continue
        if kind == "cross":
            c["Lq"] = rng.choice([1, 1, rng.randint(2, 16), _log(rng, 17, 16384), _log(rng, 17, 16384),
                                  _log(rng, 17, 16384)])
            c["Lk"] = _log(rng, 1, 32768) if c["Lq"] <= 16 else _log(rng, 16, 4800)
            c["live"] = rng.choice(["all", "lens", "mask"])
            c["short"] = c["Lk"] if c["live"] == "all" else _log(rng, 1, c["Lk"])
            if c["B"] > 1 and c["live"] != "all" and rng.random() < 0.2:
                c["short"] = 0      # a sequence without keys
            if c["B"] * c["Lk"] * c["Hk"] * c["D"] > 4e8 or c["B"] * c["H"] * c["Lq"] * c["Lk"] > 8e8:
                continue
            if c["dtype"] == "f32" and work(c)["flops"] > 4e10:
                continue
        else:
            c["S"] = rng.choice([1, _log(rng, 2, 32768), _log(rng, 2, 32768)])
            c["R"] = rng.choice([c["D"], c["D"], c["D"] // 2, c["D"] // 2 + 8])
            c["layout"], c["norm"] = rng.choice(["interleaved", "half"]), rng.choice(["none", "head", "row"])
            c["grid"] = rng.choice([True, False])
            c["scaling"] = "none" if c["grid"] else rng.choice(["none", "linear", "ntk", "yarn"])
            c["first"] = rng.choice([0, _log(rng, 1, 1000000)])
            if c["B"] * c["S"] * c["H"] * c["D"] > 1.1e8:
                continue
        if _cost(c) <= most:
            return c


# ------------------------------------------------------------------ shapes
def _lens(c):
    """Live keys of every sequence: from all down to the shortest."""
    if c["B"] == 1:
        return [c["short"]]
    return [c["Lk"] - (c["Lk"] - c["short"]) * b // (c["B"] - 1) for b in range(c["B"])]


def _axes(c):
    """Rotated dims of each axis: frame, row and column of a latent grid, or one."""
    n = 2 * (c["R"] // 6)
    return [c["R"] - 2 * n, n, n] if c["grid"] else [c["R"]]


#: A latent grid's rows and columns (720p).
_GRID = (45, 80)
_THETA, _SCALE, _ORIGINAL, _ALPHA, _BETA = 10000.0, 4.0, 8192, 1.0, 32.0


# ------------------------------------------------------------------ inputs
def _gen(seed, k):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 16 + k)
    return g


def _tokens(B, S, H, D, dtype, g):
    """What a projection leaves: noise, and a component that varies slowly along the sequence."""
    x = torch.randn((B, S, H, D), generator=g, device="cuda")
    f = torch.rand(D, generator=g, device="cuda") * (4 * math.pi / max(S, 16))
    x.add_(0.5 * torch.sin(torch.arange(S, device="cuda")[:, None] * f)[None, :, None, :])
    return x.to(dtype)


def prepare(case, seed):
    c = dict(case)
    st = {"case": c}
    g = _gen(seed, 0)
    dt, B, H, Hk, D = _DT[c["dtype"]], c["B"], c["H"], c["Hk"], c["D"]
    if c["kind"] == "cross":
        st["q"] = _tokens(B, c["Lq"], H, D, dt, g)
        if c["packed"]:
            kv = _tokens(B, c["Lk"], 2 * Hk, D, dt, g)
            st["k"], st["v"] = kv[:, :, :Hk], kv[:, :, Hk:]
        else:
            st["k"], st["v"] = _tokens(B, c["Lk"], Hk, D, dt, g), _tokens(B, c["Lk"], Hk, D, dt, g)
        st["scale"] = 1.0 / math.sqrt(D)
        st["lens"] = st["mask"] = None
        if c["live"] == "lens":
            st["lens"] = torch.tensor(_lens(c), dtype=torch.int32, device="cuda")
        elif c["live"] == "mask":
            # which keys are live: the first n of a random order
            order = torch.rand((B, c["Lk"]), generator=g, device="cuda").argsort(dim=1).argsort(dim=1)
            st["mask"] = order < torch.tensor(_lens(c), device="cuda")[:, None]
        return st
    S = c["S"]
    if c["packed"]:
        qkv = _tokens(B, S, H + 2 * Hk, D, dt, g)
        st["q"], st["k"] = qkv[:, :, :H], qkv[:, :, H:H + Hk]
    else:
        st["q"], st["k"] = _tokens(B, S, H, D, dt, g), _tokens(B, S, Hk, D, dt, g)
    n = c["first"] + torch.arange(S, device="cuda")
    if c["grid"]:
        h, w = _GRID
        st["pos"] = torch.stack([n // (h * w), n // w % h, n % w], dim=-1).to(torch.int32)[None]
    else:
        # every sequence of the batch stands at a place of its own
        st["pos"] = (n[None, :, None] + 17 * torch.arange(B, device="cuda")[:, None, None]).to(torch.int32)
    st["pos"] = st["pos"].contiguous()
    st["wq"] = st["wk"] = None
    if c["norm"] != "none":
        nq, nk = (D, D) if c["norm"] == "head" else (H * D, Hk * D)
        st["wq"] = (1 + 0.1 * torch.randn(nq, generator=g, device="cuda")).to(dt)
        st["wk"] = (1 + 0.1 * torch.randn(nk, generator=g, device="cuda")).to(dt)
    return st


# --------------------------------------------------------------------- run
def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    c = st["case"]
    op = st.get("op")
    if op is None:
        # the layer's handle, made once: frequencies, workspace
        op = st["op"] = _handle(c, st)
    if c["kind"] == "cross":
        out, lse = op(st["q"], st["k"], st["v"], kv_lens=st["lens"], key_mask=st["mask"])
        return {"out": out, "lse": lse}
    q, k = op(st["q"], st["k"], st["pos"], q_weight=st["wq"], k_weight=st["wk"])
    return {"q": q, "k": k}


def _handle(c, st):
    if c["kind"] == "cross":
        from paper_2607_15650_amd.cross import CrossAttention
        return CrossAttention(st["scale"])
    from paper_2607_15650_amd.rotary import Rotary
    scaling = None if c["scaling"] == "none" else {"kind": c["scaling"], "factor": _SCALE}
    if c["scaling"] == "yarn":
        scaling.update(original=_ORIGINAL, alpha=_ALPHA, beta=_BETA)
    return Rotary(c["D"], axes=_axes(c), theta=_THETA, layout=c["layout"], scaling=scaling, norm=c["norm"], eps=_EPS)


def _run_plain(st):
    c = st["case"]
    if c["kind"] == "cross":
        out, lse = _plain_cross(c, st["q"], st["k"], st["v"], st["scale"], st["lens"], st["mask"])
        return {"out": out, "lse": lse}
    cos, sin = _plain_angles(c, st["pos"])
    return {"q": _plain_rotary(c, st["q"], st["wq"], cos, sin), "k": _plain_rotary(c, st["k"], st["wk"], cos, sin)}


def _plain_cross(c, q, k, v, scale, lens, mask):
    B, Lq, H, D = q.shape
    Lk, Hk = k.shape[1], k.shape[2]
    kf, vf = (x.float().transpose(1, 2) for x in (k, v))
    live = None
    if lens is not None:
        live = torch.arange(Lk, device=q.device) < lens[:, None]
    elif mask is not None:
        live = mask
    if live is not None:
        kf, vf = (torch.where(live[:, None, :, None], x, 0.0) for x in (kf, vf))
    qf = q.float().reshape(B, Lq, Hk, H // Hk, D).permute(0, 2, 3, 1, 4).reshape(B * Hk, -1, D)
    s = torch.bmm(qf, kf.reshape(B * Hk, Lk, D).transpose(1, 2).contiguous()).mul_(scale).view(B, Hk, -1, Lk)
    if live is not None:
        s = torch.where(live[:, None, None, :], s, -math.inf)
    m = s.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = s.sub_(m).exp_()
    total = p.sum(dim=-1, keepdim=True)
    o = torch.bmm(p.view(B * Hk, -1, Lk), vf.reshape(B * Hk, Lk, D)).view(B, Hk, -1, D)
    o = torch.where(total > 0, o / total, 0.0)
    lse = (m + total.log()).view(B, H, Lq)
    return o.view(B, H, Lq, D).transpose(1, 2).contiguous().to(q.dtype), lse


def _plain_angles(c, pos):
    """cos and sin [B or 1, S, 1, R/2] with the scaling's factor, in 32 bits."""
    at, parts, factor = pos.double(), [], 1.0
    for a, dim in enumerate(_axes(c)):
        theta = _THETA
        if c["scaling"] == "ntk":
            theta *= _SCALE ** (dim / (dim - 2))
        f = theta ** (-torch.arange(0, dim, 2, device=pos.device, dtype=torch.float64) / dim)
        if c["scaling"] == "linear":
            f = f / _SCALE
        elif c["scaling"] == "yarn":
            turns = _ORIGINAL * f / (2 * math.pi)
            keep = ((turns - _ALPHA) / (_BETA - _ALPHA)).clamp(0, 1)
            f = f * (keep + (1 - keep) / _SCALE)
            factor = 0.1 * math.log(_SCALE) + 1
        parts.append(at[..., a:a + 1] * f)
    angle = torch.cat(parts, dim=-1)[:, :, None, :]
    return (angle.cos() * factor).float(), (angle.sin() * factor).float()


def _plain_rotary(c, x, w, cos, sin):
    y = x.float()
    if c["norm"] == "head":
        y = y * (y.square().mean(dim=-1, keepdim=True) + _EPS).rsqrt() * w.float()
    elif c["norm"] == "row":
        y = y * (y.square().mean(dim=(-2, -1), keepdim=True) + _EPS).rsqrt() * w.float().view(y.shape[2:])
    R = c["R"]
    if c["layout"] == "half":
        a, b = y[..., :R // 2], y[..., R // 2:R]
        z = torch.cat([a * cos - b * sin, a * sin + b * cos, y[..., R:]], dim=-1)
    else:
        a, b = y[..., 0:R:2], y[..., 1:R:2]
        z = torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2), y[..., R:]], dim=-1)
    return z.to(x.dtype)


# -------------------------------------------------------------------- work
def work(case):
    """Each input read once (of keys and values the live ones), each output written once."""
    c = case
    e, B, H, Hk, D = _BYTES[c["dtype"]], c["B"], c["H"], c["Hk"], c["D"]
    if c["kind"] == "cross":
        keys = sum(_lens(c))
        rows = B * c["Lq"] * H
        extra = 4 * B if c["live"] == "lens" else B * c["Lk"] if c["live"] == "mask" else 0
        return {"bytes": 2 * rows * D * e + 4 * rows + 2 * keys * Hk * D * e + extra,
                "flops": 4.0 * c["Lq"] * H * D * keys}
    n = B * c["S"] * (H + Hk) * D
    pos = 12 * c["S"] if c["grid"] else 4 * B * c["S"]
    weights = 0 if c["norm"] == "none" else 2 * D * e if c["norm"] == "head" else (H + Hk) * D * e
    return {"bytes": 2 * n * e + pos + weights,
            "flops": 3.0 * n * c["R"] / c["D"] + (0.0 if c["norm"] == "none" else 4.0 * n)}


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


# ------------------------------------------------------------------- exact
def exact(case, seed):
    st = prepare(case, seed)
    c = st["case"]
    if c["kind"] == "cross":
        return _exact_cross(c, st)
    # one complex number of absolute value `factor` for each pair
    turn, factor = [], 1.0
    for a, dim in enumerate(_axes(c)):
        for i in range(dim // 2):
            f = math.exp(-2.0 * i / dim * math.log(_THETA))
            if c["scaling"] == "linear":
                f /= _SCALE
            elif c["scaling"] == "ntk":
                f *= math.exp(-2.0 * i / (dim - 2) * math.log(_SCALE))
            elif c["scaling"] == "yarn":
                r = f * _ORIGINAL / (2 * math.pi)
                g = min(1.0, max(0.0, (r - _ALPHA) / (_BETA - _ALPHA)))
                f = (1 - g) * f / _SCALE + g * f
                factor = 1 + math.log(_SCALE) / 10
            turn.append(st["pos"][..., a].double() * f)
    z = torch.polar(torch.full_like(torch.stack(turn, -1), factor), torch.stack(turn, -1))[:, :, None, :]
    got = {}
    for name, w in (("q", st["wq"]), ("k", st["wk"])):
        x = st[name].double()
        if c["norm"] != "none":
            dims = (3,) if c["norm"] == "head" else (2, 3)
            x = x / torch.sqrt(torch.mean(x * x, dim=dims, keepdim=True) + _EPS) * w.double().reshape(-1, c["D"])
        h = c["R"] // 2
        pairs = torch.arange(c["R"], device=x.device)
        first, second = (pairs[:h], pairs[h:]) if c["layout"] == "half" else (pairs[0::2], pairs[1::2])
        y = torch.complex(x[..., first], x[..., second]) * z
        x[..., first], x[..., second] = y.real, y.imag
        got[name] = x
    return got


def _exact_cross(c, st):
    q, k, v = st["q"], st["k"], st["v"]
    B, Lq, H, D = q.shape
    out = torch.zeros((B, Lq, H, D), dtype=torch.float64, device="cuda")
    lse = torch.full((B, H, Lq), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(B):
        at = torch.arange(c["Lk"], device="cuda")
        if st["lens"] is not None:
            at = at[:int(st["lens"][b])]
        elif st["mask"] is not None:
            at = st["mask"][b].nonzero().flatten()
        if at.numel() == 0:
            continue
        for h in range(H):
            kd, vd = (x[b, :, h // (H // c["Hk"])][at].double() for x in (k, v))
            s = torch.mm(q[b, :, h].double(), kd.t().contiguous()) * st["scale"]
            lse[b, h] = torch.logsumexp(s, dim=1)
            out[b, :, h] = torch.mm(torch.softmax(s, dim=1), vd)
    return {"out": out, "lse": lse}
