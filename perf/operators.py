"""Operators around a decode step, with their plain forms in elementary torch operations.

A case is a plain dict.  Its "op" says what one pass computes:

  rotate   rotary positions of a layer's queries and keys: every frequency turns by its own position axis (time, height and
           width of images and video), binding.qk_norm_rope without weights
  norm     the same behind an RMS norm of every head's query and key with a weight per channel, in one pass
  shared   one layer's decode attention of a batch whose sequences share one committed prompt and have generated tokens of
           their own, Context.decode_attn_shared

The plain forms compute in 32 bits (angles in 64) and round once at the end.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"

_QK = {"q_heads": 32, "kv_heads": 8, "head_dim": 128, "dtype": "bf16", "rotary": 128, "axes": 1, "interleaved": False, "fused": True, "base": 1000000.0}
_SHARED = {"op": "shared", "q_heads": 32, "kv_heads": 8, "head_dim": 128, "dtype": "bf16", "keep_den": 16, "block": 2, "layer": 0}


def listed():
    return [
        # one generated token of a conversation about an image: the smallest call, all latency
        dict(_QK, name="rotate_token", op="rotate", n=1, axes=3),
        # a prompt with a long video: three axes, out of the fused projection's rows
        dict(_QK, name="rotate_video_16k", op="rotate", n=16383, axes=3),
        # an image encoder's patches in float32: two axes, neighbouring channels as pairs, narrow heads
        dict(_QK, name="rotate_image_f32", op="rotate", n=4097, axes=2, interleaved=True, q_heads=16, kv_heads=16, head_dim=64, rotary=64,
             dtype="f32", fused=False, base=10000.0),
        # a decode step of eight sequences
        dict(_QK, name="norm_batch8", op="norm", n=8),
        # a short prompt whose heads rotate half of their channels
        dict(_QK, name="norm_half_509", op="norm", n=509, rotary=64, base=10000.0),
        # a long prompt: the largest of these
        dict(_QK, name="norm_32k", op="norm", n=32768),
        # two continuations of a short prompt: latency again
        dict(_SHARED, name="shared_2k_batch2", T=2047, batch=2, tail=5),
        # a batch on one ragged prompt of usual length, blocks of four layers
        dict(_SHARED, name="shared_8k_block4", T=8191, batch=16, tail=64, block=4, layer=1),
        # the 32k workload's prompt with eight continuations, the second layer of a pair
        dict(_SHARED, name="shared_32k_batch8", T=32768, batch=8, tail=37, layer=1),
        # many users of one long system prompt: 256 query rows per KV head
        dict(_SHARED, name="shared_32k_batch64", T=32768, batch=64, tail=200),
        # the longest prompt of the repository's workloads
        dict(_SHARED, name="shared_128k_batch16", T=131072, batch=16, tail=129, keep_den=32),
        # float32 storage and head_dim 64, as the correctness workload has them
        dict(_SHARED, name="shared_4k_f32", T=4099, batch=6, tail=33, q_heads=4, kv_heads=2, head_dim=64, dtype="f32", keep_den=8),
    ]


def _size(rng, lo, hi):
    """A size between lo and hi, spread over its logarithm, as likely odd as not."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["rotate", "norm", "shared", "shared"])
    if op != "shared":
        d = rng.choice([64, 128, 128])
        kv = rng.choice([1, 2, 4, 8])
        return dict(_QK, op=op, n=_size(rng, 1, 32768), head_dim=d, kv_heads=kv, q_heads=min(32, kv * rng.choice([1, 2, 4, 7, 8])),
                    rotary=rng.choice([d, d, d // 2, 16, 48]), axes=rng.choice([1, 2, 3]), interleaved=rng.random() < 0.3, fused=rng.random() < 0.6,
                    dtype=rng.choice(["bf16", "bf16", "f32"]), base=rng.choice([10000.0, 1000000.0]))
    c = dict(_SHARED, T=_size(rng, 60, 131072), batch=_size(rng, 1, 64), tail=_size(rng, 1, 400) - 1, block=rng.choice([2, 2, 4]), keep_den=rng.choice([8, 16, 32]))
    c["kv_heads"] = rng.choice([2, 4, 8])
    c["q_heads"] = c["kv_heads"] * rng.choice([1, 2, 4, 4, 8])
    c["layer"] = rng.randrange(c["block"])
    if rng.random() < 0.2:  # the correctness workload's storage: shorter prompts, fewer heads
        c.update(dtype=rng.choice(["f32", "f32", "bf16"]), head_dim=64, kv_heads=2, q_heads=rng.choice([2, 4, 8]), T=_size(rng, 60, 6000), batch=_size(rng, 1, 16))
    c["T"] = max(60, min(c["T"], 64 * 32 * 32768 // (c["batch"] * c["q_heads"])))  # no more products than the largest listed case has
    return c


# ---------------------------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _positions(c, g):
    """Positions [axes, n]: a text of a few hundred tokens, then frames of patches, all behind an earlier conversation."""
    n, start = c["n"], int(torch.randint(0, 200000, (1,), generator=g, device=DEVICE))
    i = torch.arange(n, device=DEVICE)
    text = min(n, 300)
    wide = 23
    patch = (i - text).clamp(min=0)
    axes = torch.stack([text + patch // (wide * wide), text + patch // wide % wide, text + patch % wide])
    return (start + torch.where(i < text, i, axes)[: c["axes"]]).to(torch.int32).contiguous()


def _frequencies(c):
    """Frequency of every pair of channels, and the axis whose position turns it: sections of a quarter for time and the rest for
    height and width."""
    m = c["rotary"] // 2
    inv = [float(torch.tensor(c["base"] ** (-2.0 * i / c["rotary"]), dtype=torch.float32)) for i in range(m)]
    cut = [m] if c["axes"] == 1 else [m // 2, m] if c["axes"] == 2 else [m // 4, m // 4 + (m - m // 4) // 2, m]
    return inv, [next(a for a, end in enumerate(cut) if i < end) for i in range(m)]


def _depth_chain(g, T, heads, d, layers, dtype):
    """The rows [T, heads, d] of neighbouring layers: log-normal channel scales, correlated layers, a few tokens whose deviation is
    eight times as large."""
    rho = 0.7 + 0.25 * torch.rand((), generator=g, device=DEVICE)
    beta = torch.sqrt(1.0 - rho * rho)
    sigma = torch.exp(torch.randn((heads, d), generator=g, device=DEVICE))
    needle = torch.ones((T, heads), device=DEVICE)
    needle.scatter_(0, torch.randint(T, (max(1, T // 512), heads), generator=g, device=DEVICE), 8.0)
    u = torch.randn((T, heads, d), generator=g, device=DEVICE)
    out = [(u * sigma).to(dtype)]
    for _ in range(layers - 1):
        n = torch.randn((T, heads, d), generator=g, device=DEVICE)
        n.mul_(needle.unsqueeze(2)).mul_(beta)
        u = u.mul_(rho).add_(n)
        out.append((u * sigma).to(dtype))
    return out


def _modes(c):
    """Half of the heads shared, three of eight residual, the rest exact."""
    return [(0, 1, 0, 2, 0, 1, 0, 1)[h % 8] for h in range(c["kv_heads"])]


def _tails(c):
    """Generated tokens of every sequence: the longest first, down to half of it."""
    return [c["tail"] - b * c["tail"] // (2 * c["batch"]) for b in range(c["batch"])]


def _raw(c, seed):
    """What the prompt and the batch are, before anything is done with them."""
    g = _gen(seed)
    B, G, d = c["batch"], c["q_heads"] // c["kv_heads"], c["head_dim"]
    k = _depth_chain(g, c["T"], c["kv_heads"], d, c["block"], _dtype(c))
    v = _depth_chain(g, c["T"], c["kv_heads"], d, c["block"], _dtype(c))
    q = torch.randn((B, c["kv_heads"] * G, d), generator=g, device=DEVICE).to(_dtype(c))
    tk, tv = (torch.randn((B, c["tail"], c["kv_heads"], d), generator=g, device=DEVICE).to(_dtype(c)) for _ in range(2))
    return k, v, q, tk, tv


def _compressed(c, x):
    """The committed form of one tensor's layers for the case's layer: rows [heads, T, d], and of the residual heads the kept
    positions and what is added there."""
    f = [t.float().transpose(0, 1).contiguous() for t in x]
    at = c["layer"]
    if c["block"] == 2:
        c32 = torch.tensor(math.sqrt(0.5), dtype=torch.float32, device=DEVICE)
        z0, dev = ((f[0] + f[1]) * c32).to(x[0].dtype), ((f[0] - f[1]) * c32).to(x[0].dtype)
        key, dev, sign = dev.abs(), dev, 1.0 if at == 0 else -1.0
    else:
        z0 = (((f[0] + f[1]) + (f[2] + f[3])) * 0.5).to(x[0].dtype)
        devs = [(t - 0.5 * z0.float()).to(x[0].dtype) for t in f]
        e = [t.float() * t.float() for t in devs]
        key, dev, sign = (e[0] + e[1]) + (e[2] + e[3]), devs[at], 2.0  # (rows count half, deviations whole)
    modes = _modes(c)
    rows = torch.stack([x[at][:, h] if m == 2 else z0[h] for h, m in enumerate(modes)])
    keep = c["T"] * c["head_dim"] // c["keep_den"]
    idx, val = [], []
    for h, m in enumerate(modes):
        if m == 1:  # the largest, ties to the lowest index
            i = key[h].reshape(-1).sort(descending=True, stable=True).indices[:keep].sort().values
            idx.append(i)
            val.append(sign * dev[h].reshape(-1)[i].float())
    return rows, torch.stack(idx), torch.stack(val)


def prepare(case, seed):
    c = case
    if c["op"] != "shared":
        g = _gen(seed)
        n, Hq, Hk, d = c["n"], c["q_heads"], c["kv_heads"], c["head_dim"]
        s = {"case": c, "pos": _positions(c, g)}
        if c["fused"]:  # queries and keys as the fused projection leaves them, the values behind
            qkv = torch.randn((n, Hq + 2 * Hk, d), generator=g, device=DEVICE).mul_(2.0).to(_dtype(c))
            s["q"], s["k"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hk]
        else:
            s["q"], s["k"] = (torch.randn((n, h, d), generator=g, device=DEVICE).mul_(2.0).to(_dtype(c)) for h in (Hq, Hk))
        s["qw"], s["kw"] = ((1.0 + 0.3 * torch.randn((d,), generator=g, device=DEVICE)).to(_dtype(c)) if c["op"] == "norm" else None for _ in range(2))
        s["q_out"], s["k_out"] = (torch.empty((n, h, d), dtype=_dtype(c), device=DEVICE) for h in (Hq, Hk))
        inv, axis = _frequencies(c)
        if own:
            from paper_2607_06519_b200 import binding as B

            s["rotary"] = B.Rotary(inv, axis_of=axis, n_axes=c["axes"], interleaved=c["interleaved"], q_weight=s["qw"], k_weight=s["kw"], eps=1e-6)
        else:
            s["inv"], s["axis"] = torch.tensor(inv, dtype=torch.float32, device=DEVICE), torch.tensor(axis, device=DEVICE)
        return s
    k, v, q, tk, tv = _raw(c, seed)
    s = {"case": c, "q": q, "out": torch.empty_like(q)}
    tails = _tails(c)
    if own:
        from paper_2607_06519_b200 import binding as B

        one = (c["block"], c["q_heads"], c["kv_heads"], c["head_dim"], 1, c["T"], c["tail"] + 1, B.BF16 if c["dtype"] == "bf16" else B.F32, 1, c["keep_den"],
               B.RESIDUAL_ENTRIES, c["block"])
        many = one[:4] + (c["batch"],) + one[5:]
        rows = (c["tail"] + 128) // 128 * 128
        tail_bytes = 2 * c["block"] * c["kv_heads"] * (rows * c["head_dim"] * q.element_size() + 256)
        ctx = B.Context(B.Config(*many), device=DEVICE, arena_bytes=B.sizes(B.Config(*one))[0] + c["batch"] * tail_bytes + (1 << 20))
        ctx.compress_prefill(0, 0, 1, c["T"], k, v)
        ctx.set_modes(0, [_modes(c)])
        ctx.commit(0)
        for b, n in enumerate(tails):
            if n:
                ctx.append_tail(c["layer"], b, tk[b, :n], tv[b, :n])
        s["ctx"], s["seqs"] = ctx, torch.arange(c["batch"], dtype=torch.int32)
    else:
        s["k"], s["v"] = _compressed(c, k), _compressed(c, v)
        s["tk"], s["tv"] = tk, tv
        s["tails"] = torch.tensor(tails, device=DEVICE)
        s["residual"] = torch.tensor([h for h, m in enumerate(_modes(c)) if m == 1], device=DEVICE)
        s["scale"] = torch.tensor([1.0 if m == 2 else math.sqrt(0.5) if c["block"] == 2 else 0.5 for m in _modes(c)], device=DEVICE)
    return s


# ---------------------------------------------------------------------------------------------------------------- a pass
def _turned(x, weight, cos, sin, c):
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6) * weight.float()
    r = c["rotary"]
    if c["interleaved"]:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
    else:
        a, b = y[..., : r // 2], y[..., r // 2: r]
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turned, y[..., r:]], -1).to(x.dtype)


def _dense(packed, s):
    rows, idx, val = packed
    x = rows.to(torch.float32, copy=True)  # (float32 rows would be added to where they lie)
    flat = x.view(len(rows), -1)
    flat[s["residual"].unsqueeze(1), idx] += val
    return x * s["scale"][:, None, None]


def run(state):
    s, c = state, state["case"]
    if c["op"] != "shared":
        if own:
            from paper_2607_06519_b200 import binding as B

            return B.qk_norm_rope(s["rotary"], s["q"], s["k"], s["pos"], q_out=s["q_out"], k_out=s["k_out"])
        angle = s["pos"].double()[s["axis"]].T * s["inv"].double()
        cos, sin = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)
        return _turned(s["q"], s["qw"], cos, sin, c), _turned(s["k"], s["kw"], cos, sin, c)
    if own:
        return s["ctx"].decode_attn_shared(c["layer"], 0, s["seqs"], s["q"], out=s["out"])
    B, H, d = c["batch"], c["kv_heads"], c["head_dim"]
    G = c["q_heads"] // H
    q = s["q"].float().view(B, H, G, d).permute(1, 0, 2, 3)  # [H, B, G, d]
    prefix = (q.reshape(H, B * G, d) @ _dense(s["k"], s).transpose(1, 2)).view(H, B, G, -1)
    tail = q @ s["tk"].float().permute(2, 0, 3, 1)
    dead = torch.arange(c["tail"], device=DEVICE) >= s["tails"][:, None, None]
    tail = tail.masked_fill(dead, -math.inf)
    p = torch.cat([prefix, tail], -1) / math.sqrt(d)
    p = torch.exp(p - p.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    out = (p[..., : c["T"]].reshape(H, B * G, -1) @ _dense(s["v"], s)).view(H, B, G, d) + p[..., c["T"]:] @ s["tv"].float().permute(2, 0, 1, 3)
    return out.permute(1, 0, 2, 3).reshape(B, H * G, d).to(s["q"].dtype)


# ------------------------------------------------------------------------------------------------------ floors and 64 bits
def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] != "shared":
        values = c["n"] * (c["q_heads"] + c["kv_heads"]) * c["head_dim"]
        return {"bytes": 2 * values * e + 4 * c["axes"] * c["n"], "flops": values * (3 + (4 if c["op"] == "norm" else 0))}
    H, d, tails = c["kv_heads"], c["head_dim"], sum(_tails(c))
    kept = c["T"] * d // c["keep_den"]
    # dense rows, the residual heads' entries (a value and a 16-bit position), the tails, queries and outputs
    by = H * 2 * c["T"] * d * e + _modes(c).count(1) * 2 * kept * (e + 2) + 2 * H * tails * d * e + 2 * c["batch"] * c["q_heads"] * d * e
    return {"bytes": by, "flops": 4 * c["q_heads"] * d * (c["batch"] * c["T"] + tails)}


def _exact_heads(c, x):
    """The layer's reconstructed rows [head][T, d] in 64 bits, from the definition: the coefficients as they are stored, the kept
    ones by a key that has the index in its low bits."""
    dt, keep, out = x[0].dtype, c["T"] * c["head_dim"] // c["keep_den"], []
    for h, mode in enumerate(_modes(c)):
        t = [y[:, h].float() for y in x]
        if mode == 2:
            out.append(t[c["layer"]].double())
            continue
        if c["block"] == 2:
            c32 = float(torch.tensor(math.sqrt(0.5), dtype=torch.float32))
            z0 = torch.mul(t[0] + t[1], c32).to(dt).double()
            z1 = torch.mul(t[0] - t[1], c32).to(dt)
            size, add = z1.float().abs(), (z1.double() if c["layer"] == 0 else -z1.double())
            scale = math.sqrt(0.5)
        else:
            z0 = torch.mul((t[0] + t[1]) + (t[2] + t[3]), 0.5).to(dt)
            dev = [(y - torch.mul(z0.float(), 0.5)).to(dt) for y in t]
            sq = [torch.square(y.float()) for y in dev]
            size, add = (sq[0] + sq[1]) + (sq[2] + sq[3]), 2.0 * dev[c["layer"]].double()
            z0, scale = z0.double(), 0.5
        if mode == 1 and keep:
            n = size.numel()
            order = (size.reshape(-1).view(torch.int32).long() << 32) + (n - 1 - torch.arange(n, device=DEVICE))
            chosen = torch.topk(order, keep, sorted=False).indices
            z0.view(-1)[chosen] += add.reshape(-1)[chosen]
        out.append(z0 * scale)
    return out


def exact(case, seed):
    c = case
    if c["op"] != "shared":
        s = prepare(case, seed)
        inv, axis = _frequencies(c)
        turn = s["pos"].double()[torch.tensor(axis, device=DEVICE)] * torch.tensor(inv, dtype=torch.float64, device=DEVICE)[:, None]  # [pairs, n]
        got = []
        for x, w in ((s["q"], s["qw"]), (s["k"], s["kw"])):
            y = x.double()
            if w is not None:
                y = y / torch.sqrt((y ** 2).sum(-1, keepdim=True) / c["head_dim"] + 1e-6) * w.double()
            z = y.clone()
            for i in range(c["rotary"] // 2):
                a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + c["rotary"] // 2)
                co, si = torch.cos(turn[i])[:, None], torch.sin(turn[i])[:, None]
                z[..., a] = y[..., a] * co - y[..., b] * si
                z[..., b] = y[..., b] * co + y[..., a] * si
            got.append(z)
        return got[0], got[1]
    k, v, q, tk, tv = _raw(c, seed)
    kh, vh = _exact_heads(c, k), _exact_heads(c, v)
    G, d, tails = c["q_heads"] // c["kv_heads"], c["head_dim"], _tails(c)
    out = torch.empty(q.shape, dtype=torch.float64, device=DEVICE)
    for h in range(c["kv_heads"]):
        for b in range(c["batch"]):
            keys = torch.cat([kh[h], tk[b, : tails[b], h].double()])
            values = torch.cat([vh[h], tv[b, : tails[b], h].double()])
            logits = q[b, h * G:(h + 1) * G].double() @ keys.T / math.sqrt(d)
            out[b, h * G:(h + 1) * G] = torch.softmax(logits, -1) @ values
    return out
