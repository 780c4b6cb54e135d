"""Reference for decode attention on one shared prompt: the committed prompt's rows in 64 bits, out of what the library says it staged
(its own tests compare that with the oracle bit for bit), and attention over them and a sequence's tail."""
import math

import numpy as np
import torch


def chain(g, T, heads, d, layers, dtype):
    u = torch.randn((T, heads, d), generator=g, device="cuda")
    sigma = torch.exp(0.7 * torch.randn((heads, d), generator=g, device="cuda"))
    out = [(u * sigma).to(dtype)]
    for _ in range(layers - 1):
        u = 0.8 * u + 0.6 * torch.randn((T, heads, d), generator=g, device="cuda")
        out.append((u * sigma).to(dtype))
    return out


class Prompt:
    """A context whose slot `slot` holds a committed prompt of one block of layers, and the rows of every layer in float64."""

    def __init__(self, T, G, hkv, d, dtype, block=2, rule=0, keep=(1, 8), modes=None, max_batch=4, max_tail=300, slot=0, seed=0, max_fold=0, row_format=0,
                 max_prefill=None, device="cuda:0", kv=None):
        from paper_2607_06519_b200 import binding as B

        self.B, self.T, self.G, self.hkv, self.d, self.dtype, self.slot, self.block = B, T, G, hkv, d, dtype, slot, block
        cfg = B.Config(block, G * hkv, hkv, d, max_batch, max_prefill or T, max_tail, B.BF16 if dtype == torch.bfloat16 else B.F32, keep[0], keep[1], rule, block, max_fold,
                       row_format)
        self.ctx = B.Context(cfg, device=device)
        g = self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.k, self.v = kv or (chain(g, T, hkv, d, block, dtype), chain(g, T, hkv, d, block, dtype))
        self.modes = [h % 3 for h in range(hkv)] if modes is None else modes
        ctx = self.ctx
        ctx.compress_prefill(slot, 0, 1, T, self.k, self.v)
        if rule == 1:
            W = min(8, T)
            ctx.probe(slot, 0, 1, [torch.randn((W, G * hkv, d), generator=g, device="cuda").to(dtype) for _ in range(block)], list(range(T - W, T)), 0.0)
        ctx.set_modes(slot, self.modes)
        self.rows = [([None] * hkv, [None] * hkv) for _ in range(block)]
        for h, m in enumerate(self.modes):
            for is_v, x in enumerate((self.k, self.v)):
                z0 = ctx.get_shared(slot, 0, h, is_v, T).double()
                if m == 1 and rule == 0:
                    idx, val = ctx.get_residual(slot, 0, h, is_v)
                elif m == 1:
                    tok = ctx.get_token_set(slot, 0, h, T)[0].long()
                for l in range(block):
                    if m == 2:
                        r = x[l][:, h].double()
                    else:
                        r = z0.clone()
                        if m == 1 and rule == 0:
                            add = (val if block == 2 else val[l]).double()
                            r.view(-1)[idx.long()] += add * ((1, -1)[l] if block == 2 else 2)
                        elif m == 1:
                            f = [t[:, h].float() for t in x]
                            if block == 2:
                                dev = ((f[0] - f[1]) * torch.tensor(math.sqrt(0.5), dtype=torch.float32, device="cuda")).to(dtype).double() * (1, -1)[l]
                            else:
                                dev = (f[l] - 0.5 * z0.float()).to(dtype).double() * 2
                            r[tok] += dev[tok]
                        r *= math.sqrt(0.5) if block == 2 else 0.5
                    self.rows[l][is_v][h] = r
        ctx.commit(slot)

    def new(self, *shape, scale=1.0):
        return (scale * torch.randn(shape, generator=self.g, device="cuda")).to(self.dtype)

    def reference(self, layer, q, tails):
        """(out, tolerance) float64 [batch, Hq, d] for queries q and tails[b] = (k, v) rows [n, Hkv, d]: with A = sum_t p_t |v_t|
          - a logit of d products is off by at most d 2^-23 (twice a rounding: the tensor core cuts) of sum |q_i k_i| / sqrt(d), its
            scaling and the exponential's argument by 4 roundings of its own size: that moves p, above and below, by twice as much;
          - the sums over the tokens by n 2^-24 A;
          - bf16 storage with 128 channels rounds p to bf16 (2^-8 of it); a bf16 output once more."""
        b, hq, d = q.shape
        out = torch.empty((b, hq, d), dtype=torch.float64, device="cuda")
        tol = torch.empty_like(out)
        for i in range(b):
            for h in range(self.hkv):
                k = torch.cat([self.rows[layer][0][h], tails[i][0][:, h].double()])
                v = torch.cat([self.rows[layer][1][h], tails[i][1][:, h].double()])
                qq = q[i, h * self.G:(h + 1) * self.G].double()
                s = qq @ k.T / math.sqrt(d)
                p = torch.softmax(s, -1)
                mag = (qq.abs() @ k.abs().T / math.sqrt(d)).amax(-1, keepdim=True)
                A = p @ v.abs()
                out[i, h * self.G:(h + 1) * self.G] = p @ v
                rel = 2 * (d * 2.0 ** -23 * mag + 4 * 2.0 ** -24 * mag) + len(k) * 2.0 ** -24
                if self.dtype == torch.bfloat16 and d == 128:
                    rel = rel + 2.0 ** -8
                tol[i, h * self.G:(h + 1) * self.G] = rel * A
        return out, tol

    def check(self, got, layer, q, tails):
        ref, tol = self.reference(layer, q, tails)
        if got.dtype == torch.bfloat16:
            tol = tol + 2.0 ** -8 * ref.abs()
        err = (got.double() - ref).abs()
        assert (err <= tol).all(), (float((err / tol).max()), int((err > tol).sum()), err.numel())
        return float((err / tol).max())

    def close(self):
        assert self.ctx.device_status() == 0
        self.ctx.close()


def random_tails(p, lens):
    return [(p.new(n, p.hkv, p.d), p.new(n, p.hkv, p.d)) for n in lens]


def put_tails(p, layer, seqs, tails):
    for s, (k, v) in zip(seqs, tails):
        p.ctx.append_tail(layer, s, k, v)
