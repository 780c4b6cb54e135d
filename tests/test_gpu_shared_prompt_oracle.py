"""Attention on a shared prompt against the rows of the CPU oracle (its coefficients, its kept sets, its folded chunks) instead of what the library staged: several
sequences with tails, every mode, both block sizes, folds; and values that cancel in their two addends."""
import math

import numpy as np
import pytest
import torch

from oracle import fdkv_ref as R
from oracle import fdkv_ref_b4 as R4
from shared_util import Prompt, chain, put_tails, random_tails

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def _np(x):
    return x.float().cpu().numpy()


def _units(p, keep):
    bf16 = p.dtype == BF
    if p.block == 2:
        return [R.Unit(*[_np(x[:, h]) for x in (*p.k, *p.v)], bf16, *keep) for h in range(p.hkv)]
    return [R4.Unit4([_np(x[:, h]) for x in p.k], [_np(x[:, h]) for x in p.v], bf16, *keep) for h in range(p.hkv)]


def _take_rows(p, units):
    """The oracle's rows without the tails in place of the prompt's."""
    for l in range(p.block):
        for is_v, name in enumerate("kv"):
            for h, u in enumerate(units):
                p.rows[l][is_v][h] = torch.from_numpy(np.asarray(u.rows(name, p.modes[h], l)[:u.T], dtype=np.float64)).cuda()


@pytest.mark.parametrize("modes", [[0, 1, 2], [1, 1, 1]])
@pytest.mark.parametrize("dtype,d,G", [(BF, 128, 4), (F, 64, 2), (BF, 64, 8), (F, 128, 1)])
@pytest.mark.parametrize("block,keep", [(2, (1, 8)), (4, (1, 16))])
def test_sequences_with_tails(modes, dtype, d, G, block, keep):
    p = Prompt(531, G, 3, d, dtype, block=block, keep=keep, modes=modes, max_batch=5, seed=90)
    _take_rows(p, _units(p, keep))
    for layer in range(block):
        tails = random_tails(p, [0, 19, 140])
        put_tails(p, layer, [4, 0, 2], tails)
        for out_dtype in (0, 1):
            q = p.new(3, G * 3, d)
            p.check(p.ctx.decode_attn_shared(layer, 0, [4, 0, 2], q, out_dtype=out_dtype), layer, q, tails)
    p.close()


@pytest.mark.parametrize("modes", [[2, 2], [0, 1], [1, 1]])
@pytest.mark.parametrize("dtype,d", [(BF, 128), (F, 64)])
@pytest.mark.parametrize("block,keep", [(2, (1, 8)), (4, (1, 8))])
def test_folds(modes, dtype, d, block, keep):
    """Rows appended in bulk to the prompt's own slot, 96 of them folded into it in two steps: the prompt of every sequence then, and the rest still the slot's."""
    p = Prompt(320, 4, 2, d, dtype, block=block, keep=keep, modes=modes, max_batch=3, max_tail=130, max_fold=96, max_prefill=416, seed=91)
    units = _units(p, keep)
    own = [random_tails(p, [110])[0] for _ in range(block)]
    for l in range(block):
        p.ctx.append_tail(l, 0, *own[l])
        for h, u in enumerate(units):
            for t in range(110):
                u.append(l, _np(own[l][0][t, h]), _np(own[l][1][t, h]))
    other = random_tails(p, [37])[0]
    folded = 0
    for n in (0, 64, 32):
        if n:
            p.ctx.fold_tail(0, n)
            for u in units:
                u.fold(n, *keep)
        folded += n
        _take_rows(p, units)
        for l in range(block):
            if not n:
                p.ctx.append_tail(l, 2, *other)
            q = p.new(3, 8, d)
            tails = [(other[0], other[1]), (own[l][0][folded:], own[l][1][folded:]), random_tails(p, [0])[0]]
            for out_dtype in (0, 1):
                p.check(p.ctx.decode_attn_shared(l, 0, [2, 0, 1], q, out_dtype=out_dtype), l, q, tails)
            p.check(p.ctx.decode_attn(l, q[:1], out_dtype=0), l, q[:1], tails[1:2])
    p.close()


@pytest.mark.parametrize("dtype,d,G", [(BF, 128, 4), (F, 64, 2), (F, 128, 4), (BF, 64, 4)])
@pytest.mark.parametrize("T", [300, 5000])
def test_values_that_cancel_in_their_addends(dtype, d, G, T):
    """The second layer's rows are 2^-14 of the first's: differences of two coefficients.  The addends' products are summed apart (the tensor cores) or the addends are
    (float32), so that the tolerance takes the addends' size where a rounding is of their sums: with |z0| + |z1| of a key in place of its size for the logits, and n 2^-24 of the
    addends' weighted mean for the outputs' sums; a probability's rounding is the same for both, so that it counts with the values."""
    g = torch.Generator(device="cuda").manual_seed(92)
    k, v = chain(g, T, 2, d, 1, dtype), chain(g, T, 2, d, 1, dtype)
    for x in (k, v):
        x.append((x[0].float() * torch.randn(x[0].shape, generator=g, device="cuda") * 2.0 ** -14).to(dtype))
    p = Prompt(T, G, 2, d, dtype, keep=(1, 1), modes=[1, 1], seed=93, kv=(k, v))
    seqs, lens = [1, 2], [0, 33]
    tails = random_tails(p, lens)
    for t in tails:
        t[1].mul_(2.0 ** -14)
    put_tails(p, 1, seqs, tails)
    for out_dtype in (0, 1):
        q = p.new(2, 2 * G, d)
        out = p.ctx.decode_attn_shared(1, 0, seqs, q, out_dtype=out_dtype).double()
        for b in range(2):
            for h in range(2):
                size = [torch.cat([x[0][:, h].double().abs() * (1 + 2.0 ** -7), t[:, h].double().abs()]) for x, t in ((k, tails[b][0]), (v, tails[b][1]))]
                kk, vv = (torch.cat([p.rows[1][i][h], tails[b][i][:, h].double()]) for i in range(2))
                qq = q[b, h * G:(h + 1) * G].double()
                pr = torch.softmax(qq @ kk.T / math.sqrt(d), -1)
                mag = (qq.abs() @ size[0].T / math.sqrt(d)).amax(-1, keepdim=True)
                ref = pr @ vv
                bits = 0 if d == 64 or dtype == F else 2.0 ** -16 if out_dtype == 0 else 2.0 ** -8
                tol = (2 * (d * 2.0 ** -23 + 4 * 2.0 ** -24) * mag + bits) * (pr @ vv.abs()) + len(kk) * 2.0 ** -24 * (pr @ size[1])
                if out_dtype == 1:
                    tol = tol + 2.0 ** -8 * ref.abs()
                err = (out[b, h * G:(h + 1) * G] - ref).abs()
                assert (err <= tol).all(), float((err / tol).max())
    p.close()
