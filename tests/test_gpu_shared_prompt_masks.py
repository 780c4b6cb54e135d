"""Decode attention on a shared prompt whose keys put tokens infinitely far off, or as far as finite numbers go: whole tiles of them, in front of, between and
behind others, for all queries or for some.  References: 64 bits, over the tokens that remain."""
import pytest
import torch

from shared_util import Prompt, chain, put_tails, random_tails

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
INF = float("inf")


def _dead(kind, T, seed):
    dead = torch.zeros(T, dtype=torch.bool)
    if kind == "first":
        dead[:128] = True
    elif kind == "middle":
        dead[128:384] = True
    elif kind == "tiles":  # every other one, at random
        g = torch.Generator().manual_seed(seed)
        dead = (torch.rand((T + 127) // 128, generator=g) < 0.5).repeat_interleave(128)[:T]
        dead[-1] = False
    elif kind == "all":
        dead[:] = True
    return dead.cuda()


def _prompt(T, G, hkv, d, dtype, modes, dead, low, seed, max_batch=8):
    g = torch.Generator(device="cuda").manual_seed(seed + 100)
    k, v = chain(g, T, hkv, d, 2, dtype), chain(g, T, hkv, d, 2, dtype)
    for x in k:
        x[dead, :, 0] = low
    return Prompt(T, G, hkv, d, dtype, modes=modes, max_batch=max_batch, seed=seed, kv=(k, v))


def _check(p, got, layer, q, tails, dead):
    """Rows of q whose first channel is not zero do not see the dead tokens."""
    whole = p.rows[layer]
    every = p.reference(layer, q, tails) if (q[..., 0] == 0).any() else None
    p.rows[layer] = tuple([x[~dead] for x in side] for side in whole)
    ref, tol = p.reference(layer, q, tails)
    p.rows[layer] = whole
    if every is not None:
        sees = (q[..., :1] == 0).expand_as(ref)
        ref, tol = torch.where(sees, every[0], ref), torch.where(sees, every[1], tol)
    if got.dtype == BF:
        tol = tol + 2.0 ** -8 * ref.abs()
    err = (got.double() - ref).abs()
    assert (err <= tol).all(), (int((~(err <= tol)).sum()), int(got.isnan().sum()), err.numel())


KINDS = {"infinite": (-INF, (1.0, 2.0)), "overflows": ("lowest", (2.0,)), "finite": ("lowest", (0.5,)), "some_queries": ("lowest", (0.0, 2.0, 0.5))}


def _run(p, layer, seqs, lens, dead, first_channel, scale=1.0):
    tails = random_tails(p, lens)
    for k, _ in tails:
        k[:, :, 0] = 0
    put_tails(p, layer, seqs, tails)
    q = p.new(len(seqs), p.G * p.hkv, p.d, scale=scale)
    c = torch.tensor(first_channel, device="cuda")
    q[..., 0] = c[torch.arange(q[..., 0].numel(), device="cuda") % len(c)].view_as(q[..., 0]).to(q.dtype)
    for out_dtype in (0, None):
        _check(p, p.ctx.decode_attn_shared(layer, 0, seqs, q, out_dtype=out_dtype), layer, q, tails, dead)
    return q, tails


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("where", ["first", "middle", "tiles"])
@pytest.mark.parametrize("dtype,d", [(BF, 128), (F, 64), (BF, 64)])
def test_tiles_that_no_query_sees(kind, where, dtype, d):
    low, first_channel = KINDS[kind]
    low = torch.finfo(dtype).min if low == "lowest" else low
    dead = _dead(where, 1000, 3)
    p = _prompt(1000, 4, 2, d, dtype, [2, 2] if kind == "some_queries" else [2, 0], dead, low, 50)
    _run(p, 1, [0, 3, 2], [0, 17, 130], dead, first_channel)
    _run(p, 0, [1, 4], [0, 300], dead, first_channel, scale=8.0)
    p.close()


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("batch,scale", [(8, 1.0), (8, 8.0), (40, 1.0)])
def test_blocks_that_meet_them_before_and_between_others(kind, batch, scale):
    """Many tiles a block: the exponents' reference is set by a later tile, or moved over the whole range of float32."""
    low, first_channel = KINDS[kind]
    low = torch.finfo(BF).min if low == "lowest" else low
    dead = _dead("tiles", 20011, 4)
    p = _prompt(20011, 4, 8, 128, BF, [2] * 8 if kind == "some_queries" else [2, 0, 2, 2, 0, 0, 2, 2], dead, low, 51, max_batch=batch)
    _run(p, 1, list(range(batch)), [(7 * b) % 50 for b in range(batch)], dead, first_channel, scale=scale)
    p.close()


@pytest.mark.parametrize("dtype,d", [(BF, 128), (F, 64), (BF, 64)])
def test_prompts_that_no_query_sees(dtype, d):
    """Tails alone; and zeros where a sequence has none, as fdkv_decode_attn gives."""
    dead = _dead("all", 700, 0)
    p = _prompt(700, 4, 2, d, dtype, [2, 0], dead, -INF, 52)
    q, _ = _run(p, 0, [1, 2], [5, 200], dead, (1.0, 2.0))
    none = p.ctx.decode_attn_shared(0, 0, [3, 0], q)
    assert (none == 0).all()
    assert torch.equal(none[1:], p.ctx.decode_attn(0, q[1:].contiguous()))
    p.close()


@pytest.mark.parametrize("dtype,d", [(BF, 128), (F, 64), (BF, 64)])
def test_the_lowest_finite_logit_everywhere(dtype, d):
    """Equal logits, of -1.7e38 / sqrt(d) each: the mean of all values.  The sums are exact but for their own roundings (n 2^-24), the output's and the division's."""
    T, n = 700, 90
    low = torch.finfo(dtype).min
    p = _prompt(T, 4, 2, d, dtype, [2, 2], _dead("all", T, 0), low, 53)
    tails = random_tails(p, [0, n])
    tails[1][0][:, :, 0] = low
    put_tails(p, 1, [1, 2], tails)
    q = torch.zeros((2, 8, d), dtype=dtype, device="cuda")
    q[..., 0] = 0.5
    out = p.ctx.decode_attn_shared(1, 0, [1, 2], q, out_dtype=0).double()
    for b in range(2):
        for h in range(2):
            v = torch.cat([p.rows[1][1][h], tails[b][1][:, h].double()])
            err = (out[b, 4 * h:4 * h + 4] - v.mean(0)).abs()
            assert (err <= (len(v) + 4) * 2.0 ** -24 * v.abs().mean(0)).all(), (b, h, float(err.max()))
    p.close()
