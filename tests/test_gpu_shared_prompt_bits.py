"""Float32 outputs of the tensor-core form of attention on a shared prompt: probabilities of 16 bits, as fdkv_decode_attn has them."""
import pytest
import torch

from shared_util import Prompt, put_tails, random_tails

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def _reference(p, layer, q, tails):
    """shared_util's reference and tolerance with 2^-16 of sum p |v| for a probability's rounding in place of 2^-8: the bf16 value leaves up to 2^-8 of it, and the
    bf16 value of that up to 2^-8 of what is left."""
    p.dtype = torch.float32  # (leaves the 2^-8 out)
    ref, tol = p.reference(layer, q, tails)
    p.dtype = BF
    rows = [torch.cat([p.rows[layer][1][h], tails[i][1][:, h].double()]).abs() for i in range(len(q)) for h in range(p.hkv)]
    keys = [torch.cat([p.rows[layer][0][h], tails[i][0][:, h].double()]) for i in range(len(q)) for h in range(p.hkv)]
    qq = q.double().view(-1, p.G, p.d)
    extra = torch.stack([torch.softmax(qq[n] @ keys[n].T / p.d ** 0.5, -1) @ rows[n] for n in range(len(rows))])
    return ref, tol + 2.0 ** -16 * extra.view_as(ref)


def _run(p, layer, seqs, lens, scale):
    tails = random_tails(p, lens)
    put_tails(p, layer, seqs, tails)
    q = p.new(len(seqs), p.G * p.hkv, p.d, scale=scale)
    out = p.ctx.decode_attn_shared(layer, p.slot, seqs, q, out_dtype=0)
    ref, tol = _reference(p, layer, q, tails)
    worst = float(((out.double() - ref).abs() / tol).max())
    assert worst <= 1.0, worst


@pytest.mark.parametrize("block,rule,keep", [(2, 0, (1, 8)), (2, 1, (1, 8)), (4, 0, (1, 16)), (4, 1, (1, 4)), (2, 0, (1, 1)), (2, 0, (0, 1))])
@pytest.mark.parametrize("scale", [0.02, 1.0])
def test_modes_blocks_and_rules(block, rule, keep, scale):
    p = Prompt(1111, 4, 3, 128, BF, block=block, rule=rule, keep=keep, seed=80)
    for layer in range(block):
        _run(p, layer, [2, 0, 3], [7, 0, 90], scale)
    p.close()


@pytest.mark.parametrize("T,batch,G", [(1, 3, 1), (130, 5, 8), (9001, 7, 4), (3001, 40, 4), (2000, 70, 2)])
@pytest.mark.parametrize("scale", [0.02, 1.0])
def test_lengths_and_row_groups(T, batch, G, scale):
    p = Prompt(T, G, 4, 128, BF, modes=[1, 2, 0, 1], max_batch=batch, seed=81)
    _run(p, 1, list(range(batch)), [(11 * b) % 60 for b in range(batch)], scale)
    p.close()


def test_single_sequence_agrees_with_the_ordinary_call():
    """Both within 2^-15 of sum p |v| of one another (2^-16 each, and float32 sums)."""
    p = Prompt(4000, 4, 3, 128, BF, seed=82)
    q = p.new(1, 12, 128, scale=0.02)
    a, b = p.ctx.decode_attn_shared(0, 0, [0], q, out_dtype=0), p.ctx.decode_attn(0, q, out_dtype=0)
    ref, tol = _reference(p, 0, q, random_tails(p, [0]))
    assert ((a.double() - b.double()).abs() <= 2 * tol).all()
    p.close()
