"""Decode attention of a batch on one committed prompt (fdkv_decode_attn_shared), rows appended in bulk (fdkv_append_tail) and the
step from a fused projection row (fdkv_decode_qkv), against 64-bit references; tolerances are derived in shared_util.Prompt.reference."""
import numpy as np
import pytest
import torch

from shared_util import Prompt, put_tails, random_tails

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def _run(p, layer, seqs, lens, out_dtype=None, scale=1.0):
    tails = random_tails(p, lens)
    put_tails(p, layer, seqs, tails)
    q = p.new(len(seqs), p.G * p.hkv, p.d, scale=scale)
    out = p.ctx.decode_attn_shared(layer, p.slot, seqs, q, out_dtype=out_dtype)
    p.check(out, layer, q, tails)
    return q, out, tails


@pytest.mark.parametrize("T", [1, 15, 16, 17, 127, 128, 129, 300, 1000])
@pytest.mark.parametrize("dtype,d,G,block", [(F, 64, 2, 2), (BF, 128, 4, 2), (BF, 64, 1, 4), (F, 128, 8, 4)])
def test_lengths(T, dtype, d, G, block):
    """From one token to ragged ones; tails of none, one and some rows; a batch of one."""
    p = Prompt(T, G, 3, d, dtype, block=block, max_batch=6, seed=T)
    _run(p, 0, [0, 3, 5, 1], [0, 1, 37, 130])
    _run(p, block - 1, [2], [0], out_dtype=0)
    p.close()


@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("dtype,d", [(F, 64), (F, 128), (BF, 64), (BF, 128)])
@pytest.mark.parametrize("block,rule", [(2, 0), (2, 1), (4, 0), (4, 1)])
def test_groups_types_blocks_and_rules(G, dtype, d, block, rule):
    p = Prompt(517, G, 3, d, dtype, block=block, rule=rule, max_batch=4, seed=G)
    for layer in range(block):
        _run(p, layer, [1, 0, 2], [5, 70, 0], out_dtype=layer & 1)
    p.close()


@pytest.mark.parametrize("batch,G,T", [(33, 1, 700), (40, 4, 1500), (130, 2, 130), (64, 8, 260), (17, 8, 5000)])
@pytest.mark.parametrize("dtype,d", [(BF, 128), (F, 64)])
def test_many_query_rows(batch, G, T, dtype, d):
    """Batches whose rows fill several row groups, the last of them partly."""
    p = Prompt(T, G, 2, d, dtype, max_batch=batch + 3, max_tail=140, modes=[1, 2], seed=batch)
    seqs = list(np.random.default_rng(batch).permutation(batch + 3)[:batch])
    lens = [(7 * b) % 90 if b % 5 else 0 for b in range(batch)]
    seqs = [int(s) for s in seqs]
    _run(p, 1, seqs, lens)
    p.close()


@pytest.mark.parametrize("dtype,d", [(BF, 128), (F, 64)])
@pytest.mark.parametrize("keep", [(0, 1), (1, 64), (1, 2), (1, 1)])
def test_kept_fractions(dtype, d, keep):
    p = Prompt(419, 4, 2, d, dtype, keep=keep, modes=[1, 0], seed=9)
    _run(p, 0, [0, 1, 2], [3, 0, 129])
    p.close()
    p = Prompt(419, 2, 2, d, dtype, block=4, rule=1, keep=keep, modes=[1, 1], seed=10)
    _run(p, 2, [0, 1, 2], [3, 0, 129])
    p.close()


@pytest.mark.parametrize("hkv,modes", [(1, [1]), (8, [0, 1, 2, 1, 0, 2, 2, 1]), (5, [2] * 5), (4, [1] * 4)])
def test_long_prompts_of_every_mode(hkv, modes):
    p = Prompt(9001, 4, hkv, 128, BF, modes=modes, keep=(1, 16), max_batch=8, seed=hkv)
    _run(p, 0, [0, 1, 2, 3, 4], [0, 300, 16, 128, 129])
    _run(p, 1, [7, 2], [1, 255])
    p.close()


def test_blocks_that_walk_many_tiles_of_heads_in_different_modes():
    """Some twenty tiles per block, whose range runs from a head in one mode into a head in another (the ring of shared memory goes round several
    times in either), with calls of two contexts behind one another and nothing that waits between."""
    a = Prompt(41000, 4, 8, 128, BF, modes=[0, 1, 2, 1, 0, 0, 1, 2], keep=(1, 16), max_batch=8, seed=21)
    b = Prompt(33333, 8, 8, 128, BF, block=4, modes=[1, 2, 2, 0, 1, 1, 0, 1], keep=(1, 32), max_batch=18, seed=22)
    calls = []
    for p, layer, n in ((a, 1, 8), (b, 3, 17)):
        tails = random_tails(p, [(5 * i) % 40 for i in range(n)])
        put_tails(p, layer, list(range(n)), tails)
        calls.append((p, layer, list(range(n)), p.new(n, p.G * p.hkv, 128), tails))
    torch.cuda.synchronize()
    outs = [[p.ctx.decode_attn_shared(layer, 0, seqs, q) for p, layer, seqs, q, _ in calls] for _ in range(20)]
    torch.cuda.synchronize()
    for i, (p, layer, seqs, q, tails) in enumerate(calls):
        p.check(outs[0][i], layer, q, tails)
        assert all(torch.equal(o[i], outs[0][i]) for o in outs)
        p.close()


@pytest.mark.parametrize("dtype,d", [(BF, 128), (F, 64)])
def test_tensors_aligned_to_sixteen_bytes_only(dtype, d):
    p = Prompt(300, 4, 2, d, dtype, max_batch=5, seed=23)
    n = 16 // torch.tensor([], dtype=dtype).element_size()

    def shifted(*shape):
        return torch.cat([p.new(n), p.new(*shape).flatten()])[n:].view(shape)

    seqs, tails = [1, 2, 4], random_tails(p, [20, 0, 3])
    put_tails(p, 1, seqs, tails)
    q, kn, vn, out = shifted(3, 8, d), shifted(3, 2, d), shifted(3, 2, d), shifted(3, 8, d)
    assert q.data_ptr() % 32 == kn.data_ptr() % 32 == out.data_ptr() % 32 == 16
    p.ctx.decode_attn_shared(1, 0, seqs, q, kn, vn, out=out)
    p.check(out, 1, q, [(torch.cat([k, kn[b:b + 1]]), torch.cat([v, vn[b:b + 1]])) for b, (k, v) in enumerate(tails)])
    p.close()


def test_context_with_more_units_than_the_packed_lists_serve():
    """More than 1 024 (slots x KV heads): the residual lists keep their portable layout."""
    p = Prompt(1111, 4, 3, 128, BF, max_batch=400, max_tail=20, modes=[1, 0, 2], seed=3)
    _run(p, 1, list(range(399, 0, -13)), [b % 21 for b in range(31)])
    p.close()
    p = Prompt(300, 2, 3, 128, BF, block=4, max_batch=400, max_tail=20, modes=[1, 1, 2], seed=4)  # (the token rule refuses such contexts)
    _run(p, 3, [5, 0], [20, 1])
    p.close()


@pytest.mark.parametrize("scale", [0.0, 8.0])
@pytest.mark.parametrize("dtype,d", [(BF, 128), (F, 64)])
def test_flat_and_peaked_softmax(scale, dtype, d):
    """All logits zero, and logits of hundreds (a maximum that moves between tiles, probabilities that underflow)."""
    p = Prompt(2000, 4, 2, d, dtype, seed=6)
    _run(p, 0, [1, 2, 3], [100, 0, 9], scale=scale)
    p.close()


@pytest.mark.parametrize("dtype,d", [(BF, 128), (F, 64), (BF, 64)])
def test_generation_appends_to_the_named_slots(dtype, d):
    """Rows appended by the call are attended to by it and stay for later ones; other slots' tails, and the rows of the output behind the batch, are
    left alone; the prompt's own slot may go on as one of the batch."""
    p = Prompt(777, 2, 2, d, dtype, max_batch=5, max_tail=260, seed=11)
    seqs = [4, 0, 2]
    tails = random_tails(p, [250, 0, 127])
    put_tails(p, 1, seqs, tails)
    other = random_tails(p, [33])
    put_tails(p, 1, [3], other)
    room = torch.full((6, p.G * p.hkv, d), 5.0, dtype=dtype, device="cuda")
    for step in range(5):
        q, kn, vn = p.new(3, p.G * p.hkv, d), p.new(3, p.hkv, d), p.new(3, p.hkv, d)
        tails = [(torch.cat([k, kn[b:b + 1]]), torch.cat([v, vn[b:b + 1]])) for b, (k, v) in enumerate(tails)]
        out = p.ctx.decode_attn_shared(1, 0, torch.tensor(seqs, dtype=torch.int32), q, kn, vn, out=room[:3])
        p.check(out, 1, q, tails)
        assert (room[3:] == 5).all()
    q = p.new(1, p.G * p.hkv, d)
    p.check(p.ctx.decode_attn_shared(1, 0, [3], q), 1, q, other)
    # the slot of the prompt itself: the same rows as an ordinary decode step reads
    q = p.new(1, p.G * p.hkv, d)
    p.check(p.ctx.decode_attn_shared(1, 0, [0], q), 1, q, [tails[1]])
    p.check(p.ctx.decode_attn(1, q), 1, q, [tails[1]])
    # tails of the other layer are empty
    q = p.new(3, p.G * p.hkv, d)
    p.check(p.ctx.decode_attn_shared(0, 0, seqs, q), 0, q, random_tails(p, [0, 0, 0]))
    p.ctx.set_tail_len(3, 0)
    q = p.new(1, p.G * p.hkv, d)
    p.check(p.ctx.decode_attn_shared(1, 0, [3], q), 1, q, random_tails(p, [0]))
    p.close()


@pytest.mark.parametrize("dtype,d", [(BF, 128), (F, 64)])
def test_append_tail_before_an_ordinary_decode_step(dtype, d):
    """Rows put behind a sequence's own prompt in bulk, out of strided tensors, are what decode_attn and fold_tail see."""
    p = Prompt(160, 2, 2, d, dtype, max_batch=2, max_tail=40, max_fold=32, max_prefill=200, seed=12)
    k, v = p.new(2, 24, p.hkv, d + 8), p.new(2, 24, p.hkv, d + 8)
    k, v = k[1, 2:22, :, :d], v[1, 2:22, :, :d]
    for layer in range(2):
        p.ctx.append_tail(layer, 0, k[:13], v[:13])
        p.ctx.append_tail(layer, 0, k[13:13], v[13:13])  # nothing
        p.ctx.append_tail(layer, 0, k[13:], v[13:])
    q = p.new(1, p.G * p.hkv, d)
    p.check(p.ctx.decode_attn(1, q), 1, q, [(k, v)])
    before = p.ctx.decode_attn_shared(1, 0, [0], q)
    p.check(before, 1, q, [(k, v)])
    p.ctx.fold_tail(0, 16)
    p.check(p.ctx.decode_attn_shared(1, 0, [0], q, out_dtype=0), 1, q, [(k, v)]) if p.modes == [2, 2] else None
    a, b = p.ctx.decode_attn_shared(1, 0, [0], q, out_dtype=0), p.ctx.decode_attn(1, q, out_dtype=0)
    assert ((a - b).abs() <= 2.0 ** -7 * b.abs().max()).all()  # (both read the folded prompt)
    p.close()


@pytest.mark.parametrize("batch,hkv,G,tail", [(80, 6, 4, 90), (150, 3, 8, 40), (2, 2, 4, 2500), (1, 1, 8, 1100), (3, 8, 1, 700)])
def test_joins_of_many_units_and_of_long_tails(batch, hkv, G, tail):
    """More blocks than three on every SM; clusters of two to eight blocks that share a unit's tail and outputs."""
    p = Prompt(1500, G, hkv, 128, BF, max_batch=batch, max_tail=tail + 1, modes=[h % 3 for h in range(hkv)], seed=batch)
    lens = [max(0, tail - 7 * b) for b in range(batch)]
    tails = random_tails(p, lens)
    put_tails(p, 0, list(range(batch)), tails)
    for _ in range(2):
        q, kn, vn = p.new(batch, G * hkv, 128), p.new(batch, hkv, 128), p.new(batch, hkv, 128)
        if lens[0] < tail + 1:
            tails = [(torch.cat([k, kn[b:b + 1]]), torch.cat([v, vn[b:b + 1]])) for b, (k, v) in enumerate(tails)]
            out = p.ctx.decode_attn_shared(0, 0, list(range(batch)), q, kn, vn)
            lens[0] += 1
        else:
            out = p.ctx.decode_attn_shared(0, 0, list(range(batch)), q)
        p.check(out, 0, q, tails)
    p.close()


@pytest.mark.parametrize("dtype,d,G", [(BF, 128, 4), (BF, 128, 8), (F, 64, 2), (BF, 64, 1)])
def test_tail_rows_infinitely_far_off(dtype, d, G):
    """Keys whose logit is minus infinity: their tokens count for nothing, also where a sequence has no others, or a warp's first ones are such."""
    p = Prompt(200, G, 2, d, dtype, seed=40)
    lens, off = [1, 70, 300], [1, 65, 299]
    tails = random_tails(p, lens)
    for (k, _), m in zip(tails, off):
        k[:m, :, 0] = float("-inf")
    put_tails(p, 0, [0, 1, 2], tails)
    q = p.new(3, 2 * G, d)
    q[:, :, 0] = q[:, :, 0].abs() + 1
    out = p.ctx.decode_attn_shared(0, 0, [0, 1, 2], q)
    p.check(out, 0, q, [(k[m:], v[m:]) for (k, v), m in zip(tails, off)])
    p.close()


def test_refused_tensors():
    """Sizes, types and strides that the call would read past or misread."""
    p = Prompt(64, 2, 2, 64, F, seed=41)
    q, kn = p.new(2, 4, 64), p.new(2, 2, 64)
    for bad in (dict(q=p.new(2, 3, 64)), dict(q=q.to(BF)), dict(q=p.new(2, 64, 4).mT), dict(q=q.flatten(1)), dict(k=p.new(2, 1, 64)), dict(v=kn.to(BF)),
                dict(k=p.new(1, 2, 64)), dict(v=p.new(2, 64, 2).mT), dict(out=torch.empty_like(q[:1])), dict(out=q.to(BF)), dict(out=p.new(2, 64, 4).mT)):
        with pytest.raises(ValueError):
            p.ctx.decode_attn_shared(0, 0, [0, 1], bad.get("q", q), bad.get("k", kn), bad.get("v", kn), out=bad.get("out"))
    r = p.B.Rotary([])
    with pytest.raises(ValueError):
        p.ctx.decode_qkv(0, r, p.new(2, 8 * 64), None, 0, [0, 1], out=torch.empty_like(q[:1]))
    for k, v in ((kn, kn[:1]), (kn, kn.to(BF)), (p.new(2, 1, 64), p.new(2, 1, 64)), (kn, p.new(2, 4, 64)[:, ::2]), (p.new(2, 64, 2).mT, p.new(2, 64, 2).mT)):
        with pytest.raises(ValueError):
            p.ctx.append_tail(0, 1, k, v)
    p.check(p.ctx.decode_attn_shared(0, 0, [0, 1], q), 0, q, random_tails(p, [0, 0]))  # nothing was appended
    p.close()


def test_new_outputs_belong_to_the_stream_that_writes_them():
    from paper_2607_06519_b200 import binding as B

    p = Prompt(300, 4, 2, 64, F, seed=42)
    side = torch.cuda.Stream()
    q, pos, r = p.new(2, 8, 64), torch.zeros(2, dtype=torch.int32, device="cuda"), B.Rotary([1.0] * 32)
    row = p.new(2, 12 * 64)
    torch.cuda.synchronize()
    calls = (lambda: p.ctx.decode_attn_shared(0, 0, [0, 1], q, stream=side), lambda: B.qk_norm_rope(r, q, None, pos, stream=side)[0],
             lambda: B.qk_norm_rope(r, None, q, pos, stream=side)[1], lambda: p.ctx.decode_qkv(0, r, row, pos, 0, [2, 3], stream=side))
    for call in calls:
        out = call()
        at = out.data_ptr()
        del out  # (what frees it does not wait for the side stream)
        assert all(torch.empty((2, 8, 64), device="cuda").data_ptr() != at for _ in range(3))
    out = calls[0]()
    torch.cuda.synchronize()
    p.check(out, 0, q, random_tails(p, [0, 0]))
    p.close()


def test_one_rotation_for_calls_of_several_sizes():
    from paper_2607_06519_b200 import binding as B

    r = B.Rotary([1.0] * 32, scale=2.0)
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")
    for hq, hk, d, dtype in ((4, 2, 64, F), (1, 1, 128, BF), (4, 2, 64, F)):
        q, k = torch.randn((3, hq, d), device="cuda").to(dtype), torch.randn((3, hk, d), device="cuda").to(dtype)
        for a, b in ((q, k), (q, None), (None, k)):
            for x, y in zip((a, b), B.qk_norm_rope(r, a, b, pos)):
                assert (x is None) == (y is None)
                if x is not None:
                    assert torch.equal(y[..., :64], 2 * x[..., :64]) and torch.equal(y[..., 64:], x[..., 64:])


def test_which_kernel_serves():
    from paper_2607_06519_b200 import binding as B

    for dtype, d, kernel in ((BF, 128, B.KERNEL_SHARED_TC), (F, 128, B.KERNEL_SHARED_PORTABLE), (BF, 64, B.KERNEL_SHARED_PORTABLE)):
        p = Prompt(200, 2, 2, d, dtype, seed=1)
        before = [B.kernel_launch_count(k) for k in (B.KERNEL_SHARED_TC, B.KERNEL_SHARED_PORTABLE)]
        p.ctx.decode_attn_shared(0, 0, [1], p.new(1, 4, d))
        after = [B.kernel_launch_count(k) for k in (B.KERNEL_SHARED_TC, B.KERNEL_SHARED_PORTABLE)]
        assert [b - a for a, b in zip(before, after)] == [int(kernel == B.KERNEL_SHARED_TC), int(kernel == B.KERNEL_SHARED_PORTABLE)]
        p.close()


@pytest.mark.parametrize("rule,block", [(0, 2), (1, 4)])
def test_a_prompt_and_its_continuations(rule, block):
    """All of it as a serving program has it: a prompt's projection rows are normed and rotated into the layers' rows, compressed, probed and committed; every
    sequence's own question goes behind it in bulk; then steps from fused rows, each layer of each step against 64 bits."""
    from paper_2607_06519_b200 import binding as B

    T, G, hkv, d, n = 700, 4, 2, 128, 5
    hq = G * hkv
    g = torch.Generator(device="cuda").manual_seed(31)
    inv = [10000.0 ** (-2.0 * i / d) for i in range(d // 2)]
    axis = [i % 3 for i in range(d // 2)]
    rot = [B.Rotary(inv, axis_of=axis, n_axes=3, q_weight=torch.ones(d, device="cuda", dtype=BF) * (1 + 0.1 * l), k_weight=torch.ones(d, device="cuda", dtype=BF))
           for l in range(block)]

    def projected(rows):
        return torch.randn((rows, hq + 2 * hkv, d), generator=g, device="cuda").to(BF)

    def positions(start, rows):
        return torch.stack([start + torch.arange(rows, device="cuda") // s for s in (1, 3, 7)]).to(torch.int32)

    k, v, q_last = [], [], []
    for l in range(block):
        x = projected(T)
        rows = torch.zeros((T, hkv, d), device="cuda", dtype=BF)
        q, _ = B.qk_norm_rope(rot[l], x[:, :hq], x[:, hq:hq + hkv], positions(0, T), k_out=rows)
        k.append(rows)
        v.append(x[:, hq + hkv:].contiguous())
        q_last.append(q[-8:].contiguous())
    p = Prompt(T, G, hkv, d, BF, block=block, rule=rule, max_batch=n, max_tail=40, modes=[1, 0], seed=32, kv=(k, v))
    tails = [[None] * n for _ in range(block)]
    for l in range(block):
        for b in range(n):
            m = 3 * b + 1
            x = projected(m)
            _, own = B.qk_norm_rope(rot[l], None, x[:, hq:hq + hkv], positions(T, m))
            p.ctx.append_tail(l, b, own, x[:, hq + hkv:].contiguous())
            tails[l][b] = (own, x[:, hq + hkv:])
    for step in range(3):
        for l in range(block):
            x = projected(n)
            pos = torch.stack([torch.tensor([T + 3 * b + 1 + step for b in range(n)], device="cuda")] * 3).to(torch.int32)
            q, kn = B.qk_norm_rope(rot[l], x[:, :hq], x[:, hq:hq + hkv], pos)
            tails[l] = [(torch.cat([a, kn[b:b + 1]]), torch.cat([c, x[b:b + 1, hq + hkv:]])) for b, (a, c) in enumerate(tails[l])]
            out = p.ctx.decode_qkv(l, rot[l], x.view(n, -1), pos, 0, list(range(n)))
            p.check(out, l, q, tails[l])
    p.close()


def test_streams_and_captured_calls():
    p = Prompt(3000, 4, 2, 128, BF, max_batch=4, seed=13)
    seqs, lens = [1, 2, 3], [9, 0, 140]
    tails = random_tails(p, lens)
    put_tails(p, 0, seqs, tails)
    q = p.new(3, 8, 128)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = torch.zeros_like(q)
    with torch.cuda.stream(side):
        for _ in range(3):
            p.ctx.decode_attn_shared(0, 0, seqs, q, out=out)
    side.synchronize()
    p.check(out, 0, q, tails)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(3):  # (kernels of one call behind those of another)
            p.ctx.decode_attn_shared(0, 0, seqs, q, out=out)
        q2 = q * 0.5
        out2 = p.ctx.decode_attn_shared(0, 0, seqs, q2)
        own = p.ctx.decode_attn(0, q2[:1])
    q.copy_(p.new(3, 8, 128))
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    p.check(out, 0, q, tails)
    p.check(out2, 0, q2, tails)
    p.check(own, 0, q2[:1], random_tails(p, [0]))
    p.close()


def test_repeated_calls_give_the_same_bits():
    p = Prompt(4100, 4, 3, 128, BF, max_batch=40, seed=14)
    seqs = list(range(40))
    put_tails(p, 0, seqs, random_tails(p, [b * 7 for b in range(40)]))
    q = p.new(40, 12, 128)
    first = p.ctx.decode_attn_shared(0, 0, seqs, q, out_dtype=0)
    for _ in range(5):
        assert torch.equal(p.ctx.decode_attn_shared(0, 0, seqs, q, out_dtype=0), first)
    p.close()


@pytest.mark.parametrize("dtype,d", [(BF, 128), (F, 64)])
@pytest.mark.parametrize("shared", [True, False])
def test_step_from_a_fused_row(dtype, d, shared):
    """Norm, rotation, append and attention in one call, against the same by separate calls; then what the tail holds."""
    p = Prompt(900, 4, 2, d, dtype, max_batch=3, max_tail=9, seed=15)
    B, hq = p.B, 8
    inv = [10000.0 ** (-2.0 * i / d) for i in range(d // 2)]
    r = B.Rotary(inv, axis_of=[i % 3 for i in range(d // 2)], n_axes=3, q_weight=p.new(d), k_weight=p.new(d))
    seqs = [2, 0, 1] if shared else [0]
    n = len(seqs)
    tails = random_tails(p, [0] * n)
    for step in range(4):
        rows = p.new(n, (hq + 2 * 2) * d + 8)[:, :-8]
        pos = torch.randint(0, 9000, (3, n), device="cuda", dtype=torch.int32)
        x = rows.unflatten(1, (-1, d))
        q, k = B.qk_norm_rope(r, x[:, :hq], x[:, hq:hq + 2], pos)
        tails = [(torch.cat([a, k[b:b + 1]]), torch.cat([c, x[b:b + 1, hq + 2:]])) for b, (a, c) in enumerate(tails)]
        out = p.ctx.decode_qkv(1, r, rows, pos, 0, seqs) if shared else p.ctx.decode_qkv(1, r, rows, pos)
        p.check(out, 1, q, tails)
    q = p.new(n, hq, d)
    out = p.ctx.decode_attn_shared(1, 0, seqs, q)
    p.check(out, 1, q, tails)
    p.close()


def test_prompt_in_another_slot_and_reset():
    p = Prompt(640, 2, 2, 128, BF, max_batch=4, slot=2, seed=16)
    _run(p, 0, [0, 2, 3], [4, 8, 0])
    p.ctx.reset()
    q = p.new(1, 4, 128)
    with pytest.raises(p.B.FdkvError) as e:
        p.ctx.decode_attn_shared(0, 2, [0], q)
    assert e.value.code == 5
    p.ctx.compress_prefill(1, 0, 1, 640, p.k, p.v)
    p.ctx.set_modes(1, p.modes)
    p.ctx.commit(1)
    p.check(p.ctx.decode_attn_shared(0, 1, [0], q), 0, q, random_tails(p, [0]))  # (reset emptied the tails)
    p.close()


def test_refusals_leave_the_state_alone():
    p = Prompt(128, 2, 2, 64, F, max_batch=4, max_tail=3, seed=17)
    ctx, B = p.ctx, p.B
    q, kn = p.new(2, 4, 64), p.new(2, 2, 64)

    def code(fn):
        with pytest.raises(B.FdkvError) as e:
            fn()
        return e.value.code

    call = ctx.decode_attn_shared
    assert code(lambda: call(2, 0, [0, 1], q)) == 1            # layer
    assert code(lambda: call(-1, 0, [0, 1], q)) == 1
    assert code(lambda: call(0, 4, [0, 1], q)) == 1            # prompt slot
    assert code(lambda: call(0, -1, [0, 1], q)) == 1
    assert code(lambda: call(0, 0, [0, 4], q)) == 1            # sequence slot
    assert code(lambda: call(0, 0, [1, 1], q)) == 1            # the same slot twice
    assert code(lambda: call(0, 0, [], q[:0])) == 1            # no sequence
    assert code(lambda: call(0, 0, [0, 1, 2, 3, 0], p.new(5, 4, 64))) == 1
    assert code(lambda: call(0, 0, [0, 1], q, kn, None)) == 1
    assert code(lambda: call(0, 0, [0, 1], q, out=q, out_dtype=7)) == 1
    flat = torch.zeros(2 * 4 * 64 + 1, device="cuda")
    assert code(lambda: call(0, 0, [0, 1], flat[1:].view(2, 4, 64))) == 1
    assert code(lambda: call(0, 1, [0, 1], q)) == 5            # no prompt there
    with pytest.raises(ValueError):
        call(0, 0, [0], q)
    # a slot with a prompt of its own
    ctx.compress_prefill(3, 0, 1, 128, p.k, p.v)
    ctx.set_modes(3, p.modes)
    ctx.commit(3)
    assert code(lambda: call(0, 0, [1, 3], q)) == 5
    # tails
    k5 = p.new(5, 2, 64)
    assert code(lambda: ctx.append_tail(0, 1, k5, k5)) == 5    # more than the tail holds
    assert code(lambda: ctx.append_tail(2, 1, k5[:1], k5[:1])) == 1
    assert code(lambda: ctx.append_tail(0, 4, k5[:1], k5[:1])) == 1
    ctx.append_tail(0, 1, k5[:3], k5[:3])
    assert code(lambda: ctx.append_tail(0, 1, k5[:1], k5[:1])) == 5
    assert code(lambda: call(0, 0, [0, 1], q, kn, kn)) == 5    # slot 1 is full: nothing is appended to slot 0 either
    tails = [random_tails(p, [0])[0], (k5[:3], k5[:3])]
    p.check(call(0, 0, [0, 1], q), 0, q, tails)
    # the step from a fused row
    r = B.Rotary([1.0] * 32)
    pos = torch.zeros((1, 2), dtype=torch.int32, device="cuda")
    row = p.new(2, 8 * 64)
    assert code(lambda: ctx.decode_qkv(0, r, row, pos, 0, [0, 1])) == 5
    assert code(lambda: ctx.decode_qkv(0, r, row, pos)) == 5              # slot 1 has no prompt
    assert code(lambda: ctx.decode_qkv(0, r, row, pos, -1, [0, 1])) == 1
    assert code(lambda: ctx.decode_qkv(0, r, row, pos, 0)) == 1
    assert code(lambda: ctx.decode_qkv(0, r, row, None, 0, [0, 2])) == 1
    with pytest.raises(ValueError):
        ctx.decode_qkv(0, r, row[:, :-64], pos, 0, [0, 2])
    p.check(call(0, 0, [0, 1], q), 0, q, tails)
    p.close()
    p = Prompt(128, 2, 2, 128, BF, max_batch=2, row_format=1, modes=[2, 2], seed=18)
    assert code(lambda: p.ctx.decode_attn_shared(0, 0, [1], p.new(1, 4, 128))) == 2
    p.close()
