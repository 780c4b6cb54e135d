"""The cut of fdkv_decode_attn_shared's prompt part (host only): every (head, tile) in one range, a tile at least per range, parts of their own
for every range, head and row group within the workspace, heads with entries in fewer tiles per range."""
import ctypes as C
import random

import pytest


def _plan(T, batch, G, hkv, modes, keep=(1, 16), row_tile=128, tile=128, sms=148, d=128, max_batch=None):
    from paper_2607_06519_b200 import binding as B

    start, counts = (C.c_int32 * 161)(), (C.c_int32 * 4)()
    st = B._lib.fdkv_test_plan_shared(T, batch, max_batch or batch, G, hkv, d, (C.c_int32 * hkv)(*modes), keep[0], keep[1], row_tile, tile, sms, start, counts)
    assert st == 0, (st, T, batch, G, hkv)
    ranges, tiles, groups, rows = counts
    return list(start[: ranges + 1]), tiles, groups, rows


def test_random_calls():
    rng = random.Random(7)
    for _ in range(3000):
        hkv, G = rng.choice([1, 2, 3, 5, 8, 16]), rng.choice([1, 2, 4, 8])
        batch = rng.choice([1, 2, 3, rng.randint(1, 64), rng.randint(1, 1024)])
        row_tile, tile = rng.choice([(128, 128), (32, 32)])
        T = int(128 * 2 ** rng.uniform(-7, 11)) + 1
        sms = rng.choice([148, 148, 132, 160, 200, 7])
        start, tiles, groups, rows = _plan(T, batch, G, hkv, [rng.randint(0, 2) for _ in range(hkv)], (1, rng.choice([1, 8, 32])), row_tile, tile, sms)
        assert tiles == -(-T // tile) and groups == -(-batch * G // row_tile) and rows == min(row_tile, batch * G)
        assert start[0] == 0 and start[-1] == hkv * tiles
        assert all(b > a for a, b in zip(start, start[1:]))
        numbers = set()
        for q in range(len(start) - 1):
            for h in range(start[q] // tiles, (start[q + 1] - 1) // tiles + 1):
                for g in range(groups):
                    n = (q + h) * groups + g
                    assert n not in numbers
                    numbers.add(n)
        assert (max(numbers) + 1) * rows <= batch * G * hkv * 160


def test_blocks_fill_the_device_once():
    for batch, ranges in ((1, 148), (32, 148), (33, 74), (64, 74), (96, 49), (128, 37), (256, 18)):
        start, _, groups, _ = _plan(32768, batch, 4, 8, [0] * 8)
        assert len(start) - 1 == ranges and ranges * groups <= 148
        sizes = [b - a for a, b in zip(start, start[1:])]
        assert max(sizes) - min(sizes) <= 1


def test_heads_with_entries_get_fewer_tiles_per_range():
    start, tiles, _, _ = _plan(131072, 16, 4, 8, [0, 1, 0, 2, 0, 1, 0, 1])
    sizes = {0: [], 1: []}
    for a, b in zip(start, start[1:]):
        if a // tiles == (b - 1) // tiles:
            sizes[(a // tiles) in (1, 5, 7)].append(b - a)
    assert max(sizes[1]) < min(sizes[0])


def test_refusals():
    from paper_2607_06519_b200 import binding as B

    start, counts, modes = (C.c_int32 * 161)(), (C.c_int32 * 4)(), (C.c_int32 * 8)()
    assert B._lib.fdkv_test_plan_shared(0, 1, 1, 4, 8, 128, modes, 1, 16, 128, 128, 148, start, counts) == 1
    assert B._lib.fdkv_test_plan_shared(128, 2, 1, 4, 8, 128, modes, 1, 16, 128, 128, 148, start, counts) == 1
    assert B._lib.fdkv_test_plan_shared(128, 1, 1, 4, 8, 128, None, 1, 16, 128, 128, 148, start, counts) == 1


@pytest.mark.parametrize("bad", [dict(seqs=None), dict(batch=0)])
def test_shared_call_without_a_context(bad):
    from paper_2607_06519_b200 import binding as B

    assert B._lib.fdkv_decode_attn_shared(None, 0, 0, None, bad.get("batch", 1), None, None, None, None, 0, None) == 1
    assert B._lib.fdkv_append_tail(None, 0, 0, 1, None, None, 64, 64, None) == 1
    assert B._lib.fdkv_decode_qkv(None, 0, 0, None, 1, None, None, 0, None, None, 0, None) == 1
