"""The wait of a warp for a counter (the entries' warps of the shared prompt's kernel, which the copying warp may keep waiting for as long as a block has heads without
entries): it ends with the timeout status, and not before a second is up."""
import pytest
import torch

from shared_util import Prompt, random_tails

pytestmark = pytest.mark.gpu


def test_it_runs_out_after_a_second_or_more():
    from paper_2607_06519_b200 import binding as B

    p = Prompt(300, 4, 2, 128, torch.bfloat16, modes=[0, 1], seed=70)
    q = p.new(1, 8, 128)
    before = p.ctx.decode_attn_shared(0, 0, [1], q)
    polls, ms = 65536, []
    for _ in range(3):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        p.ctx.test_count_expiry(polls)
        b.record()
        assert p.ctx.device_status() == 7
        p.ctx.test_clear_device_status()
        ms.append(a.elapsed_time(b))
    assert min(ms) / polls * B._lib.fdkv_test_count_cap() >= 1000.0, ms
    assert p.ctx.device_status() == 0
    after = p.ctx.decode_attn_shared(0, 0, [1], q)
    assert torch.equal(before, after)
    p.check(after, 0, q, random_tails(p, [0]))
    for bad in (0, 65537):
        with pytest.raises(B.FdkvError):
            p.ctx.test_count_expiry(bad)
    print(f"{min(ms) / polls * 1e6:.0f} ns a poll")
    p.close()
