"""Arenas for fewer committed prompts than slots (fdkv_sizes_prompts): many sequences on one prompt."""
import pytest
import torch

from paper_2607_06519_b200 import binding as B


def _cfg(max_batch, n_layers=4, hkv=2, T=1000, tail=200, dtype=B.BF16, rule=0, block=2, fold=0):
    return B.Config(n_layers, 4 * hkv, hkv, 128, max_batch, T, tail, dtype, 1, 8, rule, block, fold)


@pytest.mark.parametrize("kw", [{}, dict(dtype=B.F32), dict(rule=1), dict(block=4), dict(fold=96)])
def test_sizes(kw):
    cfg = _cfg(7, **kw)
    all_, work = B.sizes(cfg)
    one, two = B.sizes(cfg, 1)[0], B.sizes(cfg, 2)[0]
    assert B.sizes(cfg, 7) == (all_, work) and B.sizes(cfg, 1)[1] == work
    assert all_ - one == 6 * (two - one)                                   # a prompt each
    e = 4 if cfg.dtype == B.F32 else 2
    assert two - one >= 2 * cfg.n_layers * cfg.n_kv_heads * 1000 * 128 * e  # ... with exact rows
    assert one - (two - one) >= 2 * cfg.n_layers * 7 * cfg.n_kv_heads * 200 * 128 * e  # tails for every slot
    for bad in (0, 8, -1):
        with pytest.raises(B.FdkvError) as err:
            B.sizes(cfg, bad)
        assert err.value.code == 1


def test_sixty_four_sequences_on_one_prompt_of_32k():
    cfg = B.Config(32, 32, 8, 128, 64, 32768, 256, B.BF16, 1, 16)
    assert B.sizes(cfg)[0] > 270e9 and B.sizes(cfg, 1)[0] < 7e9


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,rule,fold", [(B.BF16, 0, 64), (B.BF16, 1, 0), (B.F32, 0, 0)])
def test_a_context_of_that_size(dtype, rule, fold):
    """One prompt in any modes fits, with every tail in use; a second one is refused until the first is forgotten."""
    t = torch.bfloat16 if dtype == B.BF16 else torch.float32
    cfg = _cfg(6, n_layers=2, T=500, tail=30, dtype=dtype, rule=rule, fold=fold)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = ([torch.randn((500, 2, 128), generator=g, device="cuda").to(t) for _ in range(2)] for _ in range(2))
    q, row = torch.randn((6, 8, 128), generator=g, device="cuda").to(t), torch.randn((30, 2, 128), generator=g, device="cuda").to(t)
    outs = []
    for prompts in (1, None):
        ctx = B.Context(cfg, prompts=prompts)
        assert ctx.arena_bytes == B.sizes(cfg, prompts)[0]
        for modes in ([2, 2], [1, 2], [1, 0]):
            ctx.reset()
            ctx.compress_prefill(0, 0, 1, 500, k, v)
            if rule:
                ctx.probe(0, 0, 1, [q[:4].contiguous(), q[:4].contiguous()], [490, 492, 498, 499], 0.0)
            ctx.set_modes(0, modes)
            ctx.commit(0)
            for b in range(6):
                ctx.append_tail(1, b, row[b:], row[b:])
            outs.append(ctx.decode_attn_shared(1, 0, [0, 1, 2, 3, 4, 5], q))
            if prompts and modes == [2, 2]:
                ctx.compress_prefill(5, 0, 1, 500, k, v)
                if rule:
                    ctx.probe(5, 0, 1, [q[:4].contiguous(), q[:4].contiguous()], [490, 492, 498, 499], 0.0)
                ctx.set_modes(5, modes)
                with pytest.raises(B.FdkvError) as err:
                    ctx.commit(5)
                assert err.value.code == 3
                assert torch.equal(ctx.decode_attn_shared(1, 0, [0, 1, 2, 3, 4, 5], q), outs[-1])
        assert ctx.device_status() == 0
        ctx.close()
    assert all(torch.equal(a, b) for a, b in zip(outs[:3], outs[3:]))
