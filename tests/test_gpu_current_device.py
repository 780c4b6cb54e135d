"""Calls whose tensors are on another device than the current one: made with the tensors' device current, and with the same results.  (One device stands for two: the binding
is told that device 1 is current.)"""
import pytest
import torch

from shared_util import Prompt, random_tails

pytestmark = pytest.mark.gpu


@pytest.fixture
def elsewhere(monkeypatch):
    """Names device 1 as the current one from when it is called; lists the devices made current since."""
    real, made, current = torch.cuda.device, [], [1]

    class Device(real):
        def __enter__(self):
            made.append(self.idx)
            current.append(self.idx)
            return super().__enter__()

        def __exit__(self, *a):
            current.pop()
            return super().__exit__(*a)

    def begin():
        monkeypatch.setattr(torch.cuda, "device", Device)
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[-1])
        return made

    return begin


def test_results_and_devices(elsewhere):
    from paper_2607_06519_b200 import binding as B

    p = Prompt(300, 4, 2, 64, torch.float32, modes=[0, 2], seed=60)
    r, pos = B.Rotary([0.5] * 32), torch.tensor([3, 5], dtype=torch.int32, device="cuda")
    row = p.new(2, 12 * 64)
    x = row.view(2, 12, 64)
    y = x[:, :8].contiguous()
    made = elsewhere()
    for call in (lambda: B.qk_norm_rope(r, x[:, :8], x[:, 8:10], pos), lambda: p.ctx.decode_attn_shared(0, 0, [0, 1], y),
                 lambda: p.ctx.append_tail(1, 1, x[:, 8:10], x[:, 10:]), lambda: p.ctx.decode_qkv(0, r, row, pos, 0, [2, 3])):
        n = len(made)
        call()
        assert made[n:] and set(made[n:]) == {0}
    q, k = B.qk_norm_rope(r, x[:, :8], x[:, 8:10], pos)
    a = pos.double()[:, None, None] * 0.5
    for got, y in ((q, x[:, :8].double()), (k, x[:, 8:10].double())):
        want = torch.cat([y[..., :32] * a.cos() - y[..., 32:] * a.sin(), y[..., 32:] * a.cos() + y[..., :32] * a.sin()], -1)
        # the angle is a float32 number of half turns (2^-25 of a turn), sine and cosine within 2 steps, two products and a sum
        assert ((got.double() - want).abs() <= (2 * 3.1416 * 2.0 ** -25 + 2 * 2.0 ** -23 + 3 * 2.0 ** -24) * (y.abs() + y.roll(32, -1).abs())).all()
    own = [(k[b:b + 1], x[b:b + 1, 10:]) for b in range(2)]
    p.check(p.ctx.decode_attn_shared(0, 0, [2, 3], q), 0, q, own)
    p.check(p.ctx.decode_attn_shared(1, 0, [0, 1], q), 1, q, [random_tails(p, [0])[0], (x[:, 8:10], x[:, 10:])])
    p.close()
