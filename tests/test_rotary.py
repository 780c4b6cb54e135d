"""What a Rotary and qk_norm_rope check before a call: weights whose module moved them, outputs without inputs; no device is needed."""
import pytest
import torch

from paper_2607_06519_b200 import binding as B


def test_weights_that_move():
    w = torch.nn.Parameter(torch.ones(128, dtype=torch.bfloat16))
    r = B.Rotary([1.0] * 64, q_weight=w)
    first = r.c(4, 2, 128, torch.bfloat16)
    assert (first.q_weight, first.k_weight) == (w.data_ptr(), None)
    assert r.c(4, 2, 128, torch.bfloat16) is first
    other = w.data.clone()
    w.data = other  # (what Module.to and Module._apply do)
    again = r.c(4, 2, 128, torch.bfloat16)
    assert again.q_weight == other.data_ptr() != first.q_weight
    w.data = w.data.float()
    with pytest.raises(ValueError):
        r.c(4, 2, 128, torch.bfloat16)
    assert r.c(4, 2, 128, torch.float32).q_weight == w.data_ptr()
    w.data = torch.ones(256)[::2]
    with pytest.raises(ValueError):
        r.c(4, 2, 128, torch.float32)
    w.data = torch.ones(64)
    with pytest.raises(ValueError):
        r.c(4, 2, 128, torch.float32)
    assert r.c(4, 2, 64, torch.float32).q_weight == w.data_ptr()


def test_an_output_without_its_input_is_refused():
    r, x, pos = B.Rotary([1.0] * 32), torch.zeros((3, 2, 64)), torch.zeros(3, dtype=torch.int32)
    for kw in (dict(q=x, k=None, k_out=x.clone()), dict(q=None, k=x, q_out=x.clone())):
        with pytest.raises(ValueError, match="needs its input"):
            B.qk_norm_rope(r, positions=pos, **kw)
