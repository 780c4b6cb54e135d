"""Arguments that fdkv_qk_norm_rope refuses on the host: nothing is enqueued, so no device is needed."""
import ctypes as C

import pytest

OK_ARGS = dict(hq=4, hk=2, d=128, dtype=1, rotary=128, inter=0, axes=1, eps=1e-6, scale=1.0, n=3, q=0x10000, k=0x20000, pos=0x30000, ps=3, qo=0x40000,
               ko=0x50000, st=4 * 128, sh=128, qw=0, kw=0, axis=None, inv=True)


def _call(**kw):
    from paper_2607_06519_b200 import binding as B

    a = dict(OK_ARGS, **kw)
    inv = (C.c_float * 64)(*[a.get("f", 0.5)] * 64)
    axis = None if a["axis"] is None else (C.c_int32 * 64)(*[a["axis"]] * 64)
    r = B._Rotary(a["hq"], a["hk"], a["d"], a["dtype"], a["rotary"], a["inter"], a["axes"], a["eps"], a["scale"], C.addressof(inv) if a["inv"] else None,
                  None if axis is None else C.addressof(axis), a["qw"] or None, a["kw"] or None)
    return B._qk_norm_rope(r, a["n"], a["q"] or None, a["st"], a["sh"], a["k"] or None, a["st"], a["sh"], a["pos"] or None, a["ps"], a["qo"] or None, a["st"], a["sh"],
                           a["ko"] or None, a["st"], a["sh"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(hq=0), 1), (dict(hk=0), 1), (dict(hq=1025), 1), (dict(d=96), 2), (dict(d=256), 2), (dict(dtype=2), 2), (dict(rotary=8), 2), (dict(rotary=130), 1),
    (dict(rotary=-16), 1), (dict(axes=0), 1), (dict(axes=5), 1), (dict(axis=1), 1), (dict(axis=-1), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1),
    (dict(scale=float("inf")), 1), (dict(f=float("nan")), 1), (dict(inv=False), 1), (dict(n=-1), 1), (dict(n=1 << 31), 1), (dict(q=0), 1), (dict(ko=0), 1),
    (dict(q=0, qo=0, k=0, ko=0), 1), (dict(q=0x10008), 1), (dict(ko=0x50002), 1), (dict(qw=0x60004), 1), (dict(pos=0), 1), (dict(pos=0x30002), 1),
    (dict(axes=2, ps=2), 1), (dict(st=4 * 128 + 4), 1), (dict(sh=64), 1), (dict(sh=132), 1),
])
def test_refused(kw, code):
    assert _call(**kw) == code, kw


def test_no_tokens_is_no_work():
    assert _call(n=0) == 0


def test_binding_checks():
    import torch

    from paper_2607_06519_b200 import binding as B

    with pytest.raises(ValueError):
        B.Rotary([1.0] * 64, axis_of=[0] * 63)
    with pytest.raises(ValueError):
        B.Rotary([1.0] * 64, q_weight=torch.ones(256)[::2])
    r = B.Rotary([1.0] * 64, n_axes=2, q_weight=torch.ones(128))
    x = torch.zeros((3, 2, 128))
    pos = torch.zeros((2, 3), dtype=torch.int32)
    for bad in (lambda: B.qk_norm_rope(r, x.bfloat16(), None, pos),                          # weights of another type
                lambda: B.qk_norm_rope(r, x[..., :64], None, pos),                           # ... of another head_dim
                lambda: B.qk_norm_rope(r, x, x.bfloat16(), pos),                             # rows of two types
                lambda: B.qk_norm_rope(r, x, x[:2], pos),                                    # of two lengths
                lambda: B.qk_norm_rope(r, x, None, pos[0]),                                  # one axis of two
                lambda: B.qk_norm_rope(r, x, None, pos.long()),
                lambda: B.qk_norm_rope(r, x.transpose(1, 2).contiguous().transpose(1, 2), None, pos),  # not dense along d
                lambda: B.qk_norm_rope(r, x, None, pos, q_out=x[:, :1])):
        with pytest.raises(ValueError):
            bad()
