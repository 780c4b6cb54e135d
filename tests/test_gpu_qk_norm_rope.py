"""Norm and rotation of queries and keys against the formula in 64 bits: types, head layouts, strides, axes, partial and
neighbouring-channel rotation, far positions, in place, streams, captured graphs, and the decode step that goes on from a fused row.

Tolerances, in units of u = 2^-24 (a float32 rounding) of |a| + |b| of a channel pair: the sum of squares of a head is off by at most
(16 + 3 + 2) u, half of which reaches its inverse root, the root itself and the two products by 6 u, the angle (a float32 of
at most one half turn) by 3 u, sine and cosine by 4 u with their factor, the last products and sum by 3 u: 32 u in all cover
it.  bf16 outputs add one rounding, 2^-8 of the value."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _case(n, hq, hk, d, dtype, rotary, axes, seed=0, far=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randn((n, hq, d), generator=g, device="cuda").mul_(3).to(dtype)
    k = torch.randn((n, hk, d), generator=g, device="cuda").mul_(3).to(dtype)
    qw, kw = ((1 + 0.3 * torch.randn((d,), generator=g, device="cuda")).to(dtype) for _ in range(2))
    pos = torch.randint(0, 2 ** 31 - 1 if far else 5000, (axes, n), generator=g, device="cuda", dtype=torch.int32)
    inv = [10000.0 ** (-2.0 * i / rotary) for i in range(rotary // 2)]
    inv = np.asarray(inv, np.float32)
    return q, k, qw, kw, pos, inv


def _ref(x, w, pos, inv, axis, interleaved, eps, scale):
    """(the result, what a tolerance is relative to) in float64."""
    y = x.double()
    if w is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * w.double()
    out, mag = y.clone(), y.abs()
    for i in range(len(inv)):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + len(inv))
        ang = pos[axis[i]].double() * float(inv[i])
        c, s = (torch.cos(ang) * scale)[:, None], (torch.sin(ang) * scale)[:, None]
        out[..., a] = y[..., a] * c - y[..., b] * s
        out[..., b] = y[..., b] * c + y[..., a] * s
        mag[..., a] = mag[..., b] = (y[..., a].abs() + y[..., b].abs()) * max(1.0, abs(scale))
    return out, mag


def _check(got, x, w, pos, inv, axis, interleaved, eps=1e-6, scale=1.0, far=False):
    ref, mag = _ref(x, w, pos, inv, axis, interleaved, eps, scale)
    tol = 32 * U * mag + (2.0 ** -8 * ref.abs() if got.dtype == torch.bfloat16 else 0)
    if far:  # angles of 2^31: three float64 roundings of 2^-22 in the kernel (product, 1 / 2 pi, turns), one here
        tol = tol + 2.0 ** -20 * mag
    bad = (got.double() - ref).abs() > tol
    assert not bad.any(), (int(bad.sum()), float(((got.double() - ref).abs() / mag.clamp(min=1e-30)).max()))


@pytest.mark.parametrize("n", [1, 2, 5, 33, 700])
@pytest.mark.parametrize("hq,hk,d,dtype,rotary,axes,interleaved", [
    (32, 8, 128, torch.bfloat16, 128, 3, False),
    (32, 8, 128, torch.bfloat16, 64, 1, True),
    (7, 1, 128, torch.float32, 128, 2, False),
    (4, 2, 64, torch.bfloat16, 64, 4, True),
    (5, 3, 64, torch.float32, 16, 1, False),
    (3, 3, 128, torch.bfloat16, 48, 2, True),
    (1, 1, 64, torch.float32, 48, 3, False),
    (2, 1, 128, torch.float32, 0, 1, False),
])
@pytest.mark.parametrize("norm", [False, True])
def test_against_the_formula(n, hq, hk, d, dtype, rotary, axes, interleaved, norm):
    from paper_2607_06519_b200 import binding as B

    q, k, qw, kw, pos, inv = _case(n, hq, hk, d, dtype, max(rotary, 1), axes)
    inv = inv[: rotary // 2]
    axis = [(3 * i) % axes for i in range(len(inv))]
    if not norm:
        qw = kw = None
    r = B.Rotary(inv, axis_of=axis, n_axes=axes, interleaved=interleaved, q_weight=qw, k_weight=kw, eps=1e-5, scale=1.25)
    qo, ko = B.qk_norm_rope(r, q, k, pos)
    _check(qo, q, qw, pos, inv, axis, interleaved, 1e-5, 1.25)
    _check(ko, k, kw, pos, inv, axis, interleaved, 1e-5, 1.25)


def test_far_positions_keep_their_angle():
    from paper_2607_06519_b200 import binding as B

    q, k, qw, kw, pos, inv = _case(64, 4, 2, 128, torch.float32, 128, 1, far=True)
    r = B.Rotary(inv, q_weight=qw, k_weight=kw)
    qo, ko = B.qk_norm_rope(r, q, k, pos[0])
    axis = [0] * len(inv)
    _check(qo, q, qw, pos, inv, axis, False, far=True)
    _check(ko, k, kw, pos, inv, axis, False, far=True)
    pos = -pos
    qo, _ = B.qk_norm_rope(r, q, None, pos)
    _check(qo, q, qw, pos, inv, axis, False, far=True)


@pytest.mark.parametrize("n", [1, 3, 130])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides_in_place_one_side_and_guards(n, dtype):
    """Out of the fused projection into head-major rows with a gap; in place; one side alone; what lies around stays as it was."""
    from paper_2607_06519_b200 import binding as B

    hq, hk, d = 6, 2, 128
    _, _, qw, kw, pos, inv = _case(n, hq, hk, d, dtype, d, 3, seed=1)
    g = torch.Generator(device="cuda").manual_seed(5)
    qkv = torch.randn((n, (hq + 2 * hk), d), generator=g, device="cuda").to(dtype)
    keep = qkv.clone()
    axis = [i % 3 for i in range(d // 2)]
    r = B.Rotary(inv, axis_of=axis, n_axes=3, q_weight=qw)  # (keys are rotated but not normed)
    q, k = qkv[:, :hq], qkv[:, hq:hq + hk]
    room = torch.full((hq, n + 3, d), 7.0, dtype=dtype, device="cuda")
    qo = room.transpose(0, 1)[1:n + 1]
    ko = torch.full((n, hk + 1, d + 8), 7.0, dtype=dtype, device="cuda")
    B.qk_norm_rope(r, q, k, pos, q_out=qo, k_out=ko[:, :hk, :d])
    _check(qo, q, qw, pos, inv, axis, False)
    _check(ko[:, :hk, :d], k, None, pos, inv, axis, False)
    assert torch.equal(qkv, keep)
    assert (room[:, 0] == 7).all() and (room[:, n + 1:] == 7).all() and (ko[:, hk] == 7).all() and (ko[:, :, d:] == 7).all()
    want_q, want_k = qo.clone(), ko[:, :hk, :d].clone()
    B.qk_norm_rope(r, q, k, pos, q_out=q, k_out=k)  # in place
    assert torch.equal(q, want_q) and torch.equal(k, want_k) and torch.equal(qkv[:, hq + hk:], keep[:, hq + hk:])
    a, b = B.qk_norm_rope(r, None, keep[:, hq:hq + hk], pos)
    assert a is None and torch.equal(b, want_k)
    a, b = B.qk_norm_rope(r, keep[:, :hq], None, pos)
    assert b is None and torch.equal(a, want_q)


def test_zero_rows_and_values_that_are_not_finite():
    from paper_2607_06519_b200 import binding as B

    q, k, qw, kw, pos, inv = _case(9, 4, 2, 128, torch.bfloat16, 128, 1, seed=2)
    q[3] = 0
    q[5, 1, 7] = float("nan")
    k[6, 0, 3] = float("inf")
    r = B.Rotary(inv, q_weight=qw, k_weight=kw, eps=0.0)
    r1 = B.Rotary(inv, q_weight=qw, k_weight=kw, eps=1e-6)
    qo, ko = B.qk_norm_rope(r1, q, k, pos)
    assert (qo[3] == 0).all()
    assert qo[5, 1].isnan().all() and qo[5, [0, 2, 3]].isfinite().all()
    assert ko[6, 1].isfinite().all() and not ko[6, 0, 3].isfinite()
    good = [t for t in range(9) if t not in (3, 5)]
    _check(qo[good], q[good], qw, pos[:, good], inv, [0] * 64, False)
    qo0, _ = B.qk_norm_rope(r, q, k, pos)
    _check(qo0[good], q[good], qw, pos[:, good], inv, [0] * 64, False, eps=0.0)
    assert B.qk_norm_rope(r1, q[:0], k[:0], pos[:, :0])[0].shape == (0, 4, 128)  # no tokens: nothing happens


def test_on_another_stream_and_captured():
    from paper_2607_06519_b200 import binding as B

    q, k, qw, kw, pos, inv = _case(50, 8, 2, 128, torch.bfloat16, 128, 1, seed=3)
    r = B.Rotary(inv, q_weight=qw, k_weight=kw)
    want = [t.clone() for t in B.qk_norm_rope(r, q, k, pos)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    qo, ko = torch.zeros_like(q), torch.zeros_like(k)
    with torch.cuda.stream(side):
        for _ in range(3):
            B.qk_norm_rope(r, q, k, pos, q_out=qo, k_out=ko)
    side.synchronize()
    assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])
    graph = torch.cuda.CUDAGraph()
    qo.zero_()
    with torch.cuda.graph(graph):
        B.qk_norm_rope(r, q, k, pos, q_out=qo, k_out=ko)
    pos += 17  # a replay reads what the positions hold then
    graph.replay()
    torch.cuda.synchronize()
    _check(qo, q, qw, pos, inv, [0] * 64, False)
    _check(ko, k, kw, pos, inv, [0] * 64, False)
