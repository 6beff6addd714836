"""ssd_rope_axes against the definition in more than 64 bits."""
import numpy as np
import pytest
import torch

import paper_2510_18716_amd as ssd
from oracle import mx
from paged_harness import TORCH

pytestmark = pytest.mark.gpu


def _inputs(n, H, d, pairs, axes, far, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, H, d), generator=g)
    pos = torch.randint(-far, far, (axes, n), generator=g).to(torch.int32)
    axis = torch.randint(0, axes, (pairs,), generator=g).to(torch.uint8)
    inv = torch.tensor([10000.0 ** (-i / pairs) for i in range(pairs)])
    return x, pos, axis, inv


def _check(out, x, pos, axis, inv, layout, inverse, dtype):
    """cos and sin are off by 2^-23 at most (the reduced angle's and the series' roundings, half a step each and more), times each of two elements, two products and a sum
    rounded: 2^-21 of |a| + |b|; bf16 is rounded once more, by at most 2^-8 of itself."""
    name = {ssd.SSD_ROPE_HALF: "half", ssd.SSD_ROPE_INTERLEAVED: "interleaved"}[layout]
    ref = mx.rope(x.double().numpy(), pos.numpy(), inv.numpy(), None if axis is None else axis.numpy(), name, inverse)
    pairs = len(inv)
    size = np.zeros(x.shape)
    a = np.abs(x.double().numpy())
    for i in range(pairs):
        p, q = (i, i + pairs) if name == "half" else (2 * i, 2 * i + 1)
        size[..., p] = size[..., q] = a[..., p] + a[..., q]
    far = np.abs(out.double().cpu().numpy() - ref)
    tol = 2.0 ** -21 * size + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0)
    assert np.all(far <= tol), float((far - tol).max())


SHAPES = [(1, 1, 2, 1, 1, "f32"), (16, 40, 64, 32, 1, "f32"), (33, 5, 128, 64, 3, "bf16"), (7, 3, 80, 20, 2, "bf16"), (1000, 12, 128, 48, 4, "bf16"), (5, 2, 6, 3, 3, "bf16"),
          (65, 1, 256, 64, 2, "f32"), (3, 4, 10, 5, 1, "f32"), (2, 3, 1024, 512, 4, "bf16"), (9, 7, 72, 36, 3, "f32"), (4097, 2, 64, 32, 2, "bf16"), (6, 100, 34, 1, 1, "bf16")]


@pytest.mark.parametrize("layout", [ssd.SSD_ROPE_HALF, ssd.SSD_ROPE_INTERLEAVED])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("n,H,d,pairs,axes,dtype", SHAPES)
def test_rotation(n, H, d, pairs, axes, dtype, layout, inverse):
    x, pos, axis, inv = _inputs(n, H, d, pairs, axes, 5000, seed=1)
    x = x.to(TORCH[dtype])
    xd, out = x.cuda(), torch.full_like(x, 7.0, device="cuda")
    args = (n, H, d, dtype, pos.cuda(), inv.cuda())
    ssd.ssd_rope_axes(xd, out, *args, axis=axis.cuda(), n_axes=axes, layout=layout, inverse=inverse)
    _check(out, x, pos, axis, inv, layout, inverse, dtype)
    assert torch.equal(xd.cpu(), x)
    ssd.ssd_rope_axes(xd, xd, *args, axis=axis.cuda(), n_axes=axes, layout=layout, inverse=inverse)          # in place: the same bits
    assert torch.equal(xd, out)


@pytest.mark.parametrize("far", [1 << 20, 1 << 24, (1 << 31) - 1])
def test_far_positions(far):
    x, pos, _, inv = _inputs(50, 2, 64, 32, 1, far, seed=2)
    pos[0, 0], pos[0, 1], pos[0, 2] = far, -far, 0
    out = torch.empty_like(x, device="cuda")
    ssd.ssd_rope_axes(x.cuda(), out, 50, 2, 64, "f32", pos.cuda(), inv.cuda())
    _check(out, x, pos, None, inv, ssd.SSD_ROPE_HALF, False, "f32")


@pytest.mark.parametrize("most", [4.0, 1000.0, 2.0 ** 20])
def test_far_positions_at_large_frequencies(most):
    """Products of 55 bits, angles up to 2^51."""
    x, pos, _, _ = _inputs(60, 2, 64, 32, 1, (1 << 31) - 1, seed=7)
    pos[0, 0], pos[0, 1] = (1 << 31) - 1, -(1 << 31)
    inv = (torch.rand(32, generator=torch.Generator().manual_seed(8)) + 1) * (most / 2)
    inv[0], inv[1] = most, -most
    out = torch.empty_like(x, device="cuda")
    ssd.ssd_rope_axes(x.cuda(), out, 60, 2, 64, "f32", pos.cuda(), inv.cuda())
    _check(out, x, pos, None, inv, ssd.SSD_ROPE_HALF, False, "f32")


@pytest.mark.parametrize("dtype,gap,at", [("bf16", 256, 0), ("bf16", 3, 1), ("f32", 1, 0), ("f32", 6, 2), ("bf16", 4, 4), ("bf16", 2, 2)])
def test_strides_and_odd_addresses(dtype, gap, at):
    """Heads inside a projection's rows, which may lie at any element; the rest of the rows stays."""
    n, H, d = 37, 3, 64
    x, pos, axis, inv = _inputs(n, H, d, 32, 3, 900, seed=3)
    wide = torch.full((n, H * d + gap + at), 5.0, dtype=TORCH[dtype])
    wide[:, at:at + H * d] = x.flatten(1)
    x = wide[:, at:at + H * d].reshape(n, H, d).clone()
    for layout in (ssd.SSD_ROPE_HALF, ssd.SSD_ROPE_INTERLEAVED):
        w = wide.cuda()
        out = torch.empty((n, H, d), dtype=w.dtype, device="cuda")
        ssd.ssd_rope_axes(w[:, at:at + H * d], out, n, H, d, dtype, pos.cuda(), inv.cuda(), axis=axis.cuda(), n_axes=3, layout=layout)
        _check(out, x, pos, axis, inv, layout, False, dtype)
        ssd.ssd_rope_axes(w[:, at:at + H * d], w[:, at:at + H * d], n, H, d, dtype, pos.cuda(), inv.cuda(), axis=axis.cuda(), n_axes=3, layout=layout)
        assert torch.equal(w[:, at:at + H * d].reshape(n, H, d), out)
        assert torch.all(w[:, :at] == 5.0) and torch.all(w[:, at + H * d:] == 5.0)


def test_axes_that_do_not_exist_leave_pairs_as_they_are():
    x, pos, _, inv = _inputs(10, 2, 64, 32, 2, 900, seed=4)
    axis = torch.tensor([0, 1, 2, 255] * 8, dtype=torch.uint8)
    out = torch.empty_like(x, device="cuda")
    ssd.ssd_rope_axes(x.cuda(), out, 10, 2, 64, "f32", pos.cuda(), inv.cuda(), axis=axis.cuda(), n_axes=2)
    _check(out, x, pos, axis, inv, ssd.SSD_ROPE_HALF, False, "f32")
    o = out.cpu()
    assert torch.equal(o[..., 2::4], x[..., 2::4]) and torch.equal(o[..., 3::4], x[..., 3::4])


def test_inverse_is_the_gradient():
    """Against the formula's transpose, and against differences: the rotation is linear, so (f(x + h e) - f(x)) / h is a column of it."""
    x, pos, axis, inv = _inputs(3, 1, 16, 8, 3, 50, seed=5)
    up = torch.randn(x.shape, generator=torch.Generator().manual_seed(6))
    grad = torch.empty_like(x, device="cuda")
    more = dict(axis=axis.cuda(), n_axes=3, layout=ssd.SSD_ROPE_INTERLEAVED)
    ssd.ssd_rope_axes(up.cuda(), grad, 3, 1, 16, "f32", pos.cuda(), inv.cuda(), inverse=True, **more)
    base = mx.rope(x.double().numpy(), pos.numpy(), inv.numpy(), axis.numpy(), "interleaved")
    for t in range(3):
        for e in range(16):
            moved = x.double().numpy().copy()
            moved[t, 0, e] += 0.5
            slope = (mx.rope(moved, pos.numpy(), inv.numpy(), axis.numpy(), "interleaved") - base) / 0.5
            assert abs(float((slope * up.double().numpy()).sum()) - float(grad[t, 0, e])) <= 1e-5
    # and with the library's own forward: <f(x), up> = <x, f'(up)>
    out = torch.empty_like(x, device="cuda")
    ssd.ssd_rope_axes(x.cuda(), out, 3, 1, 16, "f32", pos.cuda(), inv.cuda(), **more)
    assert abs(float((out.double() * up.cuda().double()).sum() - (x.cuda().double() * grad.double()).sum())) <= 1e-5


def test_infinities_and_nan_stay_in_their_pairs_and_graphs_follow_positions():
    x, pos, axis, inv = _inputs(4, 2, 64, 32, 1, 900, seed=7)
    x[1, 0, 3], x[2, 1, 40] = float("inf"), float("nan")
    xd, out, posd = x.cuda(), torch.empty_like(x, device="cuda"), pos.cuda()
    g = torch.cuda.CUDAGraph()
    ssd.ssd_rope_axes(xd, out, 4, 2, 64, "f32", posd, inv.cuda())
    torch.cuda.synchronize()
    invd = inv.cuda()
    with torch.cuda.graph(g):
        ssd.ssd_rope_axes(xd, out, 4, 2, 64, "f32", posd, invd)
    for i in range(3):
        posd += 17
        g.replay()
        torch.cuda.synchronize()
        clean = torch.where(torch.isfinite(x), x, torch.zeros_like(x))
        bad = torch.zeros(x.shape, dtype=torch.bool)
        bad[1, 0, [3, 35]], bad[2, 1, [8, 40]] = True, True
        o = out.cpu()
        assert not torch.isfinite(o[bad]).any() and torch.isfinite(o[~bad]).all()
        _check(torch.where(bad, torch.zeros_like(o), o), torch.where(bad, torch.zeros_like(x), clean), posd.cpu(), None, inv, ssd.SSD_ROPE_HALF, False, "f32")


def test_no_rows():
    x = torch.full((4, 8), 3.0, device="cuda")
    ssd.ssd_rope_axes(x, x, 0, 1, 8, "f32", torch.zeros((1, 0), dtype=torch.int32, device="cuda"), torch.ones(4, device="cuda"))
    assert torch.all(x == 3.0)
