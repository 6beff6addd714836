"""GPU: elements of V that are infinite, against the 64-bit implementation.  They give what their definition gives: p * inf is an infinity of its sign, as
long as p is not nothing; infinities of both signs in a column give NaN; the other columns stay what they are."""
import numpy as np
import pytest
import torch

import paper_2510_18716_amd as ssd
from oracle import paged
from paged_harness import TORCH, Batch, attend

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)


def compare(bt, out, lens=None):
    """Tolerance of the finite columns: that of paged_harness.check_attend."""
    o = out.float().cpu().numpy()
    kp, vp = bt.k.float().numpy(), bt.v.float().numpy()
    for b, n in enumerate(bt.lens if lens is None else lens):
        with np.errstate(invalid="ignore"):
            ref, _, _, size = paged.paged_attend(bt.q[b].float().numpy(), kp, vp, bt.table[b], n, bt.d ** -0.5)
        np.testing.assert_array_equal(np.isnan(o[b]), np.isnan(ref), err_msg=str((b, n)))
        inf, fine = np.isinf(ref), np.isfinite(ref)
        np.testing.assert_array_equal(o[b][inf], ref[inf], err_msg=str((b, n)))
        tol = 5e-5 * size[fine] if bt.dtype == "f32" else 2.0 ** -8 * (size[fine] + np.abs(ref[fine]))
        assert np.all(np.abs(o[b][fine] - ref[fine]) <= tol + 1e-30), (b, n)


def plant(bt, b, row, columns, value):
    bt.v[bt.table[b, row // bt.page], :, row % bt.page, columns] = value


@pytest.mark.parametrize("dtype,d,H,n_kv", [("bf16", 128, 8, 2), ("bf16", 64, 3, 3), ("f32", 64, 4, 1), ("f32", 128, 2, 2), ("bf16", 128, 17, 1)])
@pytest.mark.parametrize("page", [16, 3])
def test_infinite_elements_of_v(dtype, d, H, n_kv, page):
    say("infinite v", dtype, d, H, n_kv, page)
    bt = Batch([1, 2, 40, 300, 2500, 33], H, n_kv, d, dtype, page, seed=d + H + page)
    rng = np.random.default_rng(page)
    for b, n in enumerate(bt.lens):
        for i, row in enumerate(sorted({0, n - 1, n // 2, int(rng.integers(n)), int(rng.integers(n))})):
            plant(bt, b, row, 3 * i, float("inf"))
            plant(bt, b, row, 3 * i + 1, float("-inf"))
            plant(bt, b, row, d - 1, float("inf"))               # a column that several rows have one in
            plant(bt, b, row, d - 2, float("inf") if i % 2 else float("-inf"))     # of both signs, where there are two rows
    bt.vd = bt.v.cuda()
    for weights in (False, True):
        compare(bt, attend(bt, weights=weights)[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("up", [False, True])
def test_infinite_elements_of_rows_of_little_weight(dtype, up):
    """Probabilities down to 2^-86, before and behind the rows that take everything."""
    n, d = 400, 64
    bt = Batch([n, n, 30], 2, 1, d, dtype, 16, seed=3)
    ramp = torch.linspace(-0.5, 0.5, n) * (1 if up else -1)
    for b, m in enumerate(bt.lens):
        bt.q[b] = torch.tensor([480.0] + [0.0] * (d - 1)).to(TORCH[dtype])
        for j in range(m):
            bt.k[bt.table[b, j // 16], :, j % 16, 0] = ramp[j * n // m].to(TORCH[dtype])
        for i in range(10):
            plant(bt, b, i * (m - 1) // 9, 2 * i, float("inf") if i % 3 else float("-inf"))
    bt.kd, bt.vd, bt.qd = bt.k.cuda(), bt.v.cuda(), bt.q.cuda()
    compare(bt, attend(bt)[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_elements_of_the_new_row(dtype):
    lens = [1, 17, 300, 1500, 0]
    bt = Batch(lens, 4, 2, 128, dtype, 16, seed=8)
    g = torch.Generator().manual_seed(2)
    k_new, v_new = (torch.randn((len(lens), 2, 128), generator=g).to(TORCH[dtype]) for _ in range(2))
    v_new[:, :, 5], v_new[:, 0, 100] = float("inf"), float("-inf")
    out = torch.empty((len(lens), 4, 128), dtype=TORCH[dtype], device="cuda")
    ssd.ssd_paged_decode_step(bt.cfg, bt.qd, k_new.cuda(), v_new.cuda(), bt.kd, bt.vd, bt.tabled, bt.lend, out,
                              workspace=bt.scratch(ssd.ssd_paged_workspace_bytes(bt.cfg, 0, False)))
    for b, n in enumerate(lens):
        if n:
            at = (int(bt.table[b, (n - 1) // 16]), slice(None), (n - 1) % 16)
            bt.k[at], bt.v[at] = k_new[b], v_new[b]
    compare(bt, out)
