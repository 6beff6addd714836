"""GPU: sequences whose logits are all minus infinity give what a sequence without rows gives; rows with such a logit beside others weigh nothing."""
import numpy as np
import pytest
import torch

import paper_2510_18716_amd as ssd
from oracle import paged
from paged_harness import TORCH, Batch, attend, fine_tolerance

pytestmark = pytest.mark.gpu

LENS = [1, 40, 300, 2500, 2500, 70, 0]


@pytest.mark.parametrize("dtype,d,H,n_kv", [("bf16", 128, 4, 2), ("f32", 64, 3, 1), ("bf16", 64, 20, 1)])
@pytest.mark.parametrize("step", [False, True])
@pytest.mark.parametrize("lens", [LENS, [100, 5, 64, 0]])
def test_rows_whose_logits_are_minus_infinity(dtype, d, H, n_kv, step, lens):
    print("minus infinity", dtype, d, H, n_kv, step, lens, flush=True)
    bt = Batch(lens, H, n_kv, d, dtype, 16, seed=d)
    bt.q[:, :, 0] = bt.q[:, :, 0].abs() + 0.5
    rng = np.random.default_rng(3)
    off = [np.ones(n, bool) if b % 3 != 1 else rng.random(n) < 0.5 for b, n in enumerate(lens)]       # every third sequence keeps some rows
    for b, n in enumerate(lens):
        for j in np.nonzero(off[b])[0]:
            bt.k[bt.table[b, j // 16], :, j % 16, 0] = float("-inf")
    bt.kd, bt.qd = bt.k.cuda(), bt.q.cuda()
    if step:
        at = [(int(bt.table[b, (n - 1) // 16]), (n - 1) % 16) if n else (0, 0) for b, n in enumerate(lens)]
        k_new, v_new = (torch.stack([x[p, :, i] for p, i in at]).nan_to_num(0.0, neginf=float("-inf")).cuda() for x in (bt.k, bt.v))
        out, lse = torch.full((len(lens), H, d), 7.0, dtype=TORCH[dtype], device="cuda"), torch.full((len(lens), H), 7.0, device="cuda")
        w_in = bt.weight.clone()
        for (p, i), n in zip(at, lens):
            if n:
                w_in[p, :, i] = 0.0
        w = torch.full_like(w_in, -3.0).cuda()
        ssd.ssd_paged_decode_step(bt.cfg, bt.qd, k_new, v_new, bt.kd, bt.vd, bt.tabled, bt.lend, out, lse=lse, weight_in=bt.weight.cuda(), weight_out=w,
                                  workspace=bt.scratch(ssd.ssd_paged_workspace_bytes(bt.cfg, 0, True)))
    else:
        out, lse, w = attend(bt)
        w_in = bt.weight
    for b, n in enumerate(lens):
        if off[b].all():
            assert bool((out[b] == 0).all()) and bool((lse[b] == -float("inf")).all())
            p = np.zeros((H, n))
        else:
            ref, ref_lse, p, size = paged.paged_attend(bt.q[b].float().numpy(), bt.k.float().numpy(), bt.v.float().numpy(), bt.table[b], n, d ** -0.5)
            assert np.all(np.abs(out[b].float().cpu().numpy() - ref) <= fine_tolerance(dtype, ref, size))
            assert np.all(np.abs(lse[b].cpu().numpy() - ref_lse) <= 5e-5 + 1e-6 * np.abs(ref_lse))
        for j in range(n):
            page, place = paged.slot_place(bt.table[b], j, 16)
            add = p[:, j].reshape(n_kv, -1).sum(1)
            want = w_in[page, :, place].double().numpy() + add
            assert np.all(np.abs(w[page, :, place].cpu().numpy() - want) <= 5e-5 * add + 2.0 ** -23 * np.abs(want) + 1e-30), (b, j)
