"""GPU: the paged attention's forms for more than 16 query heads per key head where rows are dealt to the workgroups, and for many sequences in the order of
their lengths."""
import numpy as np
import pytest
import torch

import paper_2510_18716_amd as ssd
from oracle import paged
from paged_harness import TORCH, Batch, attend, check_attend, check_outputs

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)


LENS = [2500, 3, 0, 1023, 700, 129]


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("H,n_kv", [(17, 1), (48, 2), (40, 1), (32, 1)])
def test_tiles_of_query_heads_where_rows_are_dealt(dtype, d, H, n_kv):
    say("tiles", dtype, d, H, n_kv)
    bt = Batch(LENS, H, n_kv, d, dtype, 16, seed=H + d)
    for weights in (True, False):
        got = attend(bt, weights=weights)
        check_attend(bt, got, weights=weights)
        check_outputs(bt, got[0])


@pytest.mark.parametrize("dtype,d,H,n_kv,page", [("bf16", 128, 17, 1, 16), ("f32", 64, 48, 2, 7), ("bf16", 64, 40, 1, 32), ("bf16", 128, 64, 2, 1)])
@pytest.mark.parametrize("weights", [True, False])
def test_steps_of_tiles_of_query_heads_where_rows_are_dealt(dtype, d, H, n_kv, page, weights):
    say("step of tiles", dtype, d, H, n_kv, page, weights)
    bt = Batch(LENS, H, n_kv, d, dtype, page, seed=H)
    g = torch.Generator().manual_seed(7)
    k_new, v_new = (torch.randn((len(LENS), n_kv, d), generator=g).to(TORCH[dtype]) for _ in range(2))
    out, lse = torch.empty((len(LENS), H, d), dtype=TORCH[dtype], device="cuda"), torch.empty((len(LENS), H), device="cuda")
    pos = bt.pos.cuda()
    w_out = torch.full_like(bt.weight, -3.0).cuda() if weights else None
    ssd.ssd_paged_decode_step(bt.cfg, bt.qd, k_new.cuda(), v_new.cuda(), bt.kd, bt.vd, bt.tabled, bt.lend, out, pos=pos, seq_pos=bt.lend + 5, lse=lse,
                              weight_in=bt.weight.cuda() if weights else None, weight_out=w_out,
                              workspace=bt.scratch(ssd.ssd_paged_workspace_bytes(bt.cfg, 0, weights)))
    k, v, rp, rw = bt.k.float().numpy(), bt.v.float().numpy(), bt.pos.numpy().copy(), bt.weight.numpy().copy()
    paged.paged_append(k, v, rp, rw, bt.table, LENS, [n + 5 for n in LENS], k_new.float().numpy(), v_new.float().numpy(), None, None)
    np.testing.assert_array_equal(bt.kd.float().cpu().numpy(), k)
    np.testing.assert_array_equal(bt.vd.float().cpu().numpy(), v)
    np.testing.assert_array_equal(pos.cpu().numpy(), rp)
    bt.k, bt.v = torch.from_numpy(k).to(TORCH[dtype]), torch.from_numpy(v).to(TORCH[dtype])
    check_attend(bt, (out, lse, w_out), weight_before=torch.from_numpy(rw))
    check_outputs(bt, out)


@pytest.mark.parametrize("B,H,n_kv,dtype,most", [(100, 11, 11, "bf16", 640), (128, 9, 9, "f32", 320), (65, 16, 16, "bf16", 300), (90, 102, 6, "bf16", 500)])
def test_many_sequences_in_the_order_of_their_lengths(B, H, n_kv, dtype, most):
    """More than 1024 units of three to five rounds, more than 64 sequences: two lengths in every lane."""
    rng = np.random.default_rng(B)
    lens = [int(x) for x in rng.integers(0, most + 1, B)]
    lens[1], lens[B - 1], lens[B - 2], lens[70 % B] = most, most, 0, 1
    lens[3:9] = [77] * 6                                          # equal ones
    say("by length", B, H, n_kv, dtype, most)
    bt = Batch(lens, H, n_kv, 64, dtype, 16, seed=B, more_blocks=0)
    assert bt.max_blocks == -(-most // 16)
    for weights in (True, False):
        got = attend(bt, weights=weights)
        check_attend(bt, got, weights=weights)
        check_outputs(bt, got[0])
