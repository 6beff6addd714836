"""ssd_paged_mx_append and ssd_paged_mx_read against the formats' definition: codes, scales and tables to the bit."""
import numpy as np
import pytest
import torch

import paper_2510_18716_amd as ssd
from mx_harness import MxBatch, new_rows, same_pools
from oracle import mx
from paged_harness import TORCH

pytestmark = pytest.mark.gpu


def _appended(bt, k_new, v_new, new, total=None):
    """The pools, scales, positions and rows touched after `new` tokens for each sequence, in its last slots."""
    codes, scales, pos = [x.copy() for x in bt.codes], [x.copy() for x in bt.scales], bt.pos.copy()
    row = 0
    for b, n_b in enumerate(new):
        for j in range(n_b):
            slot = bt.lens[b] - n_b + j
            if 0 <= slot < min(bt.lens[b], bt.max_blocks * bt.page):
                page, place = bt.table[b, slot // bt.page], slot % bt.page
                if 0 <= page < bt.n_pages:
                    for i, x in enumerate((k_new, v_new)):
                        code, scale = mx.encode(x[row].double().numpy(), bt.fmt)
                        codes[i][page, :, place], scales[i][page, :, place] = mx.pack(code, bt.fmt), scale
                    pos[page, :, place] = (bt.lens[b] if total is None else total[b]) - n_b + j
            row += 1
    return codes, scales, pos


APPENDS = [("mxfp4", "bf16", 128, 32, 16, "heads"), ("mxfp8", "bf16", 128, 4, 32, "rows"), ("mxfp4", "f32", 64, 5, 24, "both"), ("mxfp8", "f32", 64, 1, 1, "wide"),
           ("mxfp4", "bf16", 64, 3, 7, "wide"), ("mxfp8", "f32", 128, 2, 64, "heads"), ("mxfp4", "f32", 128, 1, 5, "rows"), ("mxfp8", "bf16", 64, 40, 16, "heads")]


@pytest.mark.parametrize("fmt,dtype,d,n_kv,page,layout", APPENDS)
def test_append_of_unequal_prompts_and_back(fmt, dtype, d, n_kv, page, layout):
    lens, new = [40, 1, 0, 17, 33, 100], [12, 1, 0, 17, 0, 99]
    bt = MxBatch(lens, n_kv, n_kv, d, dtype, fmt, page, seed=1, layout=layout)
    k_new, v_new = new_rows(bt, sum(new), seed=2, scale=3.0)
    k_new[0, 0, :32] = 0.0                                          # a block of zeros, one with a NaN, one with an infinity, one that is tiny
    k_new[1, 0, 5], v_new[2, 0, 33] = float("nan"), float("-inf")
    v_new[3, 0, 32:] *= 2.0 ** -120
    start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
    total = torch.tensor([n + 9 for n in lens], dtype=torch.int32, device="cuda")
    wn = torch.rand((sum(new), n_kv))
    ssd.ssd_paged_mx_append(bt.cfg, fmt, *bt.pools, bt.tabled, bt.lend, k_new.cuda(), v_new.cuda(), pos=bt.posd, weight=bt.weightd, seq_pos=total, new_start=start,
                            weight_new=wn.cuda())
    codes, scales, pos = _appended(bt, k_new, v_new, new, [n + 9 for n in lens])
    same_pools(bt, codes, scales)
    assert np.array_equal(bt.posd.cpu().numpy(), pos)
    w = bt.weightd.cpu().numpy()
    changed = pos != bt.pos
    assert np.array_equal(w[~changed], bt.weight[~changed], equal_nan=True)
    row = 0
    for b, n_b in enumerate(new):
        for j in range(n_b):
            slot = lens[b] - n_b + j
            assert np.array_equal(w[bt.table[b, slot // page], :, slot % page], wn[row].numpy())
            row += 1
    # the same rows back, and those of all sequences from the first on
    first = torch.tensor([n - m for n, m in zip(lens, new)], dtype=torch.int32, device="cuda")
    for begin, count, starts in ((first, new, start), (None, lens, torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda"))):
        k_out, v_out = (torch.full((sum(count) + 2, n_kv, d), 7.0, dtype=TORCH[dtype], device="cuda") for _ in "kv")
        ssd.ssd_paged_mx_read(bt.cfg, fmt, *bt.pools, bt.tabled, bt.lend, k_out, v_out, row_start=starts, first_slot=begin, n_rows=sum(count))
        for i, out in enumerate((k_out, v_out)):
            want = np.concatenate([bt.rows(i, b, n, codes[i], scales[i])[0][n - c:] for b, (n, c) in enumerate(zip(lens, count))])
            have = out.float().cpu().numpy()
            assert np.array_equal(have[:-2], want.astype(np.float32), equal_nan=True)
            assert np.all(have[-2:] == 7.0)                         # rows beyond the last stay


@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_level_tie_and_size_of_a_block(fmt, dtype):
    """Rows that hold every middle between two levels, at scales over the whole range of the type."""
    lv = mx.levels(fmt)
    points = np.concatenate([lv, (lv[1:] + lv[:-1]) / 2, [7.0 if fmt == "mxfp4" else 464.0]])
    points = np.concatenate([points, -points])
    rows = []
    for E in (-140, -127, -126, -125, -118, -117, -60, -3, 0, 5, 90, 118, 119):
        for i in range(0, len(points), 30):
            part = np.zeros(32)
            part[:len(points[i:i + 30])] = points[i:i + 30]
            part[31] = lv[-1]
            rows.append(part * 2.0 ** E)
            rows.append(part * 2.0 ** E * (1 + 2.0 ** -7))
    while len(rows) % 4:
        rows.append(np.zeros(32))
    x = torch.from_numpy(np.array(rows).reshape(-1, 1, 128).astype(np.float32)).to(TORCH[dtype])
    x = torch.where(torch.isfinite(x), x, torch.zeros_like(x))
    bt = MxBatch([len(x)], 1, 1, 128, dtype, fmt, 16, seed=3)
    ssd.ssd_paged_mx_append(bt.cfg, fmt, *bt.pools, bt.tabled, bt.lend, x.cuda(), x.flip(0).contiguous().cuda(), new_start=torch.tensor([0, len(x)], dtype=torch.int32, device="cuda"))
    codes, scales, _ = _appended(bt, x, x.flip(0), [len(x)])
    same_pools(bt, codes, scales)
    back = torch.empty_like(x, device="cuda")
    ssd.ssd_paged_mx_read(bt.cfg, fmt, *bt.pools, bt.tabled, bt.lend, back, torch.empty_like(back), row_start=torch.tensor([0, len(x)], dtype=torch.int32, device="cuda"))
    with np.errstate(over="ignore"):
        assert np.array_equal(back.float().cpu().numpy(), bt.rows(0, 0, None, codes[0], scales[0])[0].astype(np.float32))


@pytest.mark.parametrize("fmt,d", [("mxfp4", 128), ("mxfp8", 64)])
def test_read_of_every_code_and_scale(fmt, d):
    n = 256
    bt = MxBatch([n], 2, 2, d, "f32", fmt, 16, seed=4)
    rng = np.random.default_rng(5)
    j = np.arange(n)
    pages, places = bt.table[0][j // 16], j % 16
    for i in range(2):
        bt.codes[i][pages, :, places] = rng.integers(0, 256, bt.codes[i][pages, :, places].shape)
        bt.scales[i][pages, :, places] = (j[:, None, None] + i * 7) % 256
    bt.to_device()
    out = [torch.empty((n, 2, d), device="cuda") for _ in "kv"]
    ssd.ssd_paged_mx_read(bt.cfg, fmt, *bt.pools, bt.tabled, bt.lend, *out, row_start=torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    for i in range(2):
        with np.errstate(over="ignore"):
            want = bt.rows(i, 0)[0].astype(np.float32)
        have = out[i].cpu().numpy()
        small = np.abs(want) < 2.0 ** -126                          # such as the library does not write
        assert np.array_equal(np.where(small, 0, have), np.where(small, 0, want), equal_nan=True)
        assert np.all(np.abs(have[small]) < 2.0 ** -126)


def test_one_token_each_some_without_a_place():
    """No starts: one token per sequence.  A sequence without rows, one whose last block names no page and one beyond the table's reach take none."""
    for fmt in ("mxfp4", "mxfp8"):
        bt = MxBatch([5, 0, 16, 33, 40], 4, 4, 128, "bf16", fmt, 16, seed=6)
        bt.table[3, 2] = bt.n_pages
        bt.to_device()
        bt.lend[4] = bt.max_blocks * 16 + 5
        k_new, v_new = new_rows(bt, 5, seed=7)
        ssd.ssd_paged_mx_append(bt.cfg, fmt, *bt.pools, bt.tabled, bt.lend, k_new.cuda(), v_new.cuda(), pos=bt.posd)
        bt.lens[4] = bt.max_blocks * 16 + 5
        codes, scales, pos = _appended(bt, k_new, v_new, [1] * 5)
        same_pools(bt, codes, scales)
        assert np.array_equal(bt.posd.cpu().numpy(), pos)
        out = [torch.full((5, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
        first = torch.tensor([4, 0, 16, -1, 3], dtype=torch.int32, device="cuda")
        bt.lend[4] = 40
        ssd.ssd_paged_mx_read(bt.cfg, fmt, *bt.pools, bt.tabled, bt.lend, *out, first_slot=first)
        for i in range(2):
            have = out[i].float().cpu().numpy()
            assert np.all(have[[1, 2, 3]] == 7.0)                   # no such slot
            assert np.array_equal(have[0], bt.rows(i, 0, 5, codes[i], scales[i])[0][4]) and np.array_equal(have[4], bt.rows(i, 4, 4, codes[i], scales[i])[0][3])


def test_strided_rows_many_sequences_another_stream():
    """More sequences than the starts' place in LDS, rows of a projection, a stream of the caller's."""
    B, n_kv, d = 1500, 2, 64
    lens = [1 + i % 3 for i in range(B)]
    bt = MxBatch(lens, n_kv, n_kv, d, "bf16", "mxfp4", 4, seed=8)
    n = sum(lens)
    wide = torch.full((n, 3 * n_kv * d), float("nan"), dtype=torch.bfloat16)
    k_new, v_new = new_rows(bt, n, seed=9)
    wide[:, :n_kv * d], wide[:, n_kv * d:2 * n_kv * d] = k_new.flatten(1), v_new.flatten(1)
    wide = wide.cuda()
    bt.cfg.new_stride = 3 * n_kv * d
    start = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ssd.ssd_paged_mx_append(bt.cfg, "mxfp4", *bt.pools, bt.tabled, bt.lend, wide[:, :n_kv * d], wide[:, n_kv * d:2 * n_kv * d], new_start=start, stream=s)
    back = torch.zeros_like(wide)
    s.wait_stream(torch.cuda.current_stream())
    ssd.ssd_paged_mx_read(bt.cfg, "mxfp4", *bt.pools, bt.tabled, bt.lend, back[:, n_kv * d:2 * n_kv * d], back[:, 2 * n_kv * d:], row_start=start, stream=s)
    s.synchronize()
    codes, scales, _ = _appended(bt, k_new, v_new, lens)
    same_pools(bt, codes, scales)
    assert not back[:, :n_kv * d].any()
    assert np.array_equal(back[:, n_kv * d:2 * n_kv * d].float().cpu().numpy().reshape(n, n_kv, d), mx.held(k_new.double().numpy(), "mxfp4"))


@pytest.mark.parametrize("fmt,dtype,n_kv,d", [("mxfp4", "bf16", 8, 128), ("mxfp8", "f32", 2, 64)])
def test_many_tokens(fmt, dtype, n_kv, d):
    """Several tokens to a workgroup, runs that end inside one."""
    lens = [1300, 7, 2049, 0, 800, 5000]
    bt = MxBatch(lens, n_kv, n_kv, d, dtype, fmt, 16, seed=10)
    k_new, v_new = new_rows(bt, sum(lens), seed=11)
    start = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    ssd.ssd_paged_mx_append(bt.cfg, fmt, *bt.pools, bt.tabled, bt.lend, k_new.cuda(), v_new.cuda(), pos=bt.posd, new_start=start)
    out = [torch.empty((sum(lens), n_kv, d), dtype=TORCH[dtype], device="cuda") for _ in "kv"]
    ssd.ssd_paged_mx_read(bt.cfg, fmt, *bt.pools, bt.tabled, bt.lend, *out, row_start=start)
    for x, have in zip((k_new, v_new), out):
        assert np.array_equal(have.float().cpu().numpy(), mx.held(x.double().numpy(), fmt).astype(np.float32))
    unheld = np.ones(bt.n_pages, bool)
    unheld[bt.table[bt.table >= 0]] = False
    assert np.all(bt.kd.cpu().numpy()[unheld] == 255) and np.all(bt.vsd.cpu().numpy()[unheld] == 255)
