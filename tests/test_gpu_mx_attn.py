"""Attention and steps over pages held in 8 or 4 bits, and eviction from them, against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2510_18716_amd as ssd
from mx_harness import MxBatch, attend, check, check_written, new_rows, same_pools
from oracle import mx, paged
from paged_harness import evict_sources

pytestmark = pytest.mark.gpu

EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 200, 255, 256, 257, 300]

#         H, kv, d, dtype, fmt, page, layout
SHAPES = [(4, 4, 128, "bf16", "mxfp4", 16, "heads"), (8, 2, 128, "bf16", "mxfp8", 32, "rows"), (10, 2, 64, "f32", "mxfp8", 24, "rows"), (3, 3, 64, "bf16", "mxfp4", 64, "both"),
          (16, 1, 128, "f32", "mxfp4", 16, "wide"), (2, 1, 64, "bf16", "mxfp8", 1, "heads"), (7, 1, 128, "bf16", "mxfp4", 7, "heads"), (34, 2, 64, "f32", "mxfp4", 48, "heads"),
          (5, 1, 128, "f32", "mxfp8", 128, "heads"), (32, 1, 128, "bf16", "mxfp8", 16, "heads"), (2, 2, 64, "bf16", "mxfp4", 12, "rows"), (4, 2, 64, "bf16", "mxfp8", 16, "both")]


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("H,n_kv,d,dtype,fmt,page,layout", SHAPES)
def test_attention_at_the_edges_of_tiles_and_pages(H, n_kv, d, dtype, fmt, page, layout, weights):
    bt = MxBatch(EDGES, H, n_kv, d, dtype, fmt, page, seed=1, layout=layout)
    check(bt, attend(bt, weights=weights))
    for max_len in (1, 33, 130):                                    # longer sequences are cut to the bound
        check(bt, attend(bt, weights=weights, max_len=max_len), max_len=max_len)


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("H,n_kv,d,dtype,fmt,page,layout", SHAPES)
def test_long_and_short_sequences_together(H, n_kv, d, dtype, fmt, page, layout, weights):
    bt = MxBatch([3000, 5, 0, 1201, 64, 4097], H, n_kv, d, dtype, fmt, page, seed=2, layout=layout)
    check(bt, attend(bt, weights=weights))


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("H,n_kv,d,dtype,fmt,page,layout", SHAPES)
def test_steps(H, n_kv, d, dtype, fmt, page, layout, weights):
    for lens in (EDGES, [2500, 0, 1, 700, 1025]):
        bt = MxBatch(lens, H, n_kv, d, dtype, fmt, page, seed=3, layout=layout)
        step = new_rows(bt, len(lens), seed=4, scale=2.0)
        check(bt, attend(bt, weights=weights, step=step), step=step)
        check_written(bt, step)


@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
@pytest.mark.parametrize("n_kv,B,n", [(16, 80, 100), (32, 64, 33), (8, 40, 640)])
def test_many_units(fmt, n_kv, B, n):
    """Units of a wave's, and of a workgroup's dealt by length."""
    lens = [1 + (37 * i) % n for i in range(B)]
    bt = MxBatch(lens, n_kv, n_kv, 64, "bf16", fmt, 16, seed=5)
    check(bt, attend(bt))
    step = new_rows(bt, B, seed=6)
    check(bt, attend(bt, step=step), step=step)
    check_written(bt, step)


@pytest.mark.parametrize("H,n_kv,dtype,fmt,page", [(128, 8, "bf16", "mxfp4", 16), (128, 8, "f32", "mxfp8", 7), (40, 8, "bf16", "mxfp8", 20)])
def test_weights_from_logits_in_lds_at_their_largest(H, n_kv, dtype, fmt, page):
    """Units of up to 1000 rows taken whole, up to sixteen query heads on a key head."""
    lens = [1000 - 31 * i if i % 3 else i for i in range(33)]
    bt = MxBatch(lens, H, n_kv, 64, dtype, fmt, page, seed=23, layout="rows")
    check(bt, attend(bt))


@pytest.mark.parametrize("n_kv,q", [(4, 2), (1, 5), (3, 17)])
def test_runs_that_begin_and_end_anywhere(n_kv, q):
    """Many units of one or a few rounds between long ones: runs that begin, end or lie in what a unit costs besides its rounds."""
    for fmt in ("mxfp4", "mxfp8"):
        lens = [5000, 1, 0, 130, 127, 900, 3, 2600, 0, 0, 129, 64, 1500, 31, 400]
        bt = MxBatch(lens, n_kv * q, n_kv, 64, "bf16", fmt, 32, seed=24)
        for max_len in (0, 2000):
            check(bt, attend(bt, max_len=max_len), max_len=max_len)
        step = new_rows(bt, len(lens), seed=25)
        check(bt, attend(bt, step=step), step=step)
        check_written(bt, step)


def test_more_than_256_sequences_dealt():
    bt = MxBatch([1 + (53 * i) % 90 for i in range(299)] + [4000], 2, 1, 64, "bf16", "mxfp4", 16, seed=7)
    check(bt, attend(bt, weights=True))
    step = new_rows(bt, 300, seed=26)
    check(bt, attend(bt, step=step), step=step)
    check_written(bt, step)


def test_pages_that_do_not_exist():
    """Rows of a block that names no page are masked, all of a sequence's among them; a step's row without a page is not written."""
    for fmt, page in (("mxfp4", 16), ("mxfp8", 24)):
        bt = MxBatch([100, 40, 65, 700], 4, 2, 128, "bf16", fmt, page, seed=8)
        bt.table[0, 1], bt.table[1, :2], bt.table[2, 64 // page], bt.table[3, 3] = -1, bt.n_pages, 1 << 30, -2
        bt.to_device()
        for weights in (False, True):
            check(bt, attend(bt, weights=weights))
        step = new_rows(bt, 4, seed=9)
        got = attend(bt, step=step)
        check(bt, got, step=step)
        check_written(bt, step)


def test_lengths_outside_the_bounds():
    bt = MxBatch([50, 30], 4, 4, 64, "bf16", "mxfp4", 16, seed=10, more_blocks=0)
    bt.lend[1] = -5
    bt.lens[1] = 0
    check(bt, attend(bt))
    bt.lend[0] = 1 << 30
    bt.lens[0] = bt.max_blocks * 16
    j = np.arange(50, bt.lens[0])
    bt.codes[0][bt.table[0][j // 16], :, j % 16] = 0                # the rows it then has
    bt.codes[1][bt.table[0][j // 16], :, j % 16] = 0
    for s in bt.scales:
        s[bt.table[0][j // 16], :, j % 16] = 127
    bt.weight[bt.table[0][j // 16], :, j % 16] = 0.5
    lend = bt.lend
    bt.to_device()
    bt.lend = lend
    check(bt, attend(bt))


def test_nan_blocks_stay_with_their_sequence_and_head():
    for fmt, d in (("mxfp4", 128), ("mxfp8", 64)):
        bt = MxBatch([70, 70, 70], 4, 2, d, "bf16", fmt, 16, seed=11)
        bt.scales[0][bt.table[0, 2], 1, 3, 0] = 255                  # a key of sequence 0, head pair 1
        bt.scales[1][bt.table[1, 1], 0, 5, 1] = 255                  # the second block of a value of sequence 1, head pair 0
        bt.to_device()
        out, lse, w = attend(bt)
        o = out.float().cpu().numpy()
        assert np.isnan(o[0, 2:]).all() and np.isnan(lse[0, 2:].cpu().numpy()).all() and not np.isnan(o[0, :2]).any()
        assert np.isnan(o[1, :2, 32:64]).all() and not np.isnan(np.delete(o[1, :2], np.s_[32:64], -1)).any()
        assert not np.isnan(o[1, 2:]).any() and not np.isnan(o[2]).any() and not np.isnan(lse[1:].cpu().numpy()).any()


def test_large_and_equal_logits():
    bt = MxBatch([300, 300], 2, 1, 128, "f32", "mxfp8", 16, seed=12, qs=30.0)
    check(bt, attend(bt))
    bt.q.zero_()
    bt.to_device()
    check(bt, attend(bt))


def test_given_scale_and_strided_queries():
    bt = MxBatch([90, 20], 6, 3, 64, "f32", "mxfp4", 16, seed=13)
    bt.cfg.softmax_scale = 0.3
    check(bt, attend(bt), scale=float(np.float32(0.3)))
    wide = torch.full((2, 6 * 64 + 128), float("nan"), device="cuda")
    wide[:, :384] = bt.qd.flatten(1)
    bt.cfg.softmax_scale, bt.cfg.q_stride, bt.qd = 0.0, 512, wide[:, :384]
    check(bt, attend(bt))


def test_shared_pages_are_read_by_several_sequences():
    bt = MxBatch([64, 80, 96], 4, 4, 64, "bf16", "mxfp4", 16, seed=14)
    bt.table[1, :4] = bt.table[0, :4]
    bt.table[2, :4] = bt.table[0, :4]
    bt.to_device()
    check(bt, attend(bt, weights=False))


def test_same_bits_twice_and_whatever_the_workspace_held():
    bt = MxBatch([3000, 12, 700], 8, 2, 128, "bf16", "mxfp4", 16, seed=15)
    a = attend(bt)
    b = attend(bt, workspace=torch.zeros(ssd.ssd_paged_mx_workspace_bytes(bt.cfg, "mxfp4", 0, True) // 4 + 64, device="cuda"))
    for x, y in zip(a, b):
        assert torch.equal(x.nan_to_num(9.0), y.nan_to_num(9.0))


def test_the_codes_give_what_plain_pages_of_their_values_give():
    """The same values in a plain fp32 pool: both calls are within their tolerances of each other."""
    bt = MxBatch([500, 33, 257], 8, 2, 64, "f32", "mxfp4", 16, seed=16)
    out, lse, w = attend(bt)
    k, v = (torch.from_numpy(mx.decode(bt.codes[i], bt.scales[i], bt.fmt).astype(np.float32)).cuda().nan_to_num(0.0) for i in range(2))
    cfg = ssd.make_paged_config(3, 8, 2, 64, "f32", 16, bt.n_pages, bt.max_blocks)
    out2, lse2 = torch.empty_like(out), torch.empty_like(lse)
    ws = torch.empty(max(1, ssd.ssd_paged_workspace_bytes(cfg, 0, False)), dtype=torch.uint8, device="cuda")
    ssd.ssd_paged_decode_attn(cfg, bt.qd, k, v, bt.tabled, bt.lend, out2, lse=lse2, workspace=ws)
    assert (out - out2).abs().max() <= 1e-4 * out2.abs().max() and (lse - lse2).abs().max() <= 1e-4


@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
def test_captured_steps_follow_the_lengths(fmt):
    """Two graphs share one workspace; both are replayed several times with eager work between, and every replay is compared with the eager call."""
    make = lambda: MxBatch([700, 30, 0, 129], 8, 2, 128, "bf16", fmt, 16, seed=17, more_blocks=4)  # noqa: E731
    bt, eager = make(), make()
    step = [x.cuda() for x in new_rows(bt, 4, seed=18)]
    ws = torch.zeros(ssd.ssd_paged_mx_workspace_bytes(bt.cfg, fmt, 0, True) // 4 + 64, device="cuda")
    outs = [[torch.zeros((4, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((4, 8), device="cuda"), torch.zeros_like(bt.weightd)] for _ in range(3)]

    def call(b, kind, o, w):
        if kind == "step":
            ssd.ssd_paged_mx_decode_step(b.cfg, fmt, b.qd, *step, *b.pools, b.tabled, b.lend, o[0], pos=b.posd, lse=o[1], weight_in=b.weightd, weight_out=o[2], workspace=w)
        else:
            ssd.ssd_paged_mx_decode_attn(b.cfg, fmt, b.qd, *b.pools, b.tabled, b.lend, o[0], lse=o[1], weight_in=b.weightd, weight_out=o[2], workspace=w)

    graphs = []
    for kind, o in (("step", outs[0]), ("attn", outs[1])):
        call(bt, kind, o, ws)
        call(eager, kind, outs[2], ws)                              # the other pool has the same steps behind it
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(bt, kind, o, ws)
        graphs.append(g)
    for replay in range(4):
        for x in (bt, eager):
            x.lend += torch.tensor([1, 1, 0, 1], dtype=torch.int32, device="cuda")
            x.qd.mul_(0.9)
        for i, kind in enumerate(("step", "attn")):
            graphs[i].replay()
            torch.cuda.synchronize()
            call(eager, kind, outs[2], ws)
            torch.cuda.synchronize()
            for x, y in zip(outs[i], outs[2]):
                assert torch.equal(x.nan_to_num(9.0), y.nan_to_num(9.0)), (replay, kind)
            assert torch.equal(bt.kd, eager.kd) and torch.equal(bt.vsd, eager.vsd) and torch.equal(bt.posd, eager.posd)


def test_two_streams_at_once():
    """Steps with weights of two pools on two streams, each with a workspace of its own: the bits of either alone."""
    batches = [MxBatch([3000, 40, 900], 8, 2, 128, "bf16", "mxfp8", 16, seed=27), MxBatch([2000, 1999, 7, 0], 4, 4, 64, "f32", "mxfp4", 24, seed=28)]
    calls = []
    for i, bt in enumerate(batches):
        step = [x.cuda() for x in new_rows(bt, len(bt.lens), seed=29 + i)]
        ws = bt.scratch(ssd.ssd_paged_mx_workspace_bytes(bt.cfg, bt.fmt, 0, True))
        o = [torch.zeros((len(bt.lens), bt.H, bt.d), dtype=bt.qd.dtype, device="cuda"), torch.zeros((len(bt.lens), bt.H), device="cuda"), torch.zeros_like(bt.weightd)]
        calls.append((bt, step, ws, o, torch.cuda.Stream()))

    def call(bt, step, ws, o, stream):
        ssd.ssd_paged_mx_decode_step(bt.cfg, bt.fmt, bt.qd, *step, *bt.pools, bt.tabled, bt.lend, o[0], pos=bt.posd, lse=o[1], weight_in=bt.weightd, weight_out=o[2],
                                     workspace=ws, stream=stream)

    alone = []
    for c in calls:
        torch.cuda.synchronize()
        call(*c)
        torch.cuda.synchronize()
        alone.append([x.clone() for x in c[3]])
    for _ in range(5):
        for x in calls[0][3] + calls[1][3]:
            x.zero_()
        torch.cuda.synchronize()
        for _ in range(10):
            for c in calls:
                call(*c)
        torch.cuda.synchronize()
        for c, want in zip(calls, alone):
            for x, y in zip(c[3], want):
                assert torch.equal(x, y)


def test_captured_rotation_append_and_read_follow_positions_and_lengths():
    """A chunk of rows rotated, stored and read back as one graph, replayed while lengths and positions go on; every replay against the eager calls."""
    fmt, n, n_kv, d = "mxfp4", 6, 2, 64
    make = lambda: MxBatch([40, 90], 2, n_kv, d, "bf16", fmt, 16, seed=30, more_blocks=3, spare=6)  # noqa: E731
    pair = []
    for _ in range(2):
        bt = make()
        bt.table[0, 3:6], bt.table[1, 6:9] = [p for p in range(bt.n_pages) if p not in bt.table][:3], [p for p in range(bt.n_pages) if p not in bt.table][3:6]
        bt.to_device()
        k, v = (x.cuda() for x in new_rows(bt, n, seed=31))
        at = torch.tensor([[38, 39, 87, 88, 89, 90]], dtype=torch.int32, device="cuda")
        pair.append((bt, k, torch.zeros_like(k), v, at, torch.zeros_like(k), torch.zeros_like(k)))
    start = torch.tensor([0, 2, 6], dtype=torch.int32, device="cuda")
    inv = torch.tensor([10000.0 ** (-i / 32) for i in range(32)], device="cuda")

    def call(bt, k, turned, v, at, k_out, v_out):
        ssd.ssd_rope_axes(k, turned, n, n_kv, d, "bf16", at, inv)
        ssd.ssd_paged_mx_append(bt.cfg, fmt, *bt.pools, bt.tabled, bt.lend, turned, v, pos=bt.posd, new_start=start)
        ssd.ssd_paged_mx_read(bt.cfg, fmt, *bt.pools, bt.tabled, bt.lend, k_out, v_out, row_start=start, first_slot=first)

    first = pair[0][0].lend - torch.tensor([2, 4], dtype=torch.int32, device="cuda")
    for x in pair:
        call(*x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(*pair[0])
    for replay in range(5):
        for x in pair:
            x[0].lend += torch.tensor([2, 4], dtype=torch.int32, device="cuda")
            x[4].add_(3)
            x[1].mul_(-1.25)
        first += torch.tensor([2, 4], dtype=torch.int32, device="cuda")
        graph.replay()
        torch.cuda.synchronize()
        call(*pair[1])
        torch.cuda.synchronize()
        for i in (2, 5, 6):
            assert torch.equal(pair[0][i], pair[1][i]), (replay, i)
        for x, y in zip(pair[0][0].pools + (pair[0][0].posd,), pair[1][0].pools + (pair[1][0].posd,)):
            assert torch.equal(x, y), replay
        held = mx.held(pair[0][2].double().cpu().numpy(), fmt)
        assert np.array_equal(pair[0][5].float().cpu().numpy(), held), replay


@pytest.mark.parametrize("fmt,dtype,d,page,n_kv,lens,budget", [("mxfp4", "bf16", 128, 16, 2, [129, 129, 40, 0], 128), ("mxfp8", "f32", 64, 24, 3, [500, 1000, 10], 100),
                                                              ("mxfp4", "f32", 64, 1, 1, [60, 61], 33), ("mxfp8", "bf16", 128, 32, 8, [3000, 900], 1000),
                                                              ("mxfp4", "bf16", 64, 16, 1, [20000, 17000], 5000)] +
                                                             [("mxfp4", "bf16", 128, 16, 16, [129] * 16, 120)])
def test_eviction_moves_codes_and_scales(fmt, dtype, d, page, n_kv, lens, budget):
    bt = MxBatch(lens, n_kv, n_kv, d, dtype, fmt, page, seed=19, spread=False)
    rng = np.random.default_rng(20)
    bt.weight[...] = rng.integers(0, 50, bt.weight.shape)
    for in_place in (False, True):
        bt.to_device()
        po, wo = (bt.posd, bt.weightd) if in_place else (torch.full_like(bt.posd, -1), torch.full_like(bt.weightd, -1.0))
        after = torch.zeros_like(bt.lend)
        bud = torch.full_like(bt.lend, budget)
        ws = bt.scratch(ssd.ssd_paged_mx_evict_workspace_bytes(bt.cfg, fmt, 0))
        ssd.ssd_paged_mx_evict(bt.cfg, fmt, *bt.pools, bt.tabled, bt.lend, bud, bt.posd, po, bt.weightd, wo, after, n_sink=2, recent=5, workspace=ws)
        codes, scales = [x.copy() for x in bt.codes], [x.copy() for x in bt.scales]
        pos, weight = po.cpu().numpy(), wo.cpu().numpy()
        for b, n in enumerate(lens):
            j = np.arange(n)
            pages, places = bt.table[b][j // page], j % page
            stay = min(n, budget)
            for kv in range(n_kv):
                src = evict_sources(bt.pos[pages, kv, places], bt.weight[pages, kv, places], n, budget, 2, 5, np.ones(n, bool))
                to = (pages[:stay], kv, places[:stay])
                frm = (pages[src], kv, places[src])
                for i in range(2):
                    codes[i][to], scales[i][to] = bt.codes[i][frm], bt.scales[i][frm]
                assert np.array_equal(pos[to], bt.pos[frm]) and np.array_equal(weight[to], bt.weight[frm]), (b, kv)
        same_pools(bt, codes, scales)
        assert after.cpu().tolist() == [min(n, budget) for n in lens]


def test_a_run_of_all_calls():
    """Prompts rotated and quantised, cut to a budget, then steps with rotated rows: after every step the attention is that over the rows read back."""
    H, n_kv, d, page, fmt, budget = 8, 2, 64, 16, "mxfp8", 40
    prompts = [70, 9, 33]
    B, n, width = 3, sum(prompts), (H + 2 * n_kv) * d
    g = torch.Generator().manual_seed(21)
    bt = MxBatch([0] * B, H, n_kv, d, "bf16", fmt, page, seed=22, spare=B * 6, more_blocks=5)
    bt.table = np.arange(B * 6, dtype=np.int32).reshape(B, 6)
    bt.weight[...] = 0
    bt.to_device()
    inv = torch.tensor([10000.0 ** (-i / 32) for i in range(32)], device="cuda")
    axis = torch.tensor([i % 3 for i in range(32)], dtype=torch.uint8, device="cuda")
    bt.cfg.new_stride = bt.cfg.q_stride = width
    ws = torch.zeros(1 << 20, device="cuda")

    def project(rows, pos):
        x = torch.randn((rows, width), generator=g).to(torch.bfloat16).cuda()
        ssd.ssd_rope_axes(x, x, rows, H + n_kv, d, "bf16", pos, inv, axis=axis, n_axes=3)
        return x, x[:, :H * d], x[:, H * d:(H + n_kv) * d], x[:, (H + n_kv) * d:]

    bt.lend = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    total = bt.lend.clone()
    start = torch.tensor([0, 70, 79, 112], dtype=torch.int32, device="cuda")
    t = torch.cat([torch.arange(p) for p in prompts]).to(torch.int32).cuda()
    _, _, k, v = project(n, torch.stack([t, t // 6, t % 6]))
    ssd.ssd_paged_mx_append(bt.cfg, fmt, *bt.pools, bt.tabled, bt.lend, k, v, pos=bt.posd, weight=bt.weightd, new_start=start, weight_new=torch.rand((n, n_kv), device="cuda"))
    lens = list(prompts)
    for step in range(12):
        if step % 5 == 0:
            after = torch.zeros_like(bt.lend)
            ssd.ssd_paged_mx_evict(bt.cfg, fmt, *bt.pools, bt.tabled, bt.lend, torch.full_like(bt.lend, budget), bt.posd, bt.posd, bt.weightd, bt.weightd, after, n_sink=1,
                                   recent=4, seq_pos=total, workspace=ws)
            bt.lend, lens = after, [min(x, budget) for x in lens]
            assert after.cpu().tolist() == lens
        bt.lend, total, lens = bt.lend + 1, total + 1, [x + 1 for x in lens]
        _, q, k, v = project(B, torch.stack([total, total // 6, total % 6]))
        out, lse, wout = torch.zeros((B, H, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((B, H), device="cuda"), bt.weightd.clone()
        ssd.ssd_paged_mx_decode_step(bt.cfg, fmt, q, k, v, *bt.pools, bt.tabled, bt.lend, out, pos=bt.posd, seq_pos=total, lse=lse, weight_in=bt.weightd, weight_out=wout,
                                     workspace=ws)
        bt.codes, bt.scales = [bt.kd.cpu().numpy(), bt.vd.cpu().numpy()], [bt.ksd.cpu().numpy(), bt.vsd.cpu().numpy()]
        bt.lens, bt.q = lens, q.cpu().reshape(B, H, d)
        check(bt, (out, lse, None))
        newest = [int(bt.posd[bt.table[b, (lens[b] - 1) // page], 0, (lens[b] - 1) % page]) for b in range(B)]
        assert newest == (total - 1).tolist()
        bt.weightd = wout
        for b in range(B):                                          # every token's weight came from softmaxes: H of them a step
            assert np.isfinite(wout.cpu().numpy()[bt.table[b][np.arange(lens[b]) // page], :, np.arange(lens[b]) % page]).all()


@pytest.mark.parametrize("pool,dtype", [("mxfp4", "bf16"), ("mxfp8", "f32")])
def test_the_serving_example_on_a_quantised_pool(pool, dtype):
    import importlib.util
    import os
    import sys
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_serving.py")
    spec = importlib.util.spec_from_file_location("paged_serving", path)
    example = importlib.util.module_from_spec(spec)
    sys.modules["paged_serving"] = example
    spec.loader.exec_module(example)
    s = example.Settings(prompts=(37, 130, 8), budget=40, slack=12, steps=30, dtype=dtype, pool=pool, columns=6)
    calls = []

    def watch(layer, st):
        calls.append(layer)
        if len(calls) % 11 not in (1, 6):                            # some of the 60
            return
        k, v = (mx.decode(x.cpu().numpy(), y.cpu().numpy(), pool) for x, y in zip((st["k"], st["v"]), st["scales"]))
        table, out, q = st["table"].cpu().numpy(), st["out"].float().cpu().numpy(), st["q"].float().cpu().numpy().reshape(6, s.heads, s.head_dim)
        for b, n in enumerate(st["lens"]):
            ref, _, _, size = paged.paged_attend(q[b], k, v, table[b], n, s.head_dim ** -0.5)
            tol = 5e-5 * size if dtype == "f32" else 2.0 ** -8 * (size + np.abs(ref))
            assert np.all(np.abs(out[b] - ref) <= tol + 1e-30), (layer, b)

    tokens, lens, held = example.serve(s, watch)
    assert len(calls) == s.steps * s.layers and tokens.shape == (3, 30)
    assert bool(((tokens >= s.image_tokens[0]) & (tokens < s.image_tokens[1])).all()) and max(lens) <= s.budget + s.slack
