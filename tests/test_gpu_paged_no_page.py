"""GPU: eviction where entries of the block table name no page.  Their slots hold no row and can take none: the best rows of the others go to those slots
below n' that have a page, and no row is lost or left over but by its rank."""
import numpy as np
import pytest
import torch

import paper_2510_18716_amd as ssd
from paged_harness import evict_sources

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)


def run_case(lens, budgets, n_kv, page, gone, sink, recent, in_place, seed=1, weight_of=None, pos_of=None):
    """gone: per sequence, blocks whose entries name no page.  Rows carry their slot + 1; exact."""
    say("no page", lens, budgets, n_kv, page, gone, sink, recent, in_place, seed)
    rng = np.random.default_rng(seed)
    d, B = 64, len(lens)
    blocks = [-(-n // page) for n in lens]
    n_pages, max_blocks = sum(blocks) + 2, max(blocks + [1])
    order = rng.permutation(n_pages)
    whole = np.full((B, max_blocks), -1, np.int32)
    at = 0
    for b, n in enumerate(blocks):
        whole[b, :n] = order[at:at + n]
        at += n
    table = whole.copy()
    for b, g in enumerate(gone):
        for i, blk in enumerate(g):
            if blk < max_blocks:
                table[b, blk] = (-1, n_pages, 1 << 30, -(1 << 31))[i % 4]
    pos, weight = np.full((n_pages, n_kv, page), -9, np.int32), np.full((n_pages, n_kv, page), np.nan, np.float32)
    rows = np.zeros((n_pages, n_kv, page), np.float32)
    unit = {}
    for b, n in enumerate(lens):
        i = np.arange(n)
        pages, places = whole[b][i // page], i % page
        for kv in range(n_kv):
            p = np.arange(n) if pos_of is None else pos_of(rng, n)
            w = (rng.random(n) if weight_of is None else weight_of(rng, n)).astype(np.float32)
            pos[pages, kv, places], weight[pages, kv, places], rows[pages, kv, places] = p, w, i + 1
            unit[b, kv] = (p, w)
    kd = torch.from_numpy(rows).cuda()[..., None].expand(n_pages, n_kv, page, d).contiguous()
    vd = -kd
    pd, wd = torch.from_numpy(pos).cuda(), torch.from_numpy(weight).cuda()
    po, wo = (pd, wd) if in_place else (torch.full_like(pd, -5), torch.full_like(wd, -5.0))
    want_p, want_w = (pos.copy(), weight.copy()) if in_place else (np.full(pos.shape, -5, np.int32), np.full(pos.shape, -5.0, np.float32))
    want_r = rows.copy()
    cfg = ssd.make_paged_config(B, n_kv, n_kv, d, "f32", page, n_pages, max_blocks)
    ln = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    ws = torch.full((max(64, ssd.ssd_paged_evict_workspace_bytes(cfg, 0) // 4),), float("nan"), device="cuda")
    ssd.ssd_paged_evict(cfg, kd, vd, torch.from_numpy(table).cuda(), ints(lens), ints(budgets), pd, po, wd, wo, ln, n_sink=sink, recent=recent,
                        seq_pos=ints(lens), workspace=ws)
    assert ln.tolist() == [min(n, max(0, m)) for n, m in zip(lens, budgets)]
    for (b, kv), (p, w) in unit.items():
        n = lens[b]
        there = (table[b][np.arange(n) // page] >= 0) & (table[b][np.arange(n) // page] < n_pages)
        src = evict_sources(p, w, n, budgets[b], sink, recent, there)
        to = np.nonzero(there[:len(src)])[0]
        frm = src[to]
        pages, places = whole[b][to // page], to % page
        want_p[pages, kv, places], want_w[pages, kv, places], want_r[pages, kv, places] = p[frm], w[frm], frm + 1
    np.testing.assert_array_equal(po.cpu().numpy(), want_p)
    np.testing.assert_array_equal(wo.cpu().numpy(), want_w)
    for pool, sign in ((kd, 1), (vd, -1)):
        assert torch.equal(pool, (sign * torch.from_numpy(want_r)).cuda()[..., None].expand(pool.shape))


@pytest.mark.parametrize("sink,recent", [(0, 0), (1, 0), (4, 30)])
@pytest.mark.parametrize("in_place", [False, True])
def test_blocks_without_a_page_in_short_units(sink, recent, in_place):
    # below n', above it, both, across it, everything, nothing
    lens = [100, 100, 100, 100, 64, 90, 200, 37]
    gone = [[1], [5], [0, 6], [2, 3], [0, 1, 2, 3], [], [12], [0, 2]]
    run_case(lens, [40, 40, 40, 40, 30, 50, 100, 36], 2, 16, gone, sink, recent, in_place)
    run_case(lens, [99, 99, 97, 64, 1, 0, 199, 20], 3, 16, gone, sink, recent, in_place, seed=2)
    run_case(lens, [50, 7, 93, 20, 63, 100, 100, -3], 1, 7, gone, sink, recent, in_place, seed=3)


@pytest.mark.parametrize("n", [257, 2000, 2049, 8193])
@pytest.mark.parametrize("units", [1, 260])
@pytest.mark.parametrize("sink,recent", [(0, 0), (17, 90)])
def test_blocks_without_a_page_where_the_launches_change(n, units, sink, recent):
    lens = [n - i % 3 for i in range(units)]
    last = (n - 1) // 16
    gone = [[], [0], [last], [1, last - 1], [3, 4, 5, last // 2], list(range(last // 2))] if units > 1 else [[0, 2, last // 2, last - 1]]
    gone = [gone[i % len(gone)] for i in range(units)]
    for budget in (n - 3, n - 40, n // 2, n // 8):
        run_case(lens, [budget] * units, 1, 16, gone, sink, recent, False, seed=n)


@pytest.mark.parametrize("in_place", [False, True])
def test_blocks_without_a_page_in_slices(in_place):
    lens = [17000, 33001, 0, 300, 16385, 20000, 20000, 18000]
    gone = [[0, 100], [515], [], [2], [7, 200, 256], [0, 1, 2, 3], list(range(313)), [250]]
    budgets = [4000, 33000, 7, 100, 16384, 1, 10000, 0]
    for sink, recent in ((0, 0), (4, 100)):
        run_case(lens, budgets, 2, 64, gone, sink, recent, in_place)
        run_case(lens, [n // 2 for n in lens], 1, 64, gone, sink, recent, in_place, seed=2, weight_of=lambda r, n: r.integers(0, 4, n))
    # more protected rows than places with a page, equal keys
    run_case([20000, 18000], [900, 5000], 1, 16, [list(range(0, 40)), [0, 900]], 2000, 3000, in_place, seed=3)
    run_case([20000, 17001], [7000, 50], 1, 8, [list(range(0, 875)), [1]], 0, 0, in_place, seed=4, weight_of=lambda r, n: np.zeros(n),
             pos_of=lambda r, n: r.integers(0, 9, n))
