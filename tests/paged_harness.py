"""Inputs and comparisons shared by the tests of the paged cache: batches of unequal lengths in a pool, on the host and on the GPU."""
import numpy as np
import torch

import paper_2510_18716_amd as ssd
from oracle import paged

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


class Batch:
    """A pool with `lens` rows per sequence.  layout: "heads" [page, head, place, d]; "rows" [page, place, head, d]; "both" K and V of a
    page next to each other; "wide" rows of d elements 64 apart.  Everything past a sequence's end, and every page that no sequence
    holds, is NaN."""

    def __init__(self, lens, H, n_kv, d, dtype, page, seed, layout="heads", spare=2, more_blocks=1, qs=1.0, device="cuda", q_gap=0):
        rng = np.random.default_rng(seed)
        self.lens, self.H, self.n_kv, self.d, self.dtype, self.page = list(lens), H, n_kv, d, dtype, page
        B = len(self.lens)
        blocks = [-(-n // page) for n in self.lens]
        self.max_blocks = max(blocks + [1]) + more_blocks
        self.n_pages = sum(blocks) + spare
        order = rng.permutation(self.n_pages)
        self.table = np.full((B, self.max_blocks), -1, np.int32)
        at = 0
        for b, n in enumerate(blocks):
            self.table[b, :n] = order[at:at + n]
            at += n
        g = torch.Generator().manual_seed(seed)
        dt = TORCH[dtype]
        self.k = torch.full((self.n_pages, n_kv, page, d), float("nan"))
        self.v = self.k.clone()
        for b, n in enumerate(self.lens):
            for j in range(n):
                self.k[self.table[b, j // page], :, j % page] = torch.randn((n_kv, d), generator=g)
                self.v[self.table[b, j // page], :, j % page] = torch.randn((n_kv, d), generator=g)
        self.k, self.v = self.k.to(dt), self.v.to(dt)
        self.q = (torch.randn((B, H, d), generator=g) * qs).to(dt)
        self.pos = torch.full((self.n_pages, n_kv, page), -7, dtype=torch.int32)
        self.weight = torch.full((self.n_pages, n_kv, page), float("nan"))
        for b, n in enumerate(self.lens):
            for j in range(n):
                self.pos[self.table[b, j // page], :, j % page] = j
                self.weight[self.table[b, j // page], :, j % page] = torch.rand(n_kv, generator=g) * 4
        self.device = device
        if layout == "heads":
            self.kd, self.vd = self.k.to(device), self.v.to(device)
        elif layout == "rows":
            self.kd, self.vd = (x.transpose(1, 2).contiguous().to(device).transpose(1, 2) for x in (self.k, self.v))
        elif layout == "both":
            both = torch.stack([self.k, self.v], 1).to(device)
            self.kd, self.vd = both[:, 0], both[:, 1]
        else:
            wide = [torch.full(tuple(self.k.shape[:3]) + (d + 64,), float("nan"), dtype=dt, device=device) for _ in range(2)]
            self.kd, self.vd = wide[0][..., 64:], wide[1][..., 64:]
            self.kd.copy_(self.k.to(device))
            self.vd.copy_(self.v.to(device))
        self.q_stride = 0
        self.qd = self.q.to(device)
        if q_gap:
            big = torch.full((B, H * d + q_gap), float("nan"), dtype=dt, device=device)
            big[:, :H * d] = self.qd.reshape(B, H * d)
            self.qd, self.q_stride = big, H * d + q_gap
        self.tabled = torch.from_numpy(self.table).to(device)
        self.lend = torch.tensor(self.lens, dtype=torch.int32, device=device)
        s = self.kd.stride()
        self.cfg = ssd.make_paged_config(B, H, n_kv, d, dtype, page, self.n_pages, self.max_blocks, page_stride=s[0], head_stride=s[1],
                                         row_stride=s[2], q_stride=self.q_stride)

    def scratch(self, n_bytes):
        """Workspace of exactly that size, full of NaN: nothing in it may be relied on."""
        t = torch.full((max(1, n_bytes // 4),), float("nan"), device=self.device)
        return t if n_bytes else None


def attend(bt, weights=True, max_len=0, lse=True, stream=None, **kw):
    """One ssd_paged_decode_attn on a batch; returns (out, lse, weight_out) as device tensors."""
    out = torch.full((len(bt.lens), bt.H, bt.d), 7.0, dtype=TORCH[bt.dtype], device="cuda")
    lse_t = torch.full((len(bt.lens), bt.H), 7.0, device="cuda") if lse else None
    win = bt.weight.cuda() if weights else None
    wout = torch.full_like(win, -3.0) if weights else None
    ws = bt.scratch(ssd.ssd_paged_workspace_bytes(bt.cfg, max_len, weights))
    ssd.ssd_paged_decode_attn(bt.cfg, bt.qd, bt.kd, bt.vd, bt.tabled, bt.lend, out, lse=lse_t, weight_in=win, weight_out=wout, max_len=max_len,
                              workspace=ws, stream=stream, **kw)
    return out, lse_t, wout


def check_attend(bt, got, weights=True, max_len=0, lens=None, scale=None, table=None, weight_before=None):
    """Against the 64-bit implementation.

    Tolerances.  A logit is d products summed in fp32: off by at most d * 2^-24 * sum |q_i k_i| * scale, and by a random walk's
    sqrt(d) of that in the mean; with |q|, |k| ~ sqrt(d) that is below 2e-5, and so relative is an exponential, a probability, a sum of them (5e-5 with
    the exponential's own 2^-22 and the sums').  Output, fp32: 5e-5 of sum p |v|.  bf16: probabilities may be rounded once to 8 bits (2^-9 of each term,
    and the output once more): 2^-8 of sum p |v|, plus 2^-8 of the result.  Weights: 5e-5 of what is added, 2^-23 of the sum."""
    out, lse, wout = got
    o = out.float().cpu().numpy()
    w = None if wout is None else wout.cpu().numpy()
    kp, vp = bt.k.float().numpy(), bt.v.float().numpy()
    table = bt.table if table is None else table
    scale = 1.0 / np.sqrt(bt.d) if scale is None else scale
    G = bt.H // bt.n_kv
    touched = np.zeros(bt.weight.shape, bool)
    before = (bt.weight if weight_before is None else weight_before).numpy()
    for b, n in enumerate(bt.lens if lens is None else lens):
        n = min(n, max_len) if max_len else n
        ref, ref_lse, p, size = paged.paged_attend(bt.q[b].float().numpy(), kp, vp, table[b], n, scale)
        tol = 5e-5 * size + 1e-30 if bt.dtype == "f32" else 2.0 ** -8 * (size + np.abs(ref)) + 1e-30
        worst = np.abs(o[b] - ref) - tol
        assert worst.max() <= 0, (b, n, float(np.abs(o[b] - ref).max()), float(worst.max()))
        if lse is not None:
            l = lse[b].cpu().numpy()
            same = (l == ref_lse) | (np.abs(l - np.where(np.isfinite(ref_lse), ref_lse, 0)) <= 5e-5 + 1e-6 * np.abs(ref_lse))
            assert same.all(), (b, n, l, ref_lse)
        if w is not None:
            for j in range(n):
                page, place = paged.slot_place(table[b], j, bt.page)
                if not 0 <= page < bt.n_pages:
                    continue
                add = p[:, j].reshape(bt.n_kv, G).sum(1)
                want = before[page, :, place].astype(np.float64) + add
                assert np.all(np.abs(w[page, :, place] - want) <= 5e-5 * add + 2.0 ** -23 * np.abs(want) + 1e-30), (b, j)
                touched[page, :, place] = True
    if w is not None:
        assert np.all(w[~touched] == -3.0)            # nothing else was written


def outputs_of(bt, b, n=None, table=None):
    """(out, sum p |v|) of sequence b in 64 bits."""
    table = bt.table if table is None else table
    out, _, _, size = paged.paged_attend(bt.q[b].float().numpy(), bt.k.float().numpy(), bt.v.float().numpy(), table[b], bt.lens[b] if n is None else n,
                                         bt.d ** -0.5)
    return out, size


def fine_tolerance(dtype, ref, size):
    """What an output may be off by if the probabilities keep 16 bits.  Logits are off by 2e-5 (check_attend) and so relative are the probabilities; their two
    bf16 terms leave out at most 2^-15 and nothing of the largest's; exponentials, sums and the division are fp32's: 5.1e-5 of sum p |v| together.  A bf16 output is rounded once more, by at most
    2^-8 of itself.  One row of thousands, or the second term, is more than that."""
    return 5.1e-5 * size + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0.0) + 1e-30


def check_outputs(bt, out, lens=None, table=None):
    o = out.float().cpu().numpy()
    for b, n in enumerate(bt.lens if lens is None else lens):
        ref, size = outputs_of(bt, b, n, table)
        worst = np.abs(o[b] - ref) - fine_tolerance(bt.dtype, ref, size)
        assert worst.max() <= 0, (b, n, float(np.abs(o[b] - ref).max()), float(worst.max()))


def cancelling(lens, H, n_kv, d, dtype, seed, device):
    """A batch whose rows come in pairs of nearly the same key and opposite values: what is left of the output is the difference of probabilities that have
    their first eight bits in common."""
    bt = Batch(lens, H, n_kv, d, dtype, 16, seed=seed, device=device)
    g = torch.Generator().manual_seed(seed)
    bt.q.zero_()
    bt.q[:, :, 0] = 1.0
    for b, n in enumerate(bt.lens):
        v = torch.randn((n_kv, d), generator=g)
        for j in range(n):
            at = (bt.table[b, j // 16], slice(None), j % 16)
            bt.k[at] = 0.0
            bt.k[at][:, 0] = torch.randint(-40, 0, (n_kv,), generator=g) * 2.0 ** -6          # exact in bf16
            bt.v[at] = (v * (1 if j % 2 else -1)).to(bt.v.dtype)
    bt.kd, bt.vd, bt.qd = bt.k.to(device), bt.v.to(device), bt.q.to(device)
    return bt


def evict_sources(pos, weight, total, budget, n_sink, recent, there):
    """oracle.paged.evict_moves for long units: the slot that each slot below n' has its row from."""
    n = len(pos)
    stay = min(n, max(0, budget))
    held = np.nonzero(there)[0]
    p, w = pos[held], weight[held]
    safe = (p < n_sink) | (p >= total - recent)
    with np.errstate(invalid="ignore"):
        key = np.where(np.isnan(w), np.inf, -w.astype(np.float64))
    best = held[np.lexsort((held, p, key, np.isnan(w), ~safe))[:int(np.sum(held < stay))]]
    src = np.arange(stay)
    src[~np.isin(src, best) & there[:stay]] = np.sort(best[best >= stay])
    return src
