"""Inputs and comparisons shared by the tests of a paged cache held in 8 or 4 bits."""
import numpy as np
import torch

import paper_2510_18716_amd as ssd
from oracle import mx
from paged_harness import TORCH, fine_tolerance


class MxBatch:
    """A pool with `lens` rows per sequence.  layout: "heads" [page, head, place, bytes]; "rows" [page, place, head, bytes]; "both" K and V of a page next to
    each other; "wide" rows 64 bytes longer than they are.  Places that no sequence holds, and the bytes between rows, are 255: NaN whatever is read of them."""

    def __init__(self, lens, H, n_kv, d, dtype, fmt, page, seed, layout="heads", spare=2, more_blocks=1, qs=1.0, device="cuda", spread=True):
        rng = np.random.default_rng(seed)
        self.lens, self.H, self.n_kv, self.d, self.dtype, self.fmt, self.page, self.device = list(lens), H, n_kv, d, dtype, fmt, page, device
        self.bits, self.layout = mx.BITS[fmt], layout
        B, blocks = len(self.lens), [-(-n // page) for n in self.lens]
        self.max_blocks, self.n_pages = max(blocks + [1]) + more_blocks, sum(blocks) + spare
        order = rng.permutation(self.n_pages)
        self.table = np.full((B, self.max_blocks), -1, np.int32)
        at = 0
        for b, n in enumerate(blocks):
            self.table[b, :n] = order[at:at + n]
            at += n
        shape = (self.n_pages, n_kv, page)
        self.codes = [np.full(shape + (d * self.bits // 8,), 255, np.uint8) for _ in "kv"]
        self.scales = [np.full(shape + (d // 32,), 255, np.uint8) for _ in "kv"]
        self.pos = np.full(shape, -7, np.int32)
        self.weight = np.full(shape, np.nan, np.float32)
        for b, n in enumerate(self.lens):
            j = np.arange(n)
            pages, places = self.table[b][j // page], j % page
            for i in range(2):
                x = rng.standard_normal((n, n_kv, d))
                if spread:                                          # blocks of other sizes, a few large elements
                    x *= 2.0 ** rng.integers(-2, 2, (n, n_kv, d // 32)).repeat(32, -1)
                    x[..., 3] *= 4.0
                code, scale = mx.encode(x, fmt)
                self.codes[i][pages, :, places], self.scales[i][pages, :, places] = mx.pack(code, fmt), scale
            self.pos[pages, :, places] = j[:, None]
            self.weight[pages, :, places] = rng.random((n, n_kv)) * 4
        self.q = torch.from_numpy(rng.standard_normal((B, H, d)) * qs).to(TORCH[dtype])
        self.to_device()

    def _lay(self, x):
        x = torch.from_numpy(x)
        if self.layout == "rows":
            return x.transpose(1, 2).contiguous().to(self.device).transpose(1, 2)
        if self.layout == "wide":
            wide = torch.full(tuple(x.shape[:3]) + (x.shape[3] + 64,), 255, dtype=torch.uint8, device=self.device)
            wide[..., 64:] = x.to(self.device)
            return wide[..., 64:]
        return x.to(self.device)

    def to_device(self):
        if self.layout == "both":
            both = torch.stack([torch.from_numpy(x) for x in self.codes], 1).to(self.device)
            self.kd, self.vd = both[:, 0], both[:, 1]
        else:
            self.kd, self.vd = (self._lay(x) for x in self.codes)
        self.ksd, self.vsd = (torch.from_numpy(x).to(self.device) for x in self.scales)
        self.qd, self.tabled = self.q.to(self.device), torch.from_numpy(self.table).to(self.device)
        self.lend = torch.tensor(self.lens, dtype=torch.int32, device=self.device)
        self.posd, self.weightd = torch.from_numpy(self.pos).to(self.device), torch.from_numpy(self.weight).to(self.device)
        per, s = 8 // self.bits, self.kd.stride()
        self.cfg = ssd.make_paged_config(len(self.lens), self.H, self.n_kv, self.d, self.dtype, self.page, self.n_pages, self.max_blocks,
                                         page_stride=s[0] * per, head_stride=s[1] * per, row_stride=s[2] * per)

    @property
    def pools(self):
        return self.kd, self.vd, self.ksd, self.vsd

    def rows(self, which, b, n=None, codes=None, scales=None):
        """(values [n, kv heads, d] of sequence b's first n rows, which of them have a page)."""
        n = self.lens[b] if n is None else n
        codes, scales = self.codes[which] if codes is None else codes, self.scales[which] if scales is None else scales
        j = np.arange(n)
        pages = self.table[b][j // self.page]
        there = (pages >= 0) & (pages < self.n_pages)
        pages = np.where(there, pages, 0)
        return mx.decode(codes[pages, :, j % self.page], scales[pages, :, j % self.page], self.fmt), there

    def scratch(self, n_bytes):
        return torch.full((n_bytes // 4,), float("nan"), device=self.device) if n_bytes else None


def new_rows(bt, n, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn((n, bt.n_kv, bt.d), generator=g) * scale).to(TORCH[bt.dtype]) for _ in "kv"]


def attend(bt, weights=True, max_len=0, lse=True, step=None, stream=None, workspace=None):
    """One attention, or with step = (k_new, v_new) on the host one step; returns (out, lse, weight_out) as device tensors."""
    out = torch.full((len(bt.lens), bt.H, bt.d), 7.0, dtype=TORCH[bt.dtype], device="cuda")
    lse_t = torch.full((len(bt.lens), bt.H), 7.0, device="cuda") if lse else None
    wout = torch.full_like(bt.weightd, -3.0) if weights else None
    ws = bt.scratch(ssd.ssd_paged_mx_workspace_bytes(bt.cfg, bt.fmt, max_len, weights)) if workspace is None else workspace
    more = dict(lse=lse_t, weight_in=bt.weightd if weights else None, weight_out=wout, max_len=max_len, workspace=ws, stream=stream)
    if step is None:
        ssd.ssd_paged_mx_decode_attn(bt.cfg, bt.fmt, bt.qd, *bt.pools, bt.tabled, bt.lend, out, **more)
    else:
        ssd.ssd_paged_mx_decode_step(bt.cfg, bt.fmt, bt.qd, step[0].cuda(), step[1].cuda(), *bt.pools, bt.tabled, bt.lend, out, pos=bt.posd,
                                     seq_pos=bt.lend + 3, **more)
    return out, lse_t, wout


def check(bt, got, max_len=0, step=None, scale=None):
    """Against the definition in 64 bits.  Tolerances: see fine_tolerance for outputs; a logit is d products summed in fp32, each product exact (bf16 times four
    bits; fp32 q in three terms loses nothing), so off by at most 2e-5 where its terms' sizes add up to 40 and more in proportion; lse likewise, 5e-5 + 1e-6 of itself;
    weights 5e-5 of what is added, 2^-23 of the sum."""
    out, lse, wout = got
    o, G = out.float().cpu().numpy(), bt.H // bt.n_kv
    scale = bt.d ** -0.5 if scale is None else scale
    touched = np.zeros(bt.pos.shape, bool)
    w = None if wout is None else wout.cpu().numpy()
    for b, n in enumerate(bt.lens):
        whole, n = n, min(n, max_len) if max_len else n
        (K, there), (V, _) = bt.rows(0, b, n), bt.rows(1, b, n)
        newest = step is not None and n == whole and n > 0
        if newest:
            K[n - 1], V[n - 1] = (mx.held(x[b].double().numpy(), bt.fmt) for x in step)
        pages, places = bt.table[b][np.arange(n) // bt.page], np.arange(n) % bt.page
        for kv in range(bt.n_kv):
            q = bt.q[b, kv * G:(kv + 1) * G].double().numpy()
            k, v = K[there, kv], V[there, kv]
            if not len(k):
                assert np.all(o[b, kv * G:(kv + 1) * G] == 0), (b, kv)
                if lse is not None:
                    assert np.all(np.isneginf(lse[b, kv * G:(kv + 1) * G].cpu().numpy()))
                continue
            z = q @ k.T * scale
            terms = 2e-5 * max(1.0, float((np.abs(q) @ np.abs(k).T).max()) * scale / 40)
            top = z.max(1, keepdims=True)
            e = np.exp(z - top)
            p = e / e.sum(1, keepdims=True)
            ref, size = p @ v, p @ np.abs(v)
            tol = fine_tolerance(bt.dtype, ref, size) + 2 * (terms - 2e-5) * size
            far = np.abs(o[b, kv * G:(kv + 1) * G] - ref)
            assert np.all(far <= tol), (b, n, kv, float(far.max()), float((far - tol).max()))
            if lse is not None:
                l, ref_l = lse[b, kv * G:(kv + 1) * G].cpu().numpy(), (top + np.log(e.sum(1, keepdims=True)))[:, 0]
                assert np.all(np.abs(l - ref_l) <= 5e-5 + (terms - 2e-5) + 1e-6 * np.abs(ref_l)), (b, kv, l, ref_l)
            if w is not None:
                add = p.sum(0)
                before = bt.weight[pages[there], kv, places[there]].astype(np.float64)
                if newest and there[n - 1]:
                    before[-1] = 0
                want, have = before + add, w[pages[there], kv, places[there]]
                assert np.all(np.abs(have - want) <= 5e-5 * add + 2 * (terms - 2e-5) * add + 2.0 ** -23 * np.abs(want) + 1e-30), (b, kv)
                touched[pages[there], kv, places[there]] = True
    if w is not None:
        assert np.all(w[~touched] == -3.0)                          # nothing else was written


def check_written(bt, step):
    """The pool, scales and positions after a step: the new rows' codes, everything else as it was."""
    codes, scales, pos = [x.copy() for x in bt.codes], [x.copy() for x in bt.scales], bt.pos.copy()
    for b, n in enumerate(bt.lens):
        page = bt.table[b, (n - 1) // bt.page] if n else -1
        if not 0 <= page < bt.n_pages:
            continue
        for i in range(2):
            code, scale = mx.encode(step[i][b].double().numpy(), bt.fmt)
            codes[i][page, :, (n - 1) % bt.page], scales[i][page, :, (n - 1) % bt.page] = mx.pack(code, bt.fmt), scale
        pos[page, :, (n - 1) % bt.page] = n + 2
    same_pools(bt, codes, scales)
    assert np.array_equal(bt.posd.cpu().numpy(), pos)


def same_pools(bt, codes, scales):
    for i, (have, have_s) in enumerate(((bt.kd, bt.ksd), (bt.vd, bt.vsd))):
        assert np.array_equal(have_s.cpu().numpy(), scales[i]), "kv"[i]
        assert np.array_equal(have.cpu().numpy(), codes[i]), "kv"[i]
