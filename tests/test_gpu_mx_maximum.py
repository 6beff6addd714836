"""The running maximum of the attention over quantised pages is that of whole logits: what the matrix cores have added up when it is taken."""
import numpy as np
import pytest
import torch

import paper_2510_18716_amd as ssd
from mx_harness import MxBatch, attend, check, new_rows
from paged_harness import TORCH

pytestmark = pytest.mark.gpu

#        query heads per key head, page: groups of 16 rows with tiles of 4, 8 and 16 heads, of four rows, single rows
TILES = [(1, 16), (4, 32), (8, 16), (16, 16), (3, 24), (8, 4), (1, 7), (16, 1)]
KERNELS = [(G, page, d, dtype, fmt) for G, page in TILES for d in (64, 128) for dtype in ("bf16", "f32") for fmt in ("mxfp4", "mxfp8")]


@pytest.mark.parametrize("kernel", KERNELS, ids=lambda k: "-".join(str(x) for x in k))
def test_logits_whose_parts_cancel(kernel):
    """The last eighth of every 32 (16) elements of a key undoes the first: what is summed before it is off by hundreds, and a maximum found from that would send exp2 beyond fp32's
    range.  Tolerances: mx_harness.check's, which grow with the sizes that are summed."""
    G, page, d, dtype, fmt = kernel
    bt = MxBatch([300, 65, 700, 31], 2 * G, 2, d, dtype, fmt, page, seed=5, spread=False)
    lane = d // 4                                                   # elements that are summed by one lane, eight a step
    first = np.concatenate([np.arange(8) + g * lane for g in range(4)])
    last = first + lane - 8
    flip = 8 if fmt == "mxfp4" else 128
    codes = bt.codes[0]
    held = np.isin(np.arange(bt.n_pages), bt.table[bt.table >= 0])
    if fmt == "mxfp4":
        c = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (d,))
    else:
        c = codes.copy()
    c[..., last] = c[..., first] ^ flip
    codes[held] = ((c[..., 0::2] | c[..., 1::2] << 4) if fmt == "mxfp4" else c)[held]
    there = bt.scales[0] != 255
    bt.scales[0][there] = np.minimum(bt.scales[0][there].astype(int) + 3, 254)             # eight times larger keys
    q = torch.randn(bt.q.shape, generator=torch.Generator().manual_seed(6)) * 0.125
    q[..., first] = 64.0 * torch.sign(torch.randn(q[..., first].shape, generator=torch.Generator().manual_seed(7)))
    q[..., last] = q[..., first] + 0.5 * torch.randint(-1, 2, q[..., first].shape, generator=torch.Generator().manual_seed(8))
    bt.q = q.to(TORCH[dtype])
    bt.to_device()
    for weights in (False, True):
        check(bt, attend(bt, weights=weights))
        step = new_rows(bt, 4, seed=9)
        check(bt, attend(bt, weights=weights, step=step), step=step)
        bt.to_device()


@pytest.mark.parametrize("kernel", KERNELS, ids=lambda k: "-".join(str(x) for x in k))
def test_the_same_bits_from_call_to_call(kernel):
    """Units of many tiles to a wave, dealt and taken whole."""
    G, page, d, dtype, fmt = kernel
    bits, n_kv = (4 if fmt == "mxfp4" else 8), 8
    g = torch.Generator(device="cuda").manual_seed(1)
    for lens in ([5870, 2, 3000, 52, 0, 670, 4089, 8, 1200, 6000], [640, 500, 64, 600, 1]):
        B, blocks = len(lens), [-(-n // page) for n in lens]
        n_pages = sum(blocks) + 1
        table = torch.full((B, max(blocks)), -1, dtype=torch.int32)
        order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(2)).to(torch.int32)
        at = 0
        for b, n in enumerate(blocks):
            table[b, :n] = order[at:at + n]
            at += n
        k, v = (torch.randint(0, 256, (n_pages, n_kv, page, d * bits // 8), dtype=torch.uint8, device="cuda", generator=g) for _ in "kv")
        if fmt == "mxfp8":                                          # no NaN codes, none of the largest
            k, v = (x & 0xbf for x in (k, v))
        ks, vs = (torch.randint(125, 129, (n_pages, n_kv, page, d // 32), dtype=torch.uint8, device="cuda", generator=g) for _ in "kv")
        q = torch.randn((B, n_kv * G, d), device="cuda", generator=g).to(TORCH[dtype])
        cfg = ssd.make_paged_config(B, n_kv * G, n_kv, d, dtype, page, n_pages, table.shape[1])
        weight = torch.rand((n_pages, n_kv, page), device="cuda", generator=g)
        ws = torch.zeros(ssd.ssd_paged_mx_workspace_bytes(cfg, fmt, 0, True), dtype=torch.uint8, device="cuda")
        table, seq_len = table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
        for weights in (False, True):
            first = None
            for i in range(6):
                out, lse, wout = torch.zeros_like(q), torch.zeros((B, n_kv * G), device="cuda"), torch.zeros_like(weight)
                ws.fill_(255 * (i % 2))
                ssd.ssd_paged_mx_decode_attn(cfg, fmt, q, k, v, ks, vs, table, seq_len, out, lse=lse, weight_in=weight if weights else None, weight_out=wout if weights else None,
                                             workspace=ws)
                got = (out, lse, wout)
                assert bool(torch.isfinite(out).all())
                first = first or got
                assert all(torch.equal(x, y) for x, y in zip(first, got)), (lens, weights, i)
