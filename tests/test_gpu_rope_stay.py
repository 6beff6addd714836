"""Pairs whose axis does not exist stay to the bit, whatever they hold."""
import numpy as np
import pytest
import torch

import paper_2510_18716_amd as ssd
from oracle import mx

pytestmark = pytest.mark.gpu

WORDS = {torch.float32: (torch.int32, [0x7f800000, -0x800000, 0x7fc00001, 0x7f800001, -0x80000000, 0, 0x3f800000, -0x40800000, 1, 0x7f7fffff]),
         torch.bfloat16: (torch.int16, [0x7f80, -0x80, 0x7fc1, 0x7f81, -0x8000, 0, 0x3f80, -0x4080, 1, 0x7f7f])}     # infinities, NaN, zeros, ones, the least and the largest


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("n,H,d,pairs", [(100, 2, 64, 32), (7, 1, 6, 3), (3, 3, 40, 10), (2, 1, 2, 1), (70, 40, 128, 64)])
def test_pairs_that_stay_hold_what_they_held(n, H, d, pairs, layout, inverse, dtype):
    as_words, values = WORDS[dtype]
    rng = np.random.default_rng(n)
    x = torch.tensor(rng.choice(values, (n, H, d)), dtype=as_words)
    axis = torch.tensor([(2, 0, 255, 1)[i % 4] for i in range(pairs)], dtype=torch.uint8)
    turns = np.array([a < 2 for a in axis.tolist()])
    first, second = (np.arange(pairs), np.arange(pairs) + pairs) if layout == "half" else (2 * np.arange(pairs), 2 * np.arange(pairs) + 1)
    moved = np.concatenate([first[turns], second[turns]]).astype(int)
    plain = torch.randn((n, H, d), generator=torch.Generator().manual_seed(1)).to(dtype)
    x = x.view(dtype)
    x[..., moved] = plain[..., moved]
    pos = torch.randint(-1000, 1000, (2, n), generator=torch.Generator().manual_seed(2)).to(torch.int32)
    inv = torch.tensor([10000.0 ** (-i / pairs) for i in range(pairs)])
    args = (n, H, d, dtype, pos.cuda(), inv.cuda())
    more = dict(axis=axis.cuda(), n_axes=2, layout=ssd.SSD_ROPE_HALF if layout == "half" else ssd.SSD_ROPE_INTERLEAVED, inverse=inverse)
    out = torch.zeros_like(x, device="cuda")
    ssd.ssd_rope_axes(x.cuda(), out, *args, **more)
    same = x.cuda()
    ssd.ssd_rope_axes(same, same, *args, **more)
    stays = np.setdiff1d(np.arange(d), moved)
    for o in (out.cpu(), same.cpu()):
        assert torch.equal(o.view(as_words)[..., stays], x.view(as_words)[..., stays])
        ref = mx.rope(torch.where(torch.isfinite(x), x, torch.zeros_like(x)).double().numpy(), pos.numpy(), inv.numpy(), axis.numpy(), layout, inverse)[..., moved]
        # as in test_gpu_rope.py: 2^-21 of |a| + |b|, at most 12 here, and a bf16's rounding
        assert np.all(np.abs(o.double().numpy()[..., moved] - ref) <= 12 * 2.0 ** -21 + (2.0 ** -8 * np.abs(ref) if dtype == torch.bfloat16 else 0))
