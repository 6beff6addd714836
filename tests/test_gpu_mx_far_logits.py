"""Attention over quantised pages where logits are large, up to both ends of fp32's range: rows of equal logits count alike, and rows that exist are above those that do not."""
import numpy as np
import pytest

from mx_harness import MxBatch, attend
from oracle import mx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("G,page,d", [(1, 16, 128), (8, 24, 64), (12, 16, 64), (2, 5, 128), (6, 32, 64)])
@pytest.mark.parametrize("fmt,dtype", [("mxfp4", "f32"), ("mxfp8", "f32"), ("mxfp4", "bf16"), ("mxfp8", "bf16")])
@pytest.mark.parametrize("size", [2.0 ** 12, 2.0 ** 33, 2.0 ** 66, 1.25 * 2.0 ** 120])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_the_largest_logits_take_everything(G, page, d, fmt, dtype, size, sign):
    """Keys are 192 or 128 in one element and q a number of three bits in the same one: logits are exact, and the smaller ones have no weight beside the larger ones.  So the output is the mean
    of V over the largest ones' rows (an fp32 sum of at most n terms and a quotient), the lse their logit (its product with the scale, rounded) and log n.  The lowest logits, -3.2e38
    before the scale, are above the -2e38 below which a row would count as none."""
    lens = [1, 5, 33, 40, 700]
    bt = MxBatch(lens, G, 1, d, dtype, fmt, page, seed=2)
    largest = []
    for b, n in enumerate(lens):
        k = np.zeros((n, 1, d))
        k[..., 0] = np.where(np.arange(n) % 3 == 1, 128.0, 192.0)[:, None] if b != 3 else 192.0
        code, scale = mx.encode(k, fmt)
        j = np.arange(n)
        bt.codes[0][bt.table[b][j // page], :, j % page], bt.scales[0][bt.table[b][j // page], :, j % page] = mx.pack(code, fmt), scale
        z = sign * k[:, 0, 0]
        largest.append((z == z.max(), size * z.max()))
    bt.q.zero_()
    bt.q[:, :, 0] = sign * size
    bt.to_device()
    for weights in (False, True):
        out, lse, w = attend(bt, weights=weights)
        out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        for b, n in enumerate(lens):
            rows, z = largest[b]
            V = bt.rows(1, b)[0][rows, 0]
            tol = (n + 4) * 2.0 ** -24 * np.abs(V).mean(0) + (2.0 ** -8 * np.abs(V.mean(0)) if dtype == "bf16" else 0)
            assert np.all(np.abs(out[b] - V.mean(0)) <= tol), (weights, b)
            want = z * d ** -0.5 + np.log(rows.sum())
            assert np.all(np.abs(lse[b] - want) <= 2.0 ** -21 * abs(want)), (weights, b)
            if weights:                                             # a logit and the lse are rounded at their own size, so no more than this can be asked
                j = np.arange(n)
                at = (bt.table[b][j // page], 0, j % page)
                add = w.cpu().numpy()[at] - bt.weight[at]
                assert np.all((add >= -1e-5) & (add <= G * (1 + 1e-5))) and np.all(np.abs(add[~rows]) <= 1e-5), (weights, b)
