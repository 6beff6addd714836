"""What the attention over quantised pages leaves out of a probability: half a step of its last term, not a whole one."""
import numpy as np
import pytest
import torch

import paper_2510_18716_amd as ssd
from mx_harness import MxBatch, attend
from oracle import mx

pytestmark = pytest.mark.gpu

N = 16                                                              # rows whose probability has bits beyond two terms of bf16
P = (1 + 2.0 ** -7) * (1 - 2.0 ** -18) / 2                          # just below the next number of eight bits: what the first term leaves is all ones


def cancelling(lens, G, d, dtype, fmt, page):
    """Rows 0 .. N + 1 of every sequence: N rows of logit -s with V = 1 and two of logit 0 with V = -8 and -1/16, whose sum is nearly nothing; the others have no weight."""
    bt = MxBatch(lens, 2 * G, 2, d, dtype, fmt, page, seed=1)
    for b, n in enumerate(lens):
        k, v = np.zeros((n, 2, d)), np.ones((n, 2, d))
        k[:, :, 0] = -384.0
        order = np.random.default_rng(b).permutation(n)              # the rows that count lie anywhere
        k[order[:N], :, 0] = -1.0
        k[order[N:N + 2], :, 0], v[order[N]], v[order[N + 1]] = 0.0, -8.0, -2.0 ** -4
        j = np.arange(n)
        for i, x in enumerate((k, v)):
            code, scale = mx.encode(x, fmt)
            assert np.array_equal(mx.decode(mx.pack(code, fmt), scale, fmt), x)
            bt.codes[i][bt.table[b][j // page], :, j % page], bt.scales[i][bt.table[b][j // page], :, j % page] = mx.pack(code, fmt), scale
    bt.q.zero_()
    bt.q[:, :, 0] = 1.0
    bt.to_device()
    bt.cfg.softmax_scale = -float(np.log(P))
    return bt


@pytest.mark.parametrize("G,page", [(1, 16), (4, 64), (5, 16), (8, 32), (3, 24), (8, 4), (9, 16), (16, 16), (2, 7)])
@pytest.mark.parametrize("fmt,d", [("mxfp4", 128), ("mxfp8", 128), ("mxfp4", 64), ("mxfp8", 64)])
def test_the_last_term_of_a_probability_is_rounded(G, page, fmt, d):
    """Logits are exact, and the largest probabilities, 1, have one bit.  The N others are off by half a step of their second term, 2^-17, beside the exponential and the scale (2^-21 of them)
    and N + 2 sums of fp32; the output, of the difference, by 2^-8 of next to nothing.  A second term that is cut off leaves out 0.87 of a step."""
    lens = [N + 2, 40, 700, 3000, 33]
    bt = cancelling(lens, G, d, "bf16", fmt, page)
    p = np.exp(-np.float64(np.float32(-np.log(P))))
    l = N * p + 2
    ref, size = (N * p - 8 - 2.0 ** -4) / l, (N * p + 8 + 2.0 ** -4) / l
    tol = N * 2.0 ** -17 / l + (2.0 ** -21 + (N + 2) * 2.0 ** -24) * size + 2.0 ** -8 * abs(ref)
    assert tol < 0.75 * N * (0.875 * 2.0 ** -16) / l
    for weights in (False, True):
        out = attend(bt, weights=weights)[0].double().cpu().numpy()
        assert np.all(np.abs(out - ref) <= tol), (weights, float(np.abs(out - ref).max()), tol)
