"""fp32 calls over quantised pages: every bit of q and of the probabilities counts."""
import numpy as np
import pytest

from mx_harness import attend
from test_gpu_mx_rounding import N, P, cancelling

pytestmark = pytest.mark.gpu

SHAPES = [(1, 16), (8, 32), (3, 24), (9, 16), (2, 7)]               # two columns to a head, groups of four rows, one column, single rows
LENS = [N + 2, 40, 700, 3000]


@pytest.mark.parametrize("G,page", SHAPES)
@pytest.mark.parametrize("fmt,d", [("mxfp4", 128), ("mxfp8", 128), ("mxfp4", 64), ("mxfp8", 64)])
def test_probabilities_have_all_their_bits(G, page, fmt, d):
    """Three terms of bf16 are a number of fp32.  Left are the exponential and the scale (2^-21 of a probability together) and N + 2 sums: 2.5e-6.  Two terms, cut off
    or rounded, are off by 1.1e-5 and more."""
    bt = cancelling(LENS, G, d, "f32", fmt, page)
    p = np.exp(-np.float64(np.float32(-np.log(P))))
    l = N * p + 2
    ref, size = (N * p - 8 - 2.0 ** -4) / l, (N * p + 8 + 2.0 ** -4) / l
    tol = (2.0 ** -21 + (N + 2) * 2.0 ** -24) * size + 2.0 ** -23 * abs(ref)
    for weights in (False, True):
        out, lse, w = attend(bt, weights=weights)
        out = out.double().cpu().numpy()
        assert np.all(np.abs(out - ref) <= tol), (weights, float(np.abs(out - ref).max()), tol)
        assert np.all(np.abs(lse.double().cpu().numpy() - np.log(l)) <= 2.0 ** -21 + (N + 2) * 2.0 ** -24)


@pytest.mark.parametrize("G,page", SHAPES)
@pytest.mark.parametrize("fmt,d", [("mxfp4", 128), ("mxfp8", 128), ("mxfp4", 64), ("mxfp8", 64)])
def test_queries_have_all_their_bits(G, page, fmt, d):
    """q with 24 bits against keys that are powers of two, so that the logits are exact: probabilities and lse are off as above, weights (fp32 sums of G probabilities onto what
    was there) by as much of what is added.  A q of two terms is off by 2^-16, and so are the probabilities of logits near 1."""
    bt = cancelling(LENS, G, d, "f32", fmt, page)
    q = np.float64(np.float32(P * 2))                                # 24 bits, the last sixteen of them beyond the first term
    bt.q[:, :, 0] = float(q)
    assert float(bt.q[0, 0, 0]) == q
    scale = np.float32(0.7)
    bt.to_device()
    bt.cfg.softmax_scale = float(scale)
    p = np.exp(-q * np.float64(scale))
    l = N * p + 2
    ref, size = (N * p - 8 - 2.0 ** -4) / l, (N * p + 8 + 2.0 ** -4) / l
    off = 2.0 ** -21 + (N + 2) * 2.0 ** -24
    out, lse, w = attend(bt)
    out, lse, w = out.double().cpu().numpy(), lse.double().cpu().numpy(), w.double().cpu().numpy()
    assert np.all(np.abs(out - ref) <= off * size + 2.0 ** -23 * abs(ref)), float(np.abs(out - ref).max())
    assert np.all(np.abs(lse - np.log(l)) <= off)
    for b, n in enumerate(bt.lens):
        order = np.random.default_rng(b).permutation(n)
        add = np.zeros(n)
        add[order[:N]], add[order[N:N + 2]] = G * p / l, G / l
        j = np.arange(n)
        at = (bt.table[b][j // page], slice(None), j % page)
        want = bt.weight[at].astype(np.float64) + add[:, None]
        assert np.all(np.abs(w[at] - want) <= (2 * off + G * 2.0 ** -24) * add[:, None] + 2.0 ** -23 * want), b
