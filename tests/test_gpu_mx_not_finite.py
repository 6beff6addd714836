"""Elements of V that are no numbers, in pools written elsewhere or of blocks near fp32's largest: which outputs they reach."""
import numpy as np
import pytest

from mx_harness import MxBatch, attend, check
from oracle import mx

pytestmark = pytest.mark.gpu

#         query heads per key head, page; whether the matrix cores have a column for each of a pair's two elements
SHAPES = [(1, 16, False), (4, 64, False), (8, 16, False), (3, 24, False), (9, 16, True), (16, 48, True), (2, 7, True), (5, 1, True)]


@pytest.mark.parametrize("G,page,apart", SHAPES)
@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "f32"), (64, "bf16"), (128, "f32")])
@pytest.mark.parametrize("kind", ["mxfp8 nan", "mxfp8 inf", "mxfp4 inf"])
def test_single_elements_reach_their_pair_at_most(G, page, apart, d, dtype, kind):
    """One NaN code, or one element that reads as an infinity.  Its own column is NaN, or an infinity (NaN too where a term of a probability is zero); the other column of its pair
    (2 c, 2 c + 1) is right or NaN, right where columns are apart; all others, the other key head's and other sequences' are right, and lse and weights everywhere."""
    fmt, what = kind.split()
    lens, column = [70, 40, 900], 37
    bt = MxBatch(lens, 2 * G, 2, d, dtype, fmt, page, seed=3)
    for b, row in ((0, 33), (2, 650)):
        at, place = bt.table[b][row // page], row % page
        codes = bt.codes[1][at, 0, place]
        if fmt == "mxfp8":
            codes[32:64] = 8                                        # 2^-6; with the scale byte 254 2^121
            codes[column] = 0x7f if what == "nan" else 0x7e
        else:
            codes[16:32] = 0x11                                     # 1/2 each
            codes[column // 2] = 0x71                               # the odd element 6
        if what == "inf":
            bt.scales[1][at, 0, place, 1] = 254
    clean = [x.copy() for x in bt.codes], [x.copy() for x in bt.scales]
    bt.to_device()
    out, lse, w = attend(bt)
    o = out.float().cpu().numpy()
    for b in (0, 2):
        assert not np.isfinite(o[b, :G, column]).any(), (b, o[b, :G, column])
        pair = o[b, :G, column - 1]
        assert np.isfinite(pair).all() if apart else (np.isfinite(pair) | np.isnan(pair)).all(), (b, pair)
    # all that is finite against the definition: the same pool with the element gone
    for b, row in ((0, 33), (2, 650)):
        at, place = bt.table[b][row // page], row % page
        if fmt == "mxfp8":
            clean[0][1][at, 0, place, column] = 0
        else:
            clean[0][1][at, 0, place, column // 2] = 0x01
    bt.codes, bt.scales = clean
    skip = np.zeros(o.shape, bool)
    for b in (0, 2):
        skip[b, :G, column] = True
        skip[b, :G, column - 1] = ~np.isfinite(o[b, :G, column - 1])
    reference = MxBatch.__new__(MxBatch)
    reference.__dict__.update(bt.__dict__)
    reference.to_device()
    right = attend(reference)
    o_right = right[0].float().cpu().numpy()
    mixed = np.where(skip, o_right, o)
    check(reference, (right[0].new_tensor(mixed), lse, w))
