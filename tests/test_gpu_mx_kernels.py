"""Every kernel of the attention over quantised pages against the definition in 64 bits: by the call's type, row length, format, how many neighbouring rows a page has (16, 4 or 1) and the
query heads of a tile, each with and without weights and as a step, of units taken whole by four waves or one and of runs dealt to workgroups."""
import numpy as np
import pytest

from mx_harness import MxBatch, attend, check, check_written, new_rows

pytestmark = pytest.mark.gpu

#        query heads per key head, page: groups of 16 rows with tiles of up to 4, 8 and 16 heads; of four rows; single rows
TILES = [(3, 16), (4, 48), (5, 32), (8, 16), (9, 16), (18, 64), (2, 24), (8, 4), (1, 7), (12, 20)]
KERNELS = [(G, page, d, dtype, fmt) for G, page in TILES for d in (64, 128) for dtype in ("bf16", "f32") for fmt in ("mxfp4", "mxfp8")]
LAYOUTS = ["heads", "rows", "both", "wide"]


def batch(lens, n_kv, kernel, seed):
    G, page, d, dtype, fmt = kernel
    return MxBatch(lens, n_kv * G, n_kv, d, dtype, fmt, page, seed=seed, layout=LAYOUTS[(G + page + d // 64 + len(dtype)) % 4])


def both_ways(make, max_len=0, kinds=((False, False), (True, False), (False, True), (True, True))):
    """kinds: (with weights, as a step)."""
    for weights, is_step in kinds:
        bt = make()
        step = new_rows(bt, len(bt.lens), seed=4, scale=2.0) if is_step else None
        check(bt, attend(bt, weights=weights, step=step, max_len=max_len), step=step, max_len=max_len)
        if is_step:
            check_written(bt, step)


@pytest.mark.parametrize("kernel", KERNELS, ids=lambda k: "-".join(str(x) for x in k))
def test_units_taken_whole(kernel):
    both_ways(lambda: batch([0, 1, 17, 31, 32, 33, 64, 65, 127, 129, 256, 290], 2, kernel, 1))


@pytest.mark.parametrize("kernel", KERNELS, ids=lambda k: "-".join(str(x) for x in k))
def test_runs_dealt_to_workgroups(kernel):
    both_ways(lambda: batch([1300, 3, 0, 2049], 1, kernel, 2))


@pytest.mark.parametrize("kernel", [k for k in KERNELS if k[:2] in ((3, 16), (8, 16), (9, 16), (2, 24), (1, 7))], ids=lambda k: "-".join(str(x) for x in k))
def test_short_units_of_a_wave_each(kernel):
    both_ways(lambda: batch([int(n) for n in np.random.default_rng(3).integers(0, 129, 128)], 8, kernel, 3), max_len=128, kinds=((False, False), (True, True)))
