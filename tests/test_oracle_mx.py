"""The block formats' plain implementation against values worked out by hand."""
import numpy as np
import pytest

from oracle import mx


def _row(fmt, values):
    x = np.zeros(32)
    x[:len(values)] = values
    code, scale = mx.encode(x, fmt)
    return code, int(scale[0]), mx.decode(mx.pack(code, fmt), scale, fmt)


def test_levels():
    assert mx.levels("mxfp4").tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    lv = mx.levels("mxfp8")
    assert len(lv) == 127 and lv[1] == 2.0 ** -9 and lv[8] == 2.0 ** -6 and lv[-1] == 448


def test_ties_go_to_the_even_code_and_the_sign_stays():
    code, scale, back = _row("mxfp4", [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5, -0.0, 0.26])
    assert scale == 127 and back[:11].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, -4, 0, 0.5] and code[9] == 8
    code, scale, back = _row("mxfp8", [448, 17, 19, 2.0 ** -10, 3 * 2.0 ** -10, -464])
    assert scale == 127 and back[:6].tolist() == [448, 16, 20, 0, 2.0 ** -8, -448]


def test_scale_is_the_smallest_that_is_off_by_half_a_step_at_most():
    assert _row("mxfp4", [7.0])[1] == 127 and _row("mxfp4", [7.0])[2][0] == 6
    assert _row("mxfp4", [np.nextafter(7, 8)])[1] == 128 and _row("mxfp4", [np.nextafter(7, 8)])[2][0] == 8
    assert _row("mxfp8", [464.0])[1] == 127 and _row("mxfp8", [465.0])[1] == 128
    assert _row("mxfp4", [0.0])[1] == 2 and _row("mxfp8", [0.0])[1] == 10
    assert _row("mxfp4", [1e-39])[1] == 2 and _row("mxfp8", [2.0 ** -112])[1] == 10


@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
def test_blocks_that_hold_no_number(fmt):
    for bad in (np.inf, -np.inf, np.nan):
        x = np.ones(64)
        x[40] = bad
        code, scale = mx.encode(x, fmt)
        assert scale[1] == 255 and not code[32:].any()
        back = mx.decode(mx.pack(code, fmt), scale, fmt)
        assert np.all(back[:32] == 1) and np.isnan(back[32:]).all()


@pytest.mark.parametrize("fmt,steps", [("mxfp4", 4), ("mxfp8", 16)])
def test_no_element_is_off_by_more_than_half_a_step(fmt, steps):
    """Half a step: an eighth (a thirty-second... of the octave) relative, or of the smallest step in the block."""
    x = np.random.default_rng(0).standard_normal((200, 128)) * 2.0 ** np.random.default_rng(1).integers(-20, 20, (200, 4)).repeat(32, -1)
    code, scale = mx.encode(x, fmt)
    unit = np.repeat(2.0 ** (scale.astype(float) - 127), 32, -1)
    least = unit * (0.25 if fmt == "mxfp4" else 2.0 ** -10)
    assert np.all(np.abs(mx.held(x, fmt) - x) <= np.maximum(least, np.abs(x) / steps))


def test_rope_by_hand():
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 5.0]]])
    out = mx.rope(x, [[1], [2]], [np.pi / 2, np.pi / 4], [0, 1], "half")
    assert np.allclose(out, [[[-3, -4, 1, 2, 5]]])
    out = mx.rope(x, [[1], [2]], [np.pi / 2, np.pi / 4], [0, 1], "interleaved")
    assert np.allclose(out, [[[-2, 1, -4, 3, 5]]])
    assert np.allclose(mx.rope(out, [[1], [2]], [np.pi / 2, np.pi / 4], [0, 1], "interleaved", inverse=True), x)
    assert np.array_equal(mx.rope(x, [[7]], [1.0, 1.0], [1, 9], "half"), x)
