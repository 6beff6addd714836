"""CPU: the binding's calls on the paged cache and the logits take tensors as they lie in memory, or refuse them.  The library is replaced by a recorder."""
import pytest
import torch

import paper_2510_18716_amd as ssd
from paper_2510_18716_amd import binding

B, H, HK, D, PAGE, PAGES, BLOCKS = 5, 6, 3, 64, 8, 11, 4


class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


@pytest.fixture
def calls(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(binding, "lib", r)
    return r.calls


def _cfg(**kw):
    return ssd.make_paged_config(B, H, HK, D, "f32", PAGE, PAGES, BLOCKS, **kw)


def _pools(layout):
    """A pool [PAGES, HK, PAGE, D] and the strides it has."""
    if layout == "heads":
        t = torch.zeros(PAGES, HK, PAGE, D)
    elif layout == "rows":
        t = torch.zeros(PAGES, PAGE, HK, D).transpose(1, 2)
    elif layout == "both":
        t = torch.zeros(PAGES, 2, HK, PAGE, D)[:, 1]
    else:
        t = torch.zeros(PAGES, HK, PAGE, D + 64)[..., 64:]
    return t, dict(zip(("page_stride", "head_stride", "row_stride"), t.stride()))


def _all_calls(cfg, k, v, q=None, kn=None, vn=None):
    t, n = torch.zeros(B, BLOCKS, dtype=torch.int32), torch.zeros(B, dtype=torch.int32)
    pos, w = torch.zeros(PAGES, HK, PAGE, dtype=torch.int32), torch.zeros(PAGES, HK, PAGE)
    q = torch.zeros(B, H, D) if q is None else q
    kn = torch.zeros(B, HK, D) if kn is None else kn
    vn = torch.zeros(B, HK, D) if vn is None else vn
    out, ws = torch.zeros(B, H, D), torch.zeros(64)
    return [lambda: ssd.ssd_paged_append(cfg, k, v, t, n, kn, vn, pos=pos, weight=w, stream=1),
            lambda: ssd.ssd_paged_decode_attn(cfg, q, k, v, t, n, out, workspace=ws, stream=1),
            lambda: ssd.ssd_paged_decode_step(cfg, q, kn, vn, k, v, t, n, out, workspace=ws, stream=1),
            lambda: ssd.ssd_paged_evict(cfg, k, v, t, n, n, pos, pos, w, w, workspace=ws, stream=1)]


@pytest.mark.parametrize("layout", ["heads", "rows", "both", "wide"])
def test_pools_as_the_config_says(calls, layout):
    k, strides = _pools(layout)
    v, _ = _pools(layout)
    for call, at in zip(_all_calls(_cfg(**strides), k, v), ((1, 2), (2, 3), (4, 5), (1, 2))):
        call()
        assert [calls[-1][1][i] for i in at] == [k.data_ptr(), v.data_ptr()]
    # the same memory, without its shape
    if layout in ("heads", "rows"):
        for shape in ((-1,), (PAGES, -1), (PAGES * PAGE * HK, D)):
            raw = (k if layout == "heads" else k.transpose(1, 2)).reshape(shape)
            for call in _all_calls(_cfg(**strides), raw, raw):
                call()
    if layout == "rows":                                            # ... and in the order it has there
        for call in _all_calls(_cfg(**strides), k.transpose(1, 2), v):
            call()
    if layout == "both":
        for call in _all_calls(_cfg(**strides), k.reshape(PAGES, 1, HK, PAGE, D)[:, 0], k.flatten(1)):
            call()


def test_pools_in_another_order_than_the_config_says(calls):
    pools = {x: _pools(x)[0] for x in ("heads", "rows", "both", "wide")}
    for said in pools:
        cfg = _cfg(**_pools(said)[1])
        for k in pools:
            for v in pools:
                if k == v == said:
                    continue
                for call in _all_calls(cfg, pools[k], pools[v]):
                    with pytest.raises(ValueError, match="_pages"):
                        call()
    for bad in (torch.zeros(PAGES, PAGE, HK, D), torch.zeros(PAGES * HK * PAGE * D - 1), torch.zeros(HK, PAGES, PAGE, D).transpose(0, 1), torch.zeros(D, PAGES, HK, PAGE).permute(1, 2, 3, 0)):
        for call in _all_calls(_cfg(), bad, pools["heads"]) + _all_calls(_cfg(), pools["heads"], bad):
            with pytest.raises(ValueError, match="_pages"):
                call()
    assert not calls


def test_a_config_that_is_changed_is_read_again(calls):
    cfg = _cfg()
    k, strides = _pools("rows")
    with pytest.raises(ValueError):
        _all_calls(cfg, k, k)[1]()
    for name, value in strides.items():
        setattr(cfg, name, value)
    _all_calls(cfg, k, k)[1]()
    cfg.row_stride += 64
    with pytest.raises(ValueError):
        _all_calls(cfg, k, k)[1]()


def test_queries_and_new_rows_as_the_config_says(calls):
    k = _pools("heads")[0]
    wide = torch.zeros(B, (H + 2 * HK) * D)
    q, kn, vn = wide[:, :H * D], wide[:, H * D:(H + HK) * D], wide[:, (H + HK) * D:]
    cfg = _cfg(q_stride=wide.stride(0), new_stride=wide.stride(0))
    views = [(q, kn, vn), tuple(x.unflatten(1, (-1, D)) for x in (q, kn, vn)), (wide, wide, wide), (q[:, None], kn[:, None], vn[:, None])]
    for a, b, c in views:
        for call in _all_calls(cfg, k, k, a, b, c):
            call()
        step = calls[-2]
        assert step[0] == "ssd_paged_decode_step" and step[1][1:4] == (a.data_ptr(), b.data_ptr(), c.data_ptr())
    dense = (torch.zeros(B, H, D), torch.zeros(B, HK, D), torch.zeros(B, HK, D))
    for x in (dense, tuple(t.flatten(1) for t in dense), tuple(t.flatten() for t in dense), tuple(t.flatten(0, 1) for t in dense)):
        for call in _all_calls(_cfg(), k, k, *x)[0 if len(x[1]) == B else 1:]:          # append counts its rows by the first dimension
            call()
    # more rows than are used, and one sequence of any stride
    for call in _all_calls(_cfg(), k, k, torch.zeros(B + 3, H, D), *dense[1:])[1:3]:
        call()
    one = ssd.make_paged_config(1, H, HK, D, "f32", PAGE, PAGES, BLOCKS)
    ssd.ssd_paged_decode_attn(one, wide[2:3, :H * D], k, k, torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(1, H, D), stream=1)
    ssd.ssd_paged_append(_cfg(), k, k, torch.zeros(B, 4, dtype=torch.int32), torch.zeros(B, dtype=torch.int32), torch.zeros(0, HK, D), torch.zeros(0, HK, D),
                         new_start=torch.zeros(B + 1, dtype=torch.int32), stream=1)


def test_queries_and_new_rows_in_another_place_than_the_config_says(calls):
    k = _pools("heads")[0]
    wide = torch.zeros(B, (H + 2 * HK) * D)
    q, kn, vn = wide[:, :H * D], wide[:, H * D:(H + HK) * D], wide[:, (H + HK) * D:]
    dense = (torch.zeros(B, H, D), torch.zeros(B, HK, D), torch.zeros(B, HK, D))
    apart = wide.stride(0)
    for cfg, qs, news in ((_cfg(), (q, q.unflatten(1, (H, D)), torch.zeros(H, B, D).transpose(0, 1), torch.zeros(B, D, H).transpose(1, 2)),
                           (kn, torch.zeros(HK, B, D).transpose(0, 1), torch.zeros(B, HK, 2 * D)[..., :D])),
                          (_cfg(q_stride=apart, new_stride=apart), (dense[0], dense[0].flatten(1), torch.zeros(4 * B, H, D), wide[:, :H * D - 64]),
                           (dense[1], dense[1].flatten(1), torch.zeros(B, apart + 64)))):
        good_q, good = (q, kn) if cfg.q_stride else dense[:2]
        for bad in qs:
            for call in _all_calls(cfg, k, k, bad, good, good)[1:3]:
                with pytest.raises(ValueError, match="q of shape"):
                    call()
        for bad in news:
            for new, name in (((bad, good), "k_new"), ((good, bad), "v_new")):
                for call in _all_calls(cfg, k, k, good_q, *new)[0:3:2]:
                    with pytest.raises(ValueError, match=name + " of shape"):
                        call()
    assert not calls


def _logits(x, n, V, out, **kw):
    ssd.ssd_logits_process(x, n, V, "f32", out, stream=1, **kw)


def test_logits_are_read_where_they_lie(calls):
    n, V, Vp = 6, 100, 128

    def strides():
        args = calls[-1][1]
        return args[4] or V, args[9] or V
    padded, out = torch.zeros(n, Vp), torch.zeros(n, V)
    _logits(padded[:, :V], n, V, torch.zeros(n, Vp)[:, :V])
    assert strides() == (Vp, Vp)
    _logits(padded, n, V, out)                                       # the whole of it
    assert strides() == (Vp, V)
    _logits(torch.zeros(n, 7, V)[:, -1], n, V, out)
    assert strides() == (7 * V, V)
    _logits(torch.zeros(n, 7, Vp)[:, -1, :V], n, V, out, logits_stride=7 * Vp)
    assert strides() == (7 * Vp, V)
    for x in (torch.zeros(n, V), torch.zeros(n * V), torch.zeros(2, 3, V), torch.zeros(3, 2 * V), torch.zeros(n + 9, V), torch.zeros(1, n * V + 5)):
        _logits(x, n, V, out)
        assert strides() == (V, V)
    # guided: two rows for each
    _logits(torch.zeros(n, 2 * V), n, V, out, gamma=2.0)
    assert strides() == (V, V)
    _logits(torch.zeros(n, 2, Vp)[..., :V], n, V, out, gamma=2.0)
    assert strides() == (Vp, V)
    _logits(torch.zeros(2 * n, Vp), n, V, out, gamma=2.0, logits_stride=Vp)
    assert strides() == (Vp, V)
    _logits(torch.zeros(n * Vp), n, V, out, logits_stride=Vp)
    assert strides() == (Vp, V)
    for v in (1, 3):
        x = torch.zeros(n, 5)[:, :v]
        ssd.ssd_logits_process(x, n, v, "f32", torch.zeros(n, v), stream=1)
        assert calls[-1][1][4] == 5
    _logits(torch.zeros(1, Vp)[:, :V], 1, V, torch.zeros(1, V))
    assert strides()[0] >= V
    ssd.ssd_logits_process(1 << 20, n, V, "f32", 1 << 30, logits_stride=Vp, stream=1)
    assert strides() == (Vp, V)


def test_logits_that_do_not_lie_as_said_are_refused(calls):
    n, V, Vp = 6, 100, 128
    out = torch.zeros(n, V)
    for x, kw in ((torch.zeros(n, Vp)[:, :V], dict(logits_stride=V)), (torch.zeros(n, Vp), dict(logits_stride=V)), (torch.zeros(V, n).t(), {}), (torch.zeros(n - 1, V), {}),
                  (torch.zeros(n, V - 1), {}), (torch.zeros(n, V), dict(logits_stride=Vp)), (torch.zeros(n, V), dict(gamma=1.0)), (torch.zeros(3, 2, Vp)[:, :, :V][:, ::2], {}),
                  (torch.zeros(2, 3, 2, V)[:, :, 0], dict(logits_stride=V)), (torch.zeros(2, 4, V)[:, :3], {}), (torch.zeros(n, 2 * V)[:, ::2], {})):
        with pytest.raises(ValueError, match="logits of shape"):
            _logits(x, n, V, out, **kw)
    for x, kw in ((torch.zeros(n, Vp), dict(out_stride=V)), (torch.zeros(V, n).t(), {}), (torch.zeros(n - 1, V), {})):
        with pytest.raises(ValueError, match="out of shape"):
            _logits(out, n, V, x, **kw)
    assert not calls


def test_bias_and_mask_have_a_row_for_each_or_are_shared(calls):
    n, V = 6, 100
    x, out, words = torch.zeros(n, V), torch.zeros(n, V), -(-V // 32)

    def strides():
        p = calls[-1][1][7]._obj
        return p.bias_stride, p.mask_stride
    for bias, mask, kw, want in ((torch.zeros(n, V), torch.zeros(n, words, dtype=torch.int32), {}, (V, words)),
                                 (torch.zeros(n, V // 4, 4), torch.zeros(2, n // 2, words, dtype=torch.int32), {}, (V, words)),
                                 (torch.zeros(n * V), torch.zeros(n + 2, words, dtype=torch.int32), {}, (V, words)),
                                 (torch.zeros(V), torch.zeros(1, words, dtype=torch.int32), dict(bias_shared=True, mask_shared=True), (0, 0)),
                                 (torch.zeros(n, V), torch.zeros(words, dtype=torch.int32), dict(bias_shared=True, mask_shared=True), (0, 0)),
                                 (torch.zeros(n, V + 28), torch.zeros(n, words + 4, dtype=torch.int32), {}, (V + 28, words + 4))):       # a padded vocabulary
        _logits(x, n, V, out, bias=bias, mask=mask, **kw)
        assert strides() == want
    made = len(calls)
    for bias in (torch.zeros(V), torch.zeros(1, V), torch.zeros(n - 1, V), torch.zeros(n, V - 1)):
        with pytest.raises(ValueError, match="bias of shape"):
            _logits(x, n, V, out, bias=bias)
    with pytest.raises(ValueError, match="bias of shape"):
        _logits(x, n, V, out, bias=torch.zeros(V - 1), bias_shared=True)
    for mask in (torch.zeros(words, dtype=torch.int32), torch.zeros(n, words - 1, dtype=torch.int32), torch.zeros(n - 1, words, dtype=torch.int32)):
        with pytest.raises(ValueError, match="mask of shape"):
            _logits(x, n, V, out, mask=mask)
    assert len(calls) == made
