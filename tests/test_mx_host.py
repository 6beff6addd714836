"""CPU-only checks of the calls on a paged cache held in 8 or 4 bits and of ssd_rope_axes: what they refuse, before anything is launched, what the binding refuses, and
the sizes of workspaces."""
import ctypes as C

import pytest
import torch

import paper_2510_18716_amd as ssd
from mx_harness import MxBatch
from paper_2510_18716_amd.binding import _mx_pools
from test_paged_host import BAD_CONFIG, _cfg

FAKE = 1 << 24
BAD = ssd.SSD_ERR_INVALID_ARG


def _ref(cfg):
    return None if cfg is None else C.byref(cfg)


def _append(cfg, **kw):
    a = dict(f=4, k=FAKE, v=FAKE, ks=FAKE, vs=FAKE, pos=FAKE, weight=FAKE, table=FAKE, len=FAKE, total=FAKE, kn=FAKE, vn=FAKE, start=FAKE, n=5, wn=FAKE)
    a.update(kw)
    return ssd.lib.ssd_paged_mx_append(_ref(cfg), a["f"], a["k"], a["v"], a["ks"], a["vs"], a["pos"], a["weight"], a["table"], a["len"], a["total"], a["kn"], a["vn"], a["start"],
                                       a["n"], a["wn"], None)


def _read(cfg, **kw):
    a = dict(f=4, k=FAKE, v=FAKE, ks=FAKE, vs=FAKE, table=FAKE, len=FAKE, start=FAKE, n=5, first=FAKE, kn=FAKE, vn=FAKE)
    a.update(kw)
    return ssd.lib.ssd_paged_mx_read(_ref(cfg), a["f"], a["k"], a["v"], a["ks"], a["vs"], a["table"], a["len"], a["start"], a["n"], a["first"], a["kn"], a["vn"], None)


def _attn(cfg, **kw):
    a = dict(f=4, q=FAKE, k=FAKE, v=FAKE, ks=FAKE, vs=FAKE, wi=FAKE, wo=FAKE, table=FAKE, len=FAKE, out=FAKE, lse=FAKE, most=0, ws=FAKE, size=1 << 40)
    a.update(kw)
    return ssd.lib.ssd_paged_mx_decode_attn(_ref(cfg), a["f"], a["q"], a["k"], a["v"], a["ks"], a["vs"], a["wi"], a["wo"], a["table"], a["len"], a["out"], a["lse"], a["most"],
                                            a["ws"], a["size"], None)


def _step(cfg, **kw):
    a = dict(f=4, q=FAKE, kn=FAKE, vn=FAKE, k=FAKE, v=FAKE, ks=FAKE, vs=FAKE, pos=FAKE, wi=FAKE, wo=FAKE, table=FAKE, len=FAKE, total=FAKE, out=FAKE, lse=FAKE, most=0, ws=FAKE,
             size=1 << 40)
    a.update(kw)
    return ssd.lib.ssd_paged_mx_decode_step(_ref(cfg), a["f"], a["q"], a["kn"], a["vn"], a["k"], a["v"], a["ks"], a["vs"], a["pos"], a["wi"], a["wo"], a["table"], a["len"],
                                            a["total"], a["out"], a["lse"], a["most"], a["ws"], a["size"], None)


def _evict(cfg, **kw):
    a = dict(f=4, k=FAKE, v=FAKE, ks=FAKE, vs=FAKE, table=FAKE, len=FAKE, total=FAKE, budget=FAKE, sink=1, recent=2, pi=FAKE, po=FAKE, wi=FAKE, wo=FAKE, lo=FAKE + 64, most=0,
             ws=FAKE, size=1 << 40)
    a.update(kw)
    return ssd.lib.ssd_paged_mx_evict(_ref(cfg), a["f"], a["k"], a["v"], a["ks"], a["vs"], a["table"], a["len"], a["total"], a["budget"], a["sink"], a["recent"], a["pi"], a["po"],
                                      a["wi"], a["wo"], a["lo"], a["most"], a["ws"], a["size"], None)


CALLS = [_append, _read, _attn, _step, _evict]


@pytest.mark.parametrize("bad", [b for b in BAD_CONFIG if "row_stride" not in b], ids=lambda b: ",".join("%s=%s" % i for i in b.items()))
def test_bad_config_is_refused_by_every_call(bad):
    cfg = _cfg(**bad)
    assert ssd.ssd_paged_mx_workspace_bytes(cfg, "mxfp4", 0, True) == 0 and ssd.ssd_paged_mx_evict_workspace_bytes(cfg, "mxfp8", 0) == 0
    for call in CALLS:
        assert call(cfg) == BAD
        assert ssd.ssd_last_error() != ""
    cfg = _cfg()
    cfg.reserved[2] = 1
    for call in CALLS:
        assert call(cfg) == BAD


@pytest.mark.parametrize("call", CALLS, ids=lambda c: c.__name__)
def test_formats_pools_and_scales(call):
    assert call(None) == BAD
    for bad in (dict(f=0), dict(f=2), dict(f=16), dict(k=None), dict(v=None), dict(k=FAKE + 8), dict(v=FAKE + 4), dict(ks=None), dict(vs=None), dict(ks=FAKE + 8), dict(vs=FAKE + 4),
                dict(table=None), dict(len=None), dict(table=FAKE + 1), dict(len=FAKE + 2)):
        assert call(_cfg(), **bad) == BAD, bad
        assert ssd.ssd_last_error() != ""


def test_strides_count_elements_of_the_format():
    """16 bytes are 32 elements of four bits, 16 of eight."""
    for f, unit in ((4, 32), (8, 16)):
        for page, head, row in ((8192, 4096, 128 + unit // 2), (8192, 4096 + 8, 128), (8192 + 4, 4096, 128), (4096, 2048, 64), (1 << 49, 128, 128)):
            cfg = _cfg(page_stride=page, head_stride=head, row_stride=row)
            for call in CALLS:
                assert call(cfg, f=f) == BAD, (f, page, head, row)
        cfg = _cfg(page_stride=8192, head_stride=4096, row_stride=128 + unit)
        assert _append(cfg, f=f, n=0) == ssd.SSD_OK                  # nothing to write, nothing enqueued


def test_append_and_read_refusals():
    for bad in (dict(kn=None), dict(vn=None), dict(kn=FAKE + 4), dict(vn=FAKE + 2), dict(start=FAKE + 3), dict(n=-1), dict(start=None, n=5), dict(start=None, n=0)):
        for call in (_append, _read):
            assert call(_cfg(), **bad) == BAD, bad
            assert ssd.ssd_last_error() != ""
    for bad in (dict(pos=FAKE + 2), dict(weight=FAKE + 1), dict(total=FAKE + 1), dict(wn=FAKE + 1)):
        assert _append(_cfg(), **bad) == BAD, bad
    assert _read(_cfg(), first=FAKE + 2) == BAD
    for call in (_append, _read):
        assert call(_cfg(), n=0, kn=None, vn=None) == ssd.SSD_OK


def test_attention_refusals():
    need = ssd.ssd_paged_mx_workspace_bytes(_cfg(max_blocks=1000), "mxfp4", 0, True)
    assert need > 0
    for bad in (dict(q=None), dict(out=None), dict(q=FAKE + 8), dict(out=FAKE + 8), dict(wi=None), dict(wo=None), dict(wi=FAKE + 2), dict(wo=FAKE + 2), dict(lse=FAKE + 1), dict(most=-1),
                dict(most=16001), dict(ws=None), dict(ws=FAKE + 128), dict(size=need - 1)):
        for call in (_attn, _step):
            assert call(_cfg(max_blocks=1000), **bad) == BAD, bad
            assert ssd.ssd_last_error() != ""
    for bad in (dict(kn=None), dict(vn=None), dict(kn=FAKE + 8), dict(vn=FAKE + 8), dict(pos=FAKE + 1), dict(total=FAKE + 2)):
        assert _step(_cfg(max_blocks=1000), **bad) == BAD, bad


def test_eviction_refusals():
    need = ssd.ssd_paged_mx_evict_workspace_bytes(_cfg(), "mxfp8", 0)
    assert need > 0
    for bad in (dict(budget=None), dict(pi=None), dict(po=None), dict(wi=None), dict(wo=None), dict(po=FAKE + 4), dict(wo=FAKE + 4), dict(lo=FAKE), dict(sink=-1), dict(recent=-1),
                dict(most=-1), dict(most=161), dict(ws=None), dict(ws=FAKE + 64), dict(size=need - 1), dict(total=FAKE + 1), dict(budget=FAKE + 2), dict(lo=FAKE + 65)):
        assert _evict(_cfg(), **bad) == BAD, bad
        assert ssd.ssd_last_error() != ""


def _rope(**kw):
    a = dict(x=FAKE, out=2 * FAKE, n=4, H=2, d=64, t=0, xs=0, os=0, pos=FAKE, axes=2, axis=FAKE, inv=FAKE, pairs=32, layout=1, inverse=0)
    a.update(kw)
    return ssd.lib.ssd_rope_axes(a["x"], a["out"], a["n"], a["H"], a["d"], a["t"], a["xs"], a["os"], a["pos"], a["axes"], a["axis"], a["inv"], a["pairs"], a["layout"], a["inverse"], None)


def test_rope_refusals():
    for bad in (dict(x=None), dict(out=None), dict(pos=None), dict(inv=None), dict(x=FAKE + 2), dict(out=2 * FAKE + 1), dict(x=FAKE + 1, t=1), dict(pos=FAKE + 2), dict(inv=FAKE + 2),
                dict(n=-1), dict(n=1 << 24), dict(H=0), dict(H=4097), dict(d=0), dict(d=63), dict(d=1026), dict(t=2), dict(pairs=0), dict(pairs=33), dict(axes=0), dict(axes=5), dict(axis=None),
                dict(layout=0), dict(layout=3), dict(inverse=2), dict(xs=127), dict(os=64), dict(xs=-128), dict(xs=(1 << 28) + 1)):
        assert _rope(**bad) == BAD, bad
        assert ssd.ssd_last_error() != ""
    assert _rope(n=0) == ssd.SSD_OK and _rope(n=0, x=None, out=None, pos=None) == ssd.SSD_OK


def test_rope_onto_itself_or_apart():
    """In place with one stride, or no memory in common."""
    row = 2 * 64 * 4
    for bad in (dict(out=FAKE, os=256), dict(out=FAKE + 4), dict(out=FAKE + 3 * row), dict(out=FAKE - row), dict(out=FAKE - 1 * row + 4)):
        assert _rope(**bad) == BAD, bad
        assert "share" in ssd.ssd_last_error()


def test_binding_refuses_tensors_that_lie_otherwise():
    bt = MxBatch([20, 5], 4, 2, 64, "bf16", "mxfp4", 16, seed=1, device="cpu")
    new = torch.zeros((2, 2, 64), dtype=torch.bfloat16)
    k, v, ks, vs = bt.pools

    def call(k=k, v=v, ks=ks, vs=vs, fmt="mxfp4", cfg=bt.cfg):
        ssd.ssd_paged_mx_append(cfg, fmt, k, v, ks, vs, bt.tabled, bt.lend, new, new)

    for bad in (dict(k=k.to(torch.int32)), dict(k=k[:, :, :, :16]), dict(v=v.transpose(0, 1)), dict(v=v[:, :1]), dict(k=k[1:]), dict(ks=ks[:, :, :8]), dict(vs=vs[1:]),
                dict(vs=vs.transpose(1, 2)), dict(fmt="mxfp8"), dict(fmt="fp4"), dict(k=k.flatten()[:-1])):
        with pytest.raises(ValueError):
            call(**bad)
    for layout in ("rows", "both", "wide"):                          # and takes what lies as the config says, whichever way it is named
        other = MxBatch([20, 5], 4, 2, 64, "bf16", "mxfp8", 16, seed=1, layout=layout, device="cpu")
        for t in (other.kd, other.kd.transpose(1, 2)):
            assert _mx_pools(other.cfg, "mxfp8", t, t, other.ksd, other.vsd) == (8, t.data_ptr(), t.data_ptr(), other.ksd.data_ptr(), other.vsd.data_ptr())
        with pytest.raises(ValueError):
            _mx_pools(other.cfg, "mxfp8", bt.kd, other.vd, other.ksd, other.vsd)


def test_binding_of_the_rotation_refuses_short_arrays():
    x, pos, inv = torch.zeros((4, 2, 64)), torch.zeros((2, 4), dtype=torch.int32), torch.ones(32)
    axis = torch.zeros(32, dtype=torch.uint8)
    for bad in (dict(pos=pos[:, :3]), dict(pos=torch.zeros((1, 4), dtype=torch.int32)), dict(axis=axis[:31]), dict(inv_freq=inv[::2], n_pairs=32), dict(x=x[:3]), dict(x=x[:, :, ::2]),
                dict(out=x[:, :1])):
        a = dict(x=x, out=x.clone(), pos=pos, inv_freq=inv, axis=axis)
        a.update(bad)
        with pytest.raises(ValueError):
            ssd.ssd_rope_axes(a.pop("x"), a.pop("out"), 4, 2, 64, "f32", a.pop("pos"), a.pop("inv_freq"), n_axes=2, **a)


def test_binding_refuses_elements_of_another_size():
    bt = MxBatch([20, 5], 4, 2, 64, "bf16", "mxfp4", 16, seed=1, device="cpu")
    new, wrong = torch.zeros((2, 2, 64), dtype=torch.bfloat16), torch.zeros((2, 2, 64))
    out, wide = torch.zeros((2, 4, 64), dtype=torch.bfloat16), torch.zeros((2, 4, 64))
    head, tail = (bt.cfg, "mxfp4"), (bt.tabled, bt.lend)
    for call in (lambda: ssd.ssd_paged_mx_append(*head, *bt.pools, *tail, wrong, new), lambda: ssd.ssd_paged_mx_append(*head, *bt.pools, *tail, new, wrong),
                 lambda: ssd.ssd_paged_mx_read(*head, *bt.pools, *tail, wrong, new), lambda: ssd.ssd_paged_mx_read(*head, *bt.pools, *tail, new, wrong),
                 lambda: ssd.ssd_paged_mx_decode_attn(*head, wide, *bt.pools, *tail, out), lambda: ssd.ssd_paged_mx_decode_attn(*head, out, *bt.pools, *tail, wide),
                 lambda: ssd.ssd_paged_mx_decode_step(*head, out, wrong, new, *bt.pools, *tail, out), lambda: ssd.ssd_paged_mx_decode_step(*head, out, new, wrong, *bt.pools, *tail, out),
                 lambda: ssd.ssd_rope_axes(wide, wide, 2, 4, 64, "bf16", bt.lend, torch.ones(32)), lambda: ssd.ssd_rope_axes(out, out, 2, 4, 64, "f32", bt.lend, torch.ones(32))):
        with pytest.raises(ValueError, match="bytes are expected"):
            call()


def test_what_a_user_keeps_at_a_config_stays():
    cfg = ssd.make_paged_config(2, 4, 2, 64, "bf16", 16, 4, 2)
    cfg.note = "kept"
    assert cfg.strides and cfg.mx_strides
    cfg.page_size = 32
    assert cfg.note == "kept" and cfg.strides[0][1] == 32 * 64 and cfg.mx_strides[8][0][1] == 32 * 64


def test_binding_of_the_rotation_refuses_broadcast_rows():
    """One row in the place of many has no second row to read or write."""
    x, pos, inv = torch.zeros((4, 2, 64)), torch.zeros((1, 4), dtype=torch.int32), torch.ones(32)
    for one in (x[:1].expand(4, 2, 64), x[:1, :1].expand(4, 2, 64), x.flatten(1)[:1].expand(4, 128)):
        for a, b in ((one, x), (x, one)):
            with pytest.raises(ValueError):
                ssd.ssd_rope_axes(a, b, 4, 2, 64, "f32", pos, inv)


def test_binding_refuses_fewer_rows_than_the_call_takes():
    bt = MxBatch([20, 5], 4, 2, 64, "bf16", "mxfp4", 16, seed=1, device="cpu")
    head, tail = (bt.cfg, "mxfp4"), (bt.tabled, bt.lend)
    rows, few, heads, short = (torch.zeros(s, dtype=torch.bfloat16) for s in ((3, 2, 64), (2, 2, 64), (3, 1, 64), (3, 2, 32)))
    out, one = torch.zeros((2, 4, 64), dtype=torch.bfloat16), torch.zeros((1, 4, 64), dtype=torch.bfloat16)
    starts = torch.tensor([0, 2, 3], dtype=torch.int32)
    for call in (lambda x: ssd.ssd_paged_mx_append(*head, *bt.pools, *tail, x, rows, new_start=starts, n_new=3), lambda x: ssd.ssd_paged_mx_read(*head, *bt.pools, *tail, rows, x, row_start=starts, n_rows=3)):
        for x in (few, heads, short, rows[:, :1]):
            with pytest.raises(ValueError):
                call(x)
    for q, o in ((one, out), (out, one), (out, out[:, :2])):
        with pytest.raises(ValueError):
            ssd.ssd_paged_mx_decode_attn(*head, q, *bt.pools, *tail, o)
    with pytest.raises(ValueError):
        ssd.ssd_paged_mx_decode_step(*head, out, few[:1], few, *bt.pools, *tail, out)
