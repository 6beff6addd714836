"""CPU-only checks of the paged cache's calls and of ssd_logits_process: what they refuse, before anything is launched, and the sizes of
their workspaces."""
import ctypes as C

import pytest

import paper_2510_18716_amd as ssd
from paper_2510_18716_amd.binding import SsdLogitsParams, SsdPagedConfig, make_paged_config

FAKE = 1 << 24


def _cfg(**kw):
    cfg = make_paged_config(4, 8, 2, 128, "bf16", 16, 100, 10)
    for k, v in kw.items():
        setattr(cfg, k, v)
    return cfg


def test_struct_sizes_agree_with_the_header():
    assert C.sizeof(SsdPagedConfig) == 12 * 4 + 5 * 8 and C.sizeof(SsdLogitsParams) == 12 * 8


BAD_CONFIG = [dict(n_seqs=0), dict(n_seqs=65536), dict(n_kv_heads=0), dict(n_kv_heads=3), dict(n_heads=0), dict(n_heads=2048), dict(head_dim=96),
              dict(dtype=2), dict(page_size=0), dict(page_size=32769), dict(n_pages=0), dict(max_blocks=0), dict(max_blocks=1 << 22),
              dict(softmax_scale=-1.0), dict(softmax_scale=float("nan")), dict(page_stride=1024), dict(page_stride=4096, head_stride=2048, row_stride=120),
              dict(page_stride=4096, head_stride=2052, row_stride=128), dict(page_stride=1 << 49, head_stride=128, row_stride=128),
              dict(page_stride=-4096, head_stride=2048, row_stride=128), dict(q_stride=8), dict(q_stride=1028), dict(new_stride=100), dict(new_stride=-256)]


@pytest.mark.parametrize("bad", BAD_CONFIG, ids=lambda b: ",".join("%s=%s" % i for i in b.items()))
def test_bad_config_is_refused_by_every_call(bad):
    cfg = _cfg(**bad)
    assert ssd.ssd_paged_workspace_bytes(cfg, 0, True) == 0 and ssd.ssd_paged_evict_workspace_bytes(cfg, 0) == 0
    assert ssd.ssd_last_error() != ""
    for call in (_append, _attn, _step, _evict):
        assert call(cfg) == ssd.SSD_ERR_INVALID_ARG
    cfg = _cfg()
    cfg.reserved[1] = 1
    for call in (_append, _attn, _step, _evict):
        assert call(cfg) == ssd.SSD_ERR_INVALID_ARG


def _ref(cfg):
    return None if cfg is None else C.byref(cfg)


def _append(cfg, **kw):
    a = dict(k=FAKE, v=FAKE, pos=FAKE, weight=FAKE, table=FAKE, len=FAKE, total=FAKE, kn=FAKE, vn=FAKE, start=FAKE, n=5, wn=FAKE)
    a.update(kw)
    return ssd.lib.ssd_paged_append(_ref(cfg), a["k"], a["v"], a["pos"], a["weight"], a["table"], a["len"], a["total"], a["kn"], a["vn"], a["start"], a["n"], a["wn"], None)


def _attn(cfg, **kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, wi=FAKE, wo=FAKE, table=FAKE, len=FAKE, out=FAKE, lse=FAKE, most=0, ws=FAKE, size=1 << 30)
    a.update(kw)
    return ssd.lib.ssd_paged_decode_attn(_ref(cfg), a["q"], a["k"], a["v"], a["wi"], a["wo"], a["table"], a["len"], a["out"], a["lse"], a["most"], a["ws"], a["size"], None)


def _step(cfg, **kw):
    a = dict(q=FAKE, kn=FAKE, vn=FAKE, k=FAKE, v=FAKE, pos=FAKE, wi=FAKE, wo=FAKE, table=FAKE, len=FAKE, total=FAKE, out=FAKE, lse=FAKE, most=0, ws=FAKE, size=1 << 30)
    a.update(kw)
    return ssd.lib.ssd_paged_decode_step(_ref(cfg), a["q"], a["kn"], a["vn"], a["k"], a["v"], a["pos"], a["wi"], a["wo"], a["table"], a["len"], a["total"], a["out"],
                                         a["lse"], a["most"], a["ws"], a["size"], None)


def _evict(cfg, **kw):
    a = dict(k=FAKE, v=FAKE, table=FAKE, len=FAKE, total=FAKE, budget=FAKE, sink=1, recent=2, pi=FAKE, po=FAKE, wi=FAKE, wo=FAKE, lo=FAKE + 64, most=0, ws=FAKE,
             size=1 << 30)
    a.update(kw)
    return ssd.lib.ssd_paged_evict(_ref(cfg), a["k"], a["v"], a["table"], a["len"], a["total"], a["budget"], a["sink"], a["recent"], a["pi"], a["po"], a["wi"], a["wo"],
                                   a["lo"], a["most"], a["ws"], a["size"], None)


def _all_refused(call, bads, cfg=None):
    cfg = cfg or _cfg()
    assert call(None) == ssd.SSD_ERR_INVALID_ARG
    for bad in bads:
        assert call(cfg, **bad) == ssd.SSD_ERR_INVALID_ARG, bad
        assert ssd.ssd_last_error() != ""


def test_append_refusals():
    _all_refused(_append, [dict(k=None), dict(v=None), dict(kn=None), dict(vn=None), dict(k=FAKE + 8), dict(v=FAKE + 8), dict(kn=FAKE + 4), dict(vn=FAKE + 2),
                           dict(table=None), dict(len=None), dict(table=FAKE + 1), dict(len=FAKE + 2), dict(total=FAKE + 1), dict(pos=FAKE + 2),
                           dict(weight=FAKE + 1), dict(start=FAKE + 3), dict(wn=FAKE + 1), dict(n=-1), dict(start=None, n=5), dict(start=None, n=0)])
    assert _append(_cfg(), n=0) == ssd.SSD_OK                        # nothing to write, nothing enqueued


def test_attention_refusals():
    need = ssd.ssd_paged_workspace_bytes(_cfg(), 0, True)
    bads = [dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(q=FAKE + 8), dict(k=FAKE + 8), dict(v=FAKE + 8), dict(out=FAKE + 8), dict(table=None),
            dict(len=None), dict(wi=None), dict(wo=None), dict(wi=FAKE + 2), dict(wo=FAKE + 2), dict(lse=FAKE + 1), dict(table=FAKE + 1), dict(len=FAKE + 1), dict(most=-1), dict(most=161)]
    if need:
        bads += [dict(ws=None), dict(ws=FAKE + 128), dict(size=need - 1)]
    _all_refused(_attn, bads)
    _all_refused(_step, bads + [dict(kn=None), dict(vn=None), dict(kn=FAKE + 8), dict(vn=FAKE + 8), dict(pos=FAKE + 1), dict(total=FAKE + 2)])


def test_eviction_refusals():
    need = ssd.ssd_paged_evict_workspace_bytes(_cfg(), 0)
    assert need > 0
    _all_refused(_evict, [dict(k=None), dict(v=None), dict(k=FAKE + 8), dict(v=FAKE + 4), dict(table=None), dict(len=None), dict(budget=None), dict(pi=None), dict(po=None),
                          dict(wi=None), dict(wo=None), dict(po=FAKE + 4), dict(wo=FAKE + 4), dict(lo=FAKE), dict(sink=-1), dict(recent=-1), dict(most=-1), dict(most=161),
                          dict(ws=None), dict(ws=FAKE + 64), dict(size=need - 1), dict(table=FAKE + 1), dict(total=FAKE + 1), dict(budget=FAKE + 2),
                          dict(pi=FAKE + 1, po=FAKE + 1), dict(wi=FAKE + 1, wo=FAKE + 1), dict(lo=FAKE + 65)])


def test_lengths_after_an_eviction_need_an_array_of_their_own():
    for same in (dict(len=FAKE + 64), dict(total=FAKE + 64), dict(budget=FAKE + 64)):
        assert _evict(_cfg(), **same) == ssd.SSD_ERR_INVALID_ARG, same
        assert "seq_len_out" in ssd.ssd_last_error()


def test_attention_over_long_rows_needs_its_workspace():
    for weights in (False, True):
        cfg = _cfg(max_blocks=1000)
        need = ssd.ssd_paged_workspace_bytes(cfg, 0, weights)
        assert need > 0
        more = {} if weights else dict(wi=None, wo=None)
        for call in (_attn, _step):
            for bad in (dict(ws=None), dict(ws=FAKE + 128), dict(size=need - 1)):
                assert call(cfg, **more, **bad) == ssd.SSD_ERR_INVALID_ARG, bad
                assert "workspace" in ssd.ssd_last_error()


def test_workspaces_grow_with_the_bound_and_not_with_the_table():
    small, large = _cfg(), _cfg(max_blocks=1000)
    for size in (lambda c, n: ssd.ssd_paged_workspace_bytes(c, n, True), ssd.ssd_paged_evict_workspace_bytes):
        assert size(small, 100) == size(large, 100)
        assert size(large, 0) >= size(large, 100)
        assert size(large, 0) == size(large, 16000)


def test_logits_refusals():
    def call(p=None, **kw):
        a = dict(x=FAKE, n=4, V=100, dtype=0, xs=0, guided=0, gamma=1.0, out=FAKE + 4096, os=0)
        a.update(kw)
        s = SsdLogitsParams()
        for k, v in (p or {}).items():
            setattr(s, k, v)
        return ssd.lib.ssd_logits_process(a["x"], a["n"], a["V"], a["dtype"], a["xs"], a["guided"], a["gamma"], None if p == 0 else C.byref(s), a["out"], a["os"], None)

    for bad in (dict(x=None), dict(out=None), dict(x=FAKE + 4), dict(out=FAKE + 8), dict(n=0), dict(n=65536), dict(V=0), dict(V=(1 << 24) + 1), dict(dtype=2), dict(xs=99),
                dict(os=99), dict(xs=-1), dict(guided=2), dict(guided=1, gamma=float("nan")), dict(out=FAKE, dtype=1), dict(out=FAKE, guided=1), dict(out=FAKE, xs=104),
                dict(p=0)):
        assert call(**bad) == ssd.SSD_ERR_INVALID_ARG, bad
        assert ssd.ssd_last_error() != ""
    for bad in (dict(tokens=FAKE), dict(n_tokens=FAKE), dict(tokens=FAKE, n_tokens=FAKE, token_stride=-1), dict(tokens=FAKE, n_tokens=FAKE, token_stride=1 << 31),
                dict(bias=FAKE, bias_stride=99), dict(mask=FAKE, mask_stride=3), dict(bias=FAKE + 2), dict(mask=FAKE + 1), dict(repetition=FAKE + 1), dict(temperature=FAKE + 2),
                dict(tokens=FAKE + 2, n_tokens=FAKE)):
        assert call(p=bad) == ssd.SSD_ERR_INVALID_ARG, bad
        assert ssd.ssd_last_error() != ""
