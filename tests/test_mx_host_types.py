"""CPU: the binding refuses tensors of another type, shape or size than a call on quantised pages or a rotation reads and writes; the library is not reached."""
import pytest
import torch

import paper_2510_18716_amd as ssd
from mx_harness import MxBatch
from paper_2510_18716_amd import binding

INT, F32, BF16 = torch.int32, torch.float32, torch.bfloat16


class Stub:
    """Every entry point answers 0; `calls` are their names."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            return 0
        return call


@pytest.fixture
def stub(monkeypatch):
    s = Stub()
    monkeypatch.setattr(binding, "lib", s)
    return s


def refused(stub, call):
    with pytest.raises((ValueError, AssertionError)):
        call()
    assert stub.calls == []


def taken(stub, call):
    call()
    assert len(stub.calls) == 1
    stub.calls.clear()


# ---- the rotation's tables

def _rope(**kw):
    a = dict(x=torch.zeros((4, 2, 64)), pos=torch.zeros((2, 4), dtype=INT), inv_freq=torch.ones(32), axis=torch.zeros(32, dtype=torch.uint8), n_axes=2, dtype="f32")
    a["out"] = torch.zeros_like(a["x"])
    a.update(kw)
    ssd.ssd_rope_axes(a.pop("x"), a.pop("out"), 4, 2, 64, a.pop("dtype"), a.pop("pos"), a.pop("inv_freq"), **a)


@pytest.mark.parametrize("bad", [dict(pos=torch.zeros((2, 4), dtype=t)) for t in (torch.int64, torch.int16, torch.uint8, F32, torch.float64)] +
                         [dict(inv_freq=torch.ones(32).to(t)) for t in (torch.float64, BF16, torch.float16, INT)] +
                         [dict(axis=torch.zeros(32, dtype=t)) for t in (torch.int64, INT, torch.int16, F32, torch.float8_e4m3fn)] +
                         [dict(pos=torch.zeros((2, 8), dtype=torch.int16)), dict(pos=torch.arange(8)), dict(axis=torch.zeros(64, dtype=torch.int64)), dict(inv_freq=torch.ones(64).to(BF16))],
                         ids=lambda b: "-".join("%s-%s-%d" % (k, v.dtype, v.numel()) for k, v in b.items()))
def test_tables_of_the_rotation_of_another_type(stub, bad):
    taken(stub, _rope)
    refused(stub, lambda: _rope(**bad))


def test_axes_of_any_byte_that_is_a_whole_number(stub):
    for t in (torch.int8, torch.bool):
        taken(stub, lambda: _rope(axis=torch.zeros(32, dtype=t)))


def test_rows_of_the_rotation_of_another_type(stub):
    for t in (torch.float16, torch.int16):
        x = torch.zeros((4, 2, 64), dtype=t)
        refused(stub, lambda: _rope(x=x, dtype="bf16", out=torch.zeros((4, 2, 64), dtype=BF16)))
        refused(stub, lambda: _rope(x=torch.zeros((4, 2, 64), dtype=BF16), dtype="bf16", out=x))
    refused(stub, lambda: _rope(x=torch.zeros((4, 2, 64), dtype=INT)))


# ---- the calls on quantised pages

B, H, KV, D, PAGES, PAGE, BLOCKS = 4, 4, 2, 64, 9, 16, 3


def _args(dtype="bf16", fmt="mxfp4", **cfg):
    t = BF16 if dtype == "bf16" else F32
    bits = 4 if fmt == "mxfp4" else 8
    pool, places = (PAGES, KV, PAGE, D * bits // 8), (PAGES, KV, PAGE)
    a = {"cfg": ssd.make_paged_config(B, H, KV, D, dtype, PAGE, PAGES, BLOCKS, **cfg), "fmt": fmt}
    a.update({n: torch.zeros(pool, dtype=torch.uint8) for n in ("k_pages", "v_pages")})
    a.update({n: torch.zeros(places + (D // 32,), dtype=torch.uint8) for n in ("k_scales", "v_scales")})
    a.update(block_table=torch.zeros((B, BLOCKS), dtype=INT), seq_len=torch.zeros(B, dtype=INT), seq_pos=torch.zeros(B, dtype=INT), budget=torch.zeros(B, dtype=INT),
             new_start=torch.zeros(B + 1, dtype=INT), row_start=torch.zeros(B + 1, dtype=INT), first_slot=torch.zeros(B, dtype=INT), seq_len_out=torch.zeros(B, dtype=INT))
    a.update({n: torch.zeros(places, dtype=INT) for n in ("pos", "pos_in", "pos_out")})
    a.update({n: torch.zeros(places) for n in ("weight", "weight_in", "weight_out")})
    a.update({n: torch.zeros((B, KV, D), dtype=t) for n in ("k_new", "v_new", "k_out", "v_out")})
    a.update(q=torch.zeros((B, H, D), dtype=t), out=torch.zeros((B, H, D), dtype=t), lse=torch.zeros((B, H)), weight_new=torch.zeros((B, KV)), workspace=torch.zeros(256))
    return a


POOL = ("k_pages", "v_pages", "k_scales", "v_scales")
CALLS = {"append": (POOL + ("block_table", "seq_len", "k_new", "v_new"), ("pos", "weight", "seq_pos", "new_start", "weight_new")),
         "read": (POOL + ("block_table", "seq_len", "k_out", "v_out"), ("row_start", "first_slot")),
         "decode_attn": (("q",) + POOL + ("block_table", "seq_len", "out"), ("lse", "weight_in", "weight_out", "workspace")),
         "decode_step": (("q", "k_new", "v_new") + POOL + ("block_table", "seq_len", "out"), ("pos", "seq_pos", "lse", "weight_in", "weight_out", "workspace")),
         "evict": (POOL + ("block_table", "seq_len", "budget", "pos_in", "pos_out", "weight_in", "weight_out"), ("seq_len_out", "seq_pos", "workspace"))}


def _call(name, a, **kw):
    a = dict(a, **kw)
    first, more = CALLS[name]
    getattr(ssd, "ssd_paged_mx_" + name)(a["cfg"], a["fmt"], *[a[x] for x in first], **{x: a[x] for x in more})


def _users(arg):
    return [n for n, (first, more) in CALLS.items() if arg in first + more]


WIDE = dict(q_stride=(H + 2 * KV) * D, new_stride=(H + 2 * KV) * D)      # q and new rows lie in rows of a projection


@pytest.mark.parametrize("name", CALLS)
def test_what_the_calls_take(stub, name):
    for dtype in ("bf16", "f32"):
        for fmt in ("mxfp4", "mxfp8"):
            taken(stub, lambda: _call(name, _args(dtype, fmt)))
    a = _args(**WIDE)
    rows = torch.zeros((B, (H + 2 * KV) * D), dtype=BF16)
    flat = dict(q=rows[:, :H * D], **{n: rows[:, H * D:(H + KV) * D] for n in ("k_new", "v_new", "k_out", "v_out")})
    taken(stub, lambda: _call(name, a, **flat))
    taken(stub, lambda: _call(name, a, **{n: t.unflatten(1, (-1, D)) for n, t in flat.items()}))
    a = _args()
    taken(stub, lambda: _call(name, a, **{n: a[n].flatten(1) for n in ("q", "k_new", "v_new", "k_out", "v_out", "out", "pos", "weight_in")}))
    taken(stub, lambda: _call(name, a, **{n: a[n].view(torch.float8_e4m3fn) for n in POOL}))
    taken(stub, lambda: _call(name, a, **{n: torch.nn.Parameter(a[n]) for n in ("q", "k_new", "v_new")}))


@pytest.mark.parametrize("arg", ["q", "k_new", "v_new", "k_out", "v_out", "out"])
def test_rows_and_outputs_of_another_type(stub, arg):
    """Half as many rows of twice the size are as many bytes; 16 bits may be another number."""
    for name in _users(arg):
        a = _args()
        t = a[arg]
        for bad in (torch.zeros((B // 2,) + t.shape[1:]), torch.zeros(t.shape, dtype=torch.float16), torch.zeros(t.shape, dtype=torch.int16), torch.zeros(t.shape),
                    torch.zeros(t.shape[:2] + (D // 2,)), torch.zeros(t.shape + (2,), dtype=torch.uint8)):
            refused(stub, lambda: _call(name, a, n_rows=B, n_new=B, **{arg: bad}))
        a = _args("f32")
        for bad in (torch.zeros((2 * B,) + t.shape[1:], dtype=BF16), torch.zeros(t.shape, dtype=INT), torch.zeros(t.shape[:2] + (D // 2,), dtype=torch.float64)):
            refused(stub, lambda: _call(name, a, **{arg: bad}))


@pytest.mark.parametrize("arg", ["q", "k_new", "v_new", "k_out", "v_out"])
def test_rows_that_do_not_reach_as_far(stub, arg):
    """The config's strides and as many elements, in fewer rows."""
    heads = H if arg == "q" else KV
    row = (H + 2 * KV) * D
    memory = torch.zeros(2 * B * row, dtype=BF16)
    for name in _users(arg):
        if name in ("append", "read") and arg in ("k_new", "k_out"):
            continue                                                # its own rows say how many there are
        a = _args(**WIDE)
        good = memory[:B * row].view(B, row)
        a.update({n: good[:, :(H if n == "q" else KV) * D] for n in ("q", "k_new", "v_new", "k_out", "v_out")})
        taken(stub, lambda: _call(name, a))
        for bad in (good[:2, :2 * heads * D].unflatten(1, (2 * heads, D)), good[:2, :heads * D], good[:2, :heads * D].unflatten(1, (heads, D)), good[:3, :heads * D],
                    good[:, :heads * D].unflatten(1, (heads, D))[:, :heads - 1], good[:1, :heads * D].expand(B, heads * D), good[:, :heads * D].unflatten(1, (heads, D)).transpose(1, 2)):
            refused(stub, lambda: _call(name, a, **{arg: bad}))


@pytest.mark.parametrize("arg", ["k_pages", "v_pages"])
def test_pools_that_do_not_reach_as_far_or_are_not_bytes(stub, arg):
    """Pages farther apart than their rows need."""
    gap = 4 * KV * PAGE * D // 2
    memory = torch.zeros(PAGES * gap + 64, dtype=torch.uint8)
    a = _args(page_stride=2 * gap, head_stride=PAGE * D, row_stride=D)
    good = memory.as_strided((PAGES, KV, PAGE, D // 2), (gap, PAGE * D // 2, D // 2, 1))
    a.update(k_pages=good, v_pages=good)
    for name in CALLS:
        taken(stub, lambda: _call(name, a))
        for bad in (memory.as_strided((PAGES // 3, 3 * KV, PAGE, D // 2), good.stride()), memory.as_strided((PAGES // 3, KV, 3 * PAGE, D // 2), good.stride()), good[:-1],
                    torch.zeros(PAGES * gap, dtype=torch.int16).as_strided((PAGES // 3, KV, PAGE, D // 2), good.stride())):
            refused(stub, lambda: _call(name, a, **{arg: bad}))
    dense = _args()
    for bad in (torch.zeros((PAGES, KV, PAGE, D // 4), dtype=torch.int16), torch.zeros((PAGES, KV, PAGE, D // 2), dtype=torch.int16)):
        for name in CALLS:
            refused(stub, lambda: _call(name, dense, **{arg: bad}))


@pytest.mark.parametrize("arg", ["block_table", "seq_len", "seq_pos", "budget", "new_start", "row_start", "first_slot", "seq_len_out", "pos", "pos_in", "pos_out", "weight", "weight_in",
                                 "weight_out", "weight_new", "lse"])
def test_tables_of_another_type_or_with_fewer_entries(stub, arg):
    """torch's whole numbers have 64 bits where nothing else is said."""
    for name in _users(arg):
        a = _args()
        t = a[arg]
        for other in (torch.int64, torch.int16, torch.uint8, BF16, torch.float64, F32 if t.dtype is INT else INT):
            refused(stub, lambda: _call(name, a, **{arg: t.to(other)}))
        for bad in (t.flatten()[:-1], t.flatten()[::2], torch.zeros((2,) + t.shape, dtype=t.dtype).transpose(0, -1)):
            refused(stub, lambda: _call(name, a, **{arg: bad}))
        taken(stub, lambda: _call(name, a, **{arg: torch.zeros(t.numel() + 3, dtype=t.dtype)}))


@pytest.mark.parametrize("arg", ["k_scales", "v_scales"])
def test_scales_that_are_fewer_or_lie_apart(stub, arg):
    for name in CALLS:
        a = _args()
        for bad in (a[arg].flatten()[:-1], a[arg].transpose(1, 2), a[arg][:-1]):
            refused(stub, lambda: _call(name, a, **{arg: bad}))
