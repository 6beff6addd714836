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
