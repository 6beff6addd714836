"""GPU parity of ssd_logits_process against a plain 64-bit implementation, through the C ABI.

Tolerance: at most nine roundings to fp32 between an input and the result, each 2^-24 of a value no larger than the largest on the way
(its parts, times the repetition, over the temperature): 9 * 2^-24 of that, taken as 6e-7 * (1 + size / temperature)."""
import numpy as np
import pytest
import torch

import paper_2510_18716_amd as ssd
from oracle import paged

pytestmark = pytest.mark.gpu
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(rows, V, dtype, guided, bias, mask, history, seed, gap=0, prompt=0, params=True, in_place=False, spread=4.0):
    print("logits", rows, V, dtype, guided, bias, mask, history, seed, gap, flush=True)
    rng = np.random.default_rng(seed)
    n_in = rows * (2 if guided else 1)
    x = torch.full((n_in, V + gap), float("nan"), dtype=TORCH[dtype])
    x[:, :V] = torch.from_numpy((rng.standard_normal((n_in, V)) * spread).astype(np.float32)).to(TORCH[dtype])
    n_tok = rng.integers(0, history + 1, rows).astype(np.int32)
    n_tok[0] = history
    tok = (rng.random((rows, max(1, history))) ** 4 * (V + 2)).astype(np.int32) - 1            # -1 and V among them
    n_prompt = np.minimum(n_tok, prompt).astype(np.int32)
    rep, pres, freq, temp = (rng.random(rows).astype(np.float32) * s + o for s, o in ((1.0, 0.5), (1.0, -0.2), (0.3, -0.1), (1.0, 0.3)))
    b = None if not bias else rng.standard_normal((1 if bias == "shared" else rows, V)).astype(np.float32)
    words = -(-V // 32)
    m = None if not mask else rng.integers(0, 1 << 32, (1 if mask == "shared" else rows, words), dtype=np.uint64).astype(np.uint32)
    if mask == "row":
        m[rows - 1] = 0
    gamma = 3.5 if guided else None
    xd = x.cuda()
    od = xd if in_place else torch.full((rows, V + gap), 7.0, device="cuda")
    more = {}
    if history:
        more.update(tokens=torch.from_numpy(tok).cuda(), n_tokens=torch.from_numpy(n_tok).cuda(), n_prompt=torch.from_numpy(n_prompt).cuda() if prompt else None)
    if params:
        more.update(repetition=torch.from_numpy(rep).cuda(), presence=torch.from_numpy(pres).cuda(), frequency=torch.from_numpy(freq).cuda(),
                    temperature=torch.from_numpy(temp).cuda())
    if b is not None:
        more.update(bias=torch.from_numpy(b).cuda(), bias_shared=bias == "shared")
    if m is not None:
        more.update(mask=torch.from_numpy(m.view(np.int32)).cuda(), mask_shared=mask == "shared")
    ssd.ssd_logits_process(xd, rows, V, dtype, od, gamma=gamma, logits_stride=V + gap, out_stride=V + gap, **more)
    got = od.cpu().numpy()
    if gap and not in_place:
        assert np.all(got[:, V:] == 7.0)
    for i in range(rows):
        c = x[2 * i if guided else i, :V].float().numpy()
        u = x[2 * i + 1, :V].float().numpy() if guided else None
        allowed = None
        if m is not None:
            w = m[0 if mask == "shared" else i]
            allowed = ((w[np.arange(V) // 32] >> (np.arange(V) % 32).astype(np.uint32)) & 1).astype(bool)
        t = tok[i, :n_tok[i]] if history else []
        r, p, f, te = (float(z[i]) for z in (rep, pres, freq, temp)) if params else (1.0, 0.0, 0.0, 1.0)
        bi = None if b is None else b[0 if bias == "shared" else i]
        want = paged.process_logits(c, u, gamma or 0.0, bi, t, int(n_prompt[i]), r, p, f, te, allowed)
        size = (np.abs(c) + (0 if u is None else gamma * (np.abs(c) + np.abs(u))) + (0 if bi is None else np.abs(bi))) * max(r, 1 / r)
        size = size + len(t) * abs(f) + abs(p)
        g = got[i, :V]
        inf = np.isinf(want)
        assert np.array_equal(g[inf], want[inf].astype(np.float32)), i
        assert np.all(np.abs(g[~inf] - want[~inf]) <= 6e-7 * (1 + size[~inf] / te)), (i, np.abs(g[~inf] - want[~inf]).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("guided", [False, True])
@pytest.mark.parametrize("V", [1, 2, 31, 32, 33, 257, 1000, 8191, 8192, 8193, 20001, 32768])
def test_rows_of_every_size(dtype, guided, V):
    _case(3, V, dtype, guided, "row", "row", 40, V, prompt=9)
    _case(2, V, dtype, guided, None, None, 40, V + 1, gap=5)


@pytest.mark.parametrize("bias", [None, "shared", "row"])
@pytest.mark.parametrize("mask", [None, "shared", "row"])
def test_what_may_be_left_out(bias, mask):
    for history in (0, 7):
        for params in (False, True):
            _case(5, 3001, "f32", False, bias, mask, history, 3, params=params, gap=3)
            _case(4, 4096, "bf16", True, bias, mask, history, 4, params=params)


def test_long_histories():
    _case(3, 40000, "f32", False, None, None, 30000, 5, prompt=5000)
    _case(2, 100, "bf16", False, None, None, 20000, 6, prompt=100)


def test_in_place():
    _case(3, 5000, "f32", False, "shared", "row", 60, 7, in_place=True)
    _case(3, 5001, "f32", False, None, None, 60, 8, in_place=True, gap=2)


def test_more_rows_than_workgroups():
    _case(700, 50, "bf16", True, None, "shared", 5, 9)


def test_large_vocabulary():
    _case(2, 262147, "bf16", True, "shared", "row", 500, 10)


@pytest.mark.parametrize("V", [64, 5000, 30001])
def test_masked_places_hide_whatever_they_hold(V):
    x = torch.randn((2, V), device="cuda")
    x[0, ::3], x[0, 1::3], x[1, ::2] = float("nan"), float("inf"), float("-inf")
    out = torch.zeros((2, V), device="cuda")
    none = torch.zeros((2, -(-V // 32)), dtype=torch.int32, device="cuda")
    ssd.ssd_logits_process(x, 2, V, "f32", out, mask=none)
    assert bool((out == -float("inf")).all())
    # where they are allowed they come through as they are, under every penalty that keeps them
    ssd.ssd_logits_process(x, 2, V, "f32", out, tokens=torch.arange(V, dtype=torch.int32, device="cuda").repeat(2, 1).contiguous(),
                           n_tokens=torch.full((2,), V, dtype=torch.int32, device="cuda"), repetition=torch.full((2,), 1.5, device="cuda"),
                           presence=torch.ones(2, device="cuda"), temperature=torch.full((2,), 0.5, device="cuda"))
    assert bool(torch.isnan(out[0, ::3]).all()) and bool((out[0, 1::3] == float("inf")).all()) and bool((out[1, ::2] == -float("inf")).all())
    assert bool(torch.isfinite(out[1, 1::2]).all())


def test_parameters_that_are_not_above_zero_count_as_one():
    x = torch.randn((4, 300), device="cuda")
    out = torch.zeros_like(x)
    tok = torch.arange(300, dtype=torch.int32, device="cuda").repeat(4, 1).contiguous()
    bad = torch.tensor([0.0, -2.0, float("nan"), 1.0], device="cuda")
    ssd.ssd_logits_process(x, 4, 300, "f32", out, tokens=tok, n_tokens=torch.full((4,), 300, dtype=torch.int32, device="cuda"), repetition=bad, temperature=bad)
    assert torch.equal(out, x)
    # a history whose length is none, and one longer than its places
    ssd.ssd_logits_process(x, 4, 300, "f32", out, tokens=tok[:, :10].contiguous(), n_tokens=torch.tensor([-3, 0, 10, 1 << 30], dtype=torch.int32, device="cuda"),
                           presence=torch.ones(4, device="cuda"))
    want = x.clone()
    want[2:, :10] -= 1.0
    assert torch.equal(out, want)


def test_guided_rows_equal_the_mix():
    p = torch.randn((128, 16384), device="cuda").to(torch.bfloat16)
    a, b = torch.zeros((64, 16384), device="cuda"), torch.zeros((64, 16384), device="cuda")
    ssd.ssd_cfg_mix(p, 128, 16384, "bf16", 5.0, a)
    ssd.ssd_logits_process(p, 64, 16384, "bf16", b, gamma=5.0)
    assert bool(((a - b).abs() <= 2.0 ** -22 * (11 * p.float().abs().amax())).all())


def test_logits_in_a_graph():
    x = torch.zeros((4, 9001), device="cuda")
    out, tok = torch.zeros((2, 9001), device="cuda"), torch.zeros((2, 64), dtype=torch.int32, device="cuda")
    n, one = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.full((2,), 0.7, device="cuda")

    def call(to):
        ssd.ssd_logits_process(x, 2, 9001, "f32", to, gamma=2.0, tokens=tok, n_tokens=n, presence=one, temperature=one)
    call(out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for i in range(5):
        x.copy_(torch.randn_like(x))
        tok.random_(0, 9001)
        n.fill_(10 * i)
        graph.replay()
        torch.cuda.synchronize()
        eager = torch.zeros_like(out)
        call(eager)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
