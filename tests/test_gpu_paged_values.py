"""GPU: outputs of the paged attention to the bits they are computed with (paged_harness.fine_tolerance), where a row taken from the wrong place shows whatever
the length."""
import importlib.util
import os
import sys

import numpy as np
import pytest
import torch

import paper_2510_18716_amd as ssd
from oracle import paged
from paged_harness import TORCH, Batch, attend, cancelling, check_outputs, fine_tolerance

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("H,n_kv,page", [(8, 2, 16), (3, 3, 7), (16, 1, 64)])
def test_every_row_counts(dtype, d, H, n_kv, page):
    say("fine", dtype, d, H, n_kv, page)
    bt = Batch([2500, 3, 1023, 0, 129, 640, 1, 33], H, n_kv, d, dtype, page, seed=d + H, layout="rows" if page == 7 else "heads")
    check_outputs(bt, attend(bt)[0])
    check_outputs(bt, attend(bt, weights=False)[0])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_probabilities_keep_sixteen_bits(dtype, d):
    say("cancelling", dtype, d)
    bt = cancelling([2, 4, 30, 64, 300, 1400], 4, 2, d, dtype, 5, "cuda")
    check_outputs(bt, attend(bt)[0])


@pytest.mark.parametrize("dtype,d,page", [("bf16", 128, 1), ("bf16", 128, 3), ("bf16", 64, 8), ("f32", 64, 1), ("bf16", 128, 64)])
def test_long_rows_in_pages_of_any_size(dtype, d, page):
    """24 sequences of up to 4096 rows: runs longer than the part of the block table that a workgroup has in LDS."""
    say("long pages", dtype, d, page)
    B, n_kv, G, n = 24, 8, 2, 4096
    g = torch.Generator(device="cuda").manual_seed(page)
    lens = torch.randint(3500, n + 1, (B,), device="cuda", generator=g).to(torch.int32)
    blocks = -(-n // page)
    table = torch.randperm(B * blocks, device="cuda", generator=g).to(torch.int32).reshape(B, blocks)
    k, v = (torch.randn((B * blocks, n_kv, page, d), device="cuda", generator=g).to(TORCH[dtype]) for _ in range(2))
    q = torch.randn((B, G * n_kv, d), device="cuda", generator=g).to(TORCH[dtype])
    cfg = ssd.make_paged_config(B, G * n_kv, n_kv, d, dtype, page, B * blocks, blocks)
    for weights in (False, True):
        out = torch.zeros_like(q)
        w = torch.zeros((B * blocks, n_kv, page), device="cuda") if weights else None
        ws = torch.empty(max(256, ssd.ssd_paged_workspace_bytes(cfg, n, weights)), dtype=torch.uint8, device="cuda")
        ssd.ssd_paged_decode_attn(cfg, q, k, v, table, lens, out, weight_in=w, weight_out=w, max_len=n, workspace=ws)
        for b in range(B):
            m = int(lens[b])
            K, V = (x[table[b].long()].transpose(0, 1).reshape(n_kv, -1, d)[:, :m].double() for x in (k, v))
            for kv in range(n_kv):
                p = torch.softmax(K[kv] @ q[b, G * kv:G * kv + G].double().t() / d ** 0.5, 0)
                ref, size = ((p.t() @ x).cpu().numpy() for x in (V[kv], V[kv].abs()))
                got = out[b, G * kv:G * kv + G].float().cpu().numpy()
                assert np.all(np.abs(got - ref) <= fine_tolerance(dtype, ref, size)), (b, kv)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_serving_example_to_the_bits_it_computes_with(dtype):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_serving.py")
    spec = importlib.util.spec_from_file_location("paged_serving", path)
    example = importlib.util.module_from_spec(spec)
    sys.modules["paged_serving"] = example
    spec.loader.exec_module(example)
    s = example.Settings(prompts=(37, 130, 8), budget=40, slack=12, steps=14, dtype=dtype)
    calls = []

    def watch(layer, st):
        calls.append(layer)
        if len(calls) % 9 != 1:
            return
        k, v, table = st["k"].float().cpu().numpy(), st["v"].float().cpu().numpy(), st["table"].cpu().numpy()
        out, q = st["out"].float().cpu().numpy(), st["q"].float().cpu().numpy().reshape(6, s.heads, s.head_dim)
        for b, n in enumerate(st["lens"]):
            ref, _, _, size = paged.paged_attend(q[b], k, v, table[b], n, s.head_dim ** -0.5)
            assert np.all(np.abs(out[b] - ref) <= fine_tolerance(dtype, ref, size)), (layer, b)

    example.serve(s, watch)
    assert len(calls) == s.steps * s.layers
