"""CPU: the fine check of attention outputs (paged_harness.check_outputs) passes what the kernels compute and fails what they must not.  The outputs are made
here: probabilities in two bf16 terms, sums in 64 bits, one rounding to bf16.  The mistakes are planted in that copy."""
import numpy as np
import pytest
import torch

from oracle import paged
from paged_harness import Batch, cancelling, check_outputs


def made(bt, terms=2, taken=None):
    """taken: {row: the row whose V is taken instead} of sequence 0."""
    out = torch.zeros((len(bt.lens), bt.H, bt.d), dtype=torch.float64)
    G = bt.H // bt.n_kv
    for b, n in enumerate(bt.lens):
        if n == 0:
            continue
        for h in range(bt.H):
            K, _ = paged.rows_of(bt.k.float().numpy(), bt.table[b], n, bt.page, h // G)
            V, _ = paged.rows_of(bt.v.float().numpy(), bt.table[b], n, bt.page, h // G)
            if taken and b == 0:
                for to, at in taken.items():
                    V[to] = V[at]
            z = K @ bt.q[b, h].double().numpy() * bt.d ** -0.5
            p = torch.from_numpy(np.exp(z - z.max())).float()
            first = (p * (1 - 2.0 ** -8) if terms == 2 else p).to(torch.bfloat16).float()
            used = first.double() + ((p - first).to(torch.bfloat16).double() if terms == 2 else 0.0)
            out[b, h] = (used @ torch.from_numpy(V)) / p.double().sum()
    return out.to(torch.bfloat16)


def test_outputs_as_they_are_computed_pass():
    for bt in (Batch([2000, 33, 1, 0], 4, 2, 64, "bf16", 16, seed=1, device="cpu"), cancelling([2, 4, 30], 2, 2, 64, "bf16", 2, "cpu")):
        check_outputs(bt, made(bt))


@pytest.mark.parametrize("to,at", [(3, 4), (777, 1200), (1999, 0), (1024, 1023)])
def test_one_exchanged_row_of_two_thousand_fails(to, at):
    bt = Batch([2000], 4, 2, 64, "bf16", 16, seed=1, device="cpu")
    with pytest.raises(AssertionError):
        check_outputs(bt, made(bt, taken={to: at}))


def test_probabilities_of_eight_bits_fail():
    for n in (2, 4, 30):
        bt = cancelling([n], 2, 2, 64, "bf16", 2, "cpu")
        with pytest.raises(AssertionError):
            check_outputs(bt, made(bt, terms=1))
