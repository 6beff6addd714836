"""GPU: temperatures whose reciprocal is no normal number, against the definition in 64 bits.

Tolerance: at most two roundings to fp32 (of the reciprocal and of the product), 2^-24 each, taken as 1.25e-7 of the result; or the smallest subnormal number."""
import numpy as np
import pytest
import torch

import paper_2510_18716_amd as ssd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_temperatures_at_the_ends_of_the_range(dtype):
    print("temperatures", dtype, flush=True)
    temp = np.array([1e-45, 1e-40, 2e-39, 2.9387359e-39, 2.938736e-39, 1.1754944e-38, 1e-20, 1.0, 1e30, 8.507059e37, 8.50706e37, 2e38, 3.4028235e38], np.float32)
    V = 400
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((len(temp), V)) * 10.0 ** rng.integers(-40, 38, (len(temp), V))).astype(np.float32)
    x[:, :6] = [0.0, -0.0, 1.0, -1.0, np.inf, -np.inf]
    xt = torch.from_numpy(x).to(torch.float32 if dtype == "f32" else torch.bfloat16)
    out = torch.full((len(temp), V), 7.0, device="cuda")
    ssd.ssd_logits_process(xt.cuda(), len(temp), V, dtype, out, temperature=torch.from_numpy(temp).cuda())
    got, exact = out.cpu().numpy(), xt.double().numpy() / temp.astype(np.float64)[:, None]
    with np.errstate(over="ignore"):
        want = exact.astype(np.float32)
    edge = np.abs(exact) > 3.4028e38                            # rounding may take these to either side of the largest number
    for i in range(len(temp)):
        sure = np.isfinite(want[i]) & ~edge[i]
        assert np.all(np.abs(got[i][sure] - exact[i][sure]) <= 1.25e-7 * np.abs(exact[i][sure]) + 2.0 ** -149), (i, temp[i])
        far = np.abs(exact[i]) > 3.41e38
        np.testing.assert_array_equal(got[i][far], want[i][far], err_msg=str(temp[i]))
