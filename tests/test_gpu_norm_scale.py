"""mxq_rmsnorm of rows whose squares FP32 does not hold: from the smallest subnormal to the largest finite numbers, with eps = 0, with an eps that
covers the row and with one of the row's own size."""
import numpy as np
import pytest
import torch

import paper_2503_13565_b200 as mxq
import step_plain as plain
from test_gpu_norm import Y_REL, check_pair, near

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
SIZES = [1e-45, 1e-42, 1e-38, 1e-30, 1e-25, 1e-21, 1e-19, 3e-16, 7e-16, 1e-8, 1.0, 1e10, 1e17, 6e18, 1.7e19, 1e20, 1e30, 1e37]


@pytest.mark.parametrize("eps", [0.0, 1e-45, 1e-40, 1e-36, 1e-31, 7.8e-31, 8e-31, 1e-12, 1e-5, 1e30, 3e38])
@pytest.mark.parametrize("k,x,w", [(32, F32, F32), (96, BF16, F32), (4096, F32, BF16), (4096, BF16, BF16), (8224, F32, F32), (32768, BF16, F32)])
def test_rows_of_every_size(k, x, w, eps):
    eps = float(np.float32(eps))
    g = torch.Generator(device="cuda").manual_seed(k)
    rows = torch.randn(len(SIZES), k, generator=g, device="cuda").clamp(-30, 30).double() * torch.tensor(SIZES, device="cuda", dtype=torch.float64).unsqueeze(1)
    rows = rows.float().to(x)
    weight = (1 + 0.3 * torch.randn(k, generator=g, device="cuda")).to(w)
    y, codes, scales = mxq.mxq_rmsnorm(rows, weight, eps, mxfp8=True)
    h, want = plain.rmsnorm(rows, None, weight, eps)
    some = (h != 0).any(1) if eps == 0 else torch.ones(len(SIZES), dtype=torch.bool, device="cuda")        # (zero by zero is no number)
    near(y[some], want[some], 2.0 ** -8 + 2 * Y_REL, 2.0 ** -134)
    normal = some & (want.abs().amax(1) > 1e-30)
    check_pair(codes[normal], scales[normal], want[normal])
    assert bool(y[~some].isnan().all()) and bool((scales[~some] == 255).all())
    # a row's neighbours do not matter
    for i in (0, 4, 10, 17):
        assert torch.equal(mxq.mxq_rmsnorm(rows[i:i + 1], weight, eps).view(torch.int16), y[i:i + 1].view(torch.int16))


@pytest.mark.parametrize("size", [1e-25, 1e20])
def test_the_residual_s_sum_is_not_in_other_units(size):
    m, k = 5, 768
    g = torch.Generator(device="cuda").manual_seed(1)
    x, r = ((torch.randn(m, k, generator=g, device="cuda") * size) for _ in range(2))
    total, weight = torch.empty_like(r), torch.ones(k, device="cuda")
    y = mxq.mxq_rmsnorm(x, weight, 0.0, residual=r, residual_out=total)
    assert torch.equal(total, x + r)
    near(y, plain.rmsnorm(total, None, weight, 0.0)[1], 2.0 ** -8 + 2 * Y_REL)


def test_one_large_element_and_an_infinite_one():
    x = torch.zeros(3, 256, device="cuda")
    x[0, 9], x[1, 9], x[2, 9] = 3e38, 1e-45, float("inf")
    x[2, 10] = 3e38
    y = mxq.mxq_rmsnorm(x, torch.ones(256, device="cuda"), 0.0).float()
    assert y[0, 9] == 16 and y[1, 9] == 16 and bool((y[:2].sum(1) == 16).all())        # h / sqrt(h^2 / 256)
    assert bool(y[2, 9].isnan()) and float(y[2, 10]) == 0 and bool((y[2, :9] == 0).all())
