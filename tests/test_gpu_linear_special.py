"""Special values through the staged kernels of the row-grouped products."""

import pytest
import torch

from paper_2601_13776_amd import orth

from gpu_util import DEV
from test_gpu_linear import rand

pytestmark = pytest.mark.gpu


def tiny(shape, seed):
    """Values of either sign in [1, 2) 2^-118: their second bfloat16 pieces lie
    at the end of its normal range, their third ones past it."""
    g = torch.Generator().manual_seed(seed)
    v = (1 + torch.rand(*shape, generator=g)) * torch.where(torch.rand(*shape, generator=g) < 0.5, -1.0, 1.0)
    return (v * 2.0 ** -118).to(DEV)


def apart(got, ref):
    """Relative 2-norms of the differences, row by row."""
    return torch.linalg.vector_norm(got.double() - ref, dim=1) / torch.linalg.vector_norm(ref, dim=1)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("n_out", [3577, 3584])
def test_tiny_rows_beside_ordinary_ones(n_out, transposed):
    """fp32 rows 2^-118 of the others' size have the precision that they have
    among rows of their own size, application and gradient: that of sums on the
    fp32 MFMA, whose steps of 2 k's round by 2^-24 / sqrt(3) of a partial sum that
    grows as the root of their number n = K / 2.  The squares add up to n^2 / 2 of
    them against n: 2^-24 sqrt(K / 12) of the norm, 1.03e-6 at K = 3577, and half
    as much again for chance.  Without their low pieces they would be 2^-17 off."""
    print(f"[linear tiny rows] {n_out} {transposed}", flush=True)
    k, n = (n_out, 264) if transposed else (264, n_out)
    x, w = rand((2000, k), 1, torch.float32), rand((n_out, 264), 2, torch.float32, 16.0)
    at = [0, 1, 17, 130, 777, 1999]
    small = tiny((2000, k), 3)
    x[at] = small[at]
    y = orth.orth_linear_apply(x, w, transposed=transposed)
    m = w.double() if transposed else w.double().t().contiguous()
    assert torch.all(apart(y, torch.mm(x.double(), m)) <= 1.5 * 2.0 ** -24 * (k / 12) ** 0.5)
    assert torch.equal(y[at], orth.orth_linear_apply(small, w, transposed=transposed)[at])
    # the gradient's rows are the columns of dy
    gy, xs = rand((700, 1100), 4, torch.float32), rand((700, 520), 5, torch.float32)
    gy[:, at[:5]] = tiny((700, 5), 6)
    gw = orth.orth_linear_grad_weight(gy, xs)
    assert torch.all(apart(gw, torch.mm(gy.double().t().contiguous(), xs.double()))
                     <= 1.5 * 2.0 ** -24 * (700 / 12) ** 0.5)


@pytest.mark.parametrize("rows,k,n_out", [(20, 264, 90), (3, 1000, 77), (2000, 264, 3577)])
def test_tiny_rows_of_a_matrix(rows, k, n_out):
    """The same of outputs whose weights are that small beside the others', with
    and without staging."""
    print(f"[linear tiny weights] {rows} {k} {n_out}", flush=True)
    x, w = rand((rows, k), 7, torch.float32, 16.0), rand((n_out, k), 8, torch.float32)
    at = [0, 5, 6, 33, 76]
    w[at] = tiny((5, k), 9)
    y = orth.orth_linear_apply(x, w)
    far = apart(y.t().contiguous(), torch.mm(w.double(), x.double().t()))
    # (norms of a few rows only: twice for chance)
    assert torch.all(far <= 2 * 2.0 ** -24 * (k / 12) ** 0.5), float(far.max())
