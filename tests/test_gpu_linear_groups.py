"""Row-grouped products with very many groups: past what one launch dimension
counts (65535) and up to the largest number taken."""

import pytest
import torch

from paper_2601_13776_amd import orth

from gpu_util import DEV

pytestmark = pytest.mark.gpu


def rand(shape, seed, dtype):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g).to(dtype).to(DEV)


def offsets_of(groups, rows, seed):
    g = torch.Generator().manual_seed(seed)
    cuts = torch.sort(torch.randint(0, rows + 1, (groups - 1,), generator=g))[0]
    return torch.cat([torch.tensor([0]), cuts, torch.tensor([rows])]).to(torch.int32).to(DEV)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_more_groups_than_a_grid_dimension(dtype):
    """70000 small matrices, 5000 rows: rounding alone, after sums in fp32 of
    K products (K 2^-24 of the sum of magnitudes, the split's share with it)."""
    print(f"[linear groups] 70000 {dtype}", flush=True)
    groups, rows, n_in, n_out = 70000, 5000, 16, 8
    offsets = offsets_of(groups, rows, 1)
    group = torch.searchsorted(offsets, torch.arange(rows, device=DEV, dtype=torch.int32), right=True) - 1
    x, w, gy = rand((rows, n_in), 2, dtype), rand((groups, n_out, n_in), 3, dtype), rand((rows, n_out), 4, dtype)
    half = torch.finfo(dtype).eps / 2
    for tr, a, k in ((False, x, n_in), (True, gy, n_out)):
        y = orth.orth_linear_apply(a, w, offsets, transposed=tr)
        m = w[group].double() if not tr else w[group].double().transpose(1, 2).contiguous()
        ref, mag = (m * a.double()[:, None, :]).sum(2), (m * a.double()[:, None, :]).abs().sum(2)
        assert torch.all((y.double() - ref).abs() <= half * ref.abs() + (k + 4) * 2.0 ** -24 * mag)
    gw = orth.orth_linear_grad_weight(gy, x, offsets, dtype=torch.float32)
    ref = torch.zeros(groups, n_out, n_in, dtype=torch.float64, device=DEV)
    outer = gy.double()[:, :, None] * x.double()[:, None, :]
    ref.index_add_(0, group, outer)
    mag = torch.zeros_like(ref).index_add_(0, group, outer.abs())
    most = int((offsets[1:] - offsets[:-1]).max())
    assert torch.all((gw.double() - ref).abs() <= (most + 4) * 2.0 ** -24 * mag)


def test_the_most_groups():
    """2^20 groups of one matrix, most of them empty: the same as one group."""
    print("[linear groups] 2^20", flush=True)
    rows = 100
    x, w = rand((rows, 32), 5, torch.bfloat16), rand((24, 32), 6, torch.bfloat16)
    offsets = offsets_of(2 ** 20, rows, 7)
    y = orth.orth_linear_apply(x, w.expand(2 ** 20, 24, 32), offsets)
    assert torch.equal(y, orth.orth_linear_apply(x, w))
