"""Precision of the classification head's bf16 gradients (orth_linear_xent_vjp):
dz is held in 16 bits or more, so that a gradient is off by its own rounding
and little else, whatever values grad_loss takes.

Tolerance: that of test_gpu_xent.py with dz off by 2^-16 of its value where one
rounding to bfloat16 would be off by 2^-8.  By arithmetic: bfloat16 has 8
significant bits, so neighbours of a value in [1, 2) are 2^-7 = finfo.eps apart
and a rounding is off by up to half of that, 2^-8 of the value; the second of
two pieces holds that remainder, at most 2^-8, and its rounding is off by 2^-8
of it, 2^-16.  Its products are 2 k sums."""

import pytest
import torch

from paper_2601_13776_amd import orth

from gpu_util import DEV
from test_gpu_xent import definition, rand, targets_of

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
HALF = torch.finfo(BF16).eps / 2   # a rounding's share: 2^-8

CASES = [  # rows, features, classes, scale, classes per piece
    # few rows (the kernels without staging), one and several pieces
    (1, 64, 40, 1.0, 0), (7, 200, 3001, 2.0, 0), (16, 856, 16537, 1.0, 0), (30, 130, 2000, 1.0, 700),
    # staged tiles of both edges, aligned and not; dx in slices; dW in slices
    (200, 328, 5003, 2.0, 0), (300, 99, 1500, 1.0, 0), (700, 264, 4000, 1.0, 1504), (2048, 136, 8000, 2.0, 0),
    (1000, 1344, 20001, 2.0, 8192), (6000, 100, 300, 1.0, 0), (4096, 512, 9000, 1.0, 0),
    # dx on 256-tiles, the last one half full: stored, summed over pieces
    (4020, 2048, 3001, 1.0, 0), (4020, 2048, 7003, 1.0, 3000),
]


def grad_losses(rows, seed):
    """Weights of a few kinds of rows, each halfway between two bfloat16
    values, and some rows of very small and of zero weight."""
    g = torch.Generator().manual_seed(seed)
    kinds = torch.tensor([1 + 2.0 ** -8, 3 * (1 + 3 * 2.0 ** -8), -0.3, 1.0 / 3, 2.0 ** -70, 0.0])
    return kinds[torch.randint(0, len(kinds), (rows,), generator=g)].to(DEV)


@pytest.mark.parametrize("case", range(len(CASES)))
def test_gradients_are_off_by_their_own_rounding(case):
    rows, d, classes, scale, piece = CASES[case]
    print(f"[xent precision] {CASES[case]}", flush=True)
    x, w = rand((rows, d), 1, BF16), rand((classes, d), 2, BF16, d ** -0.5)
    t, gl = targets_of(rows, classes, 3), grad_losses(rows, 4)
    lse = orth.orth_linear_xent(x, w, t, scale=scale)[1]
    gx, gw = orth.orth_linear_xent_vjp(x, w, t, lse, gl, scale=scale, piece=piece)
    _, r_lse, dz, size, _ = definition(x, w, t, scale, gl)
    zmax = abs(scale) * torch.mm(x.double().abs(), w.double().abs().t()).amax(1)
    e = (d + 4) * 2.0 ** -24 * zmax + 2.0 ** -23 * zmax
    tol = 2 * e + (classes + 20) * 2.0 ** -24 + 2.0 ** -23 * r_lse.abs()
    off = (torch.expm1(e + tol)[:, None] + 4 * 2.0 ** -23) * size + 2.0 ** -16 * dz.abs()
    for got, ref, mag, slack, k in (
            (gx, torch.mm(dz, w.double()), torch.mm(size, w.double().abs()), torch.mm(off, w.double().abs()), classes),
            (gw, torch.mm(dz.t(), x.double()), torch.mm(size.t(), x.double().abs()),
             torch.mm(off.t(), x.double().abs()), rows)):
        bound = HALF * ref.abs() + (2 * k + 8) * 2.0 ** -24 * mag + slack * (1 + HALF) + 1e-37
        err = (got.double() - ref).abs()
        assert torch.all(err <= bound * 1.001), f"off by {float((err / bound).max()):.3g} bounds"


@pytest.mark.parametrize("rows,d,classes", [(20, 96, 700), (900, 264, 3000)])
def test_rows_do_not_depend_on_each_others_grad_loss(rows, d, classes):
    print(f"[xent rows apart] {rows}", flush=True)
    x, w = rand((rows, d), 5, BF16), rand((classes, d), 6, BF16, d ** -0.5)
    t, gl = targets_of(rows, classes, 7, ignored=0.0), torch.full((rows,), 0.37, device=DEV)
    lse = orth.orth_linear_xent(x, w, t)[1]
    before = orth.orth_linear_xent_vjp(x, w, t, lse, gl, want=(True, False))[0]
    gl[0], gl[3] = 1.9, -1e-3
    after = orth.orth_linear_xent_vjp(x, w, t, lse, gl, want=(True, False))[0]
    same = [r for r in range(rows) if r not in (0, 3)]
    assert torch.equal(before[same], after[same])


def test_infinite_and_overflowing_grad_loss():
    """An infinite weight makes its row's gradient infinite where the formula
    does: dW of a class is inf x, never inf - inf of two pieces."""
    print("[xent infinite weight]", flush=True)
    x, w = rand((3, 64), 8, BF16).abs() + 0.5, rand((50, 64), 9, BF16, 0.125)
    t = torch.tensor([4, 7, 9], device=DEV)
    gl = torch.tensor([1.0, float("inf"), 1.0], device=DEV)
    lse = orth.orth_linear_xent(x, w, t)[1]
    gw = orth.orth_linear_xent_vjp(x, w, t, lse, gl, want=(False, True))[1]
    assert torch.all(gw[7] == -float("inf"))
    rest = [c for c in range(50) if c != 7]
    assert torch.all(gw[rest] == float("inf"))
