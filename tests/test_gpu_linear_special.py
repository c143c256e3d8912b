"""Special values through the staged kernels of the row-grouped products and
the head's loss: rows of NaN, infinity and of very small values beside ordinary
ones, rows without a target, malformed offsets.  (The small sizes of
test_gpu_linear.py and test_gpu_xent.py are computed without staging.)

Tolerances as there: half a step of the output's type and (K + 4) 2^-24 of the sum
of magnitudes, with nothing added but a step of the smallest numbers (2^-149 per
product), so that tiny rows are held to their own size.  Rows beside special ones
are held to be the same, bit for bit, as without them."""

import pytest
import torch

from paper_2601_13776_amd import orth

from gpu_util import DEV
from test_gpu_linear import DT, bounds_of, rand
from test_gpu_xent import definition, targets_of

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def check(got, ref, mag, k, dtype):
    err = (got.double() - ref).abs()
    bound = torch.finfo(dtype).eps / 2 * ref.abs() + (k + 4) * 2.0 ** -24 * mag + k * 2.0 ** -149
    assert torch.all(err <= bound * 1.001), f"off by {float((err / bound).max()):.3g} bounds"


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


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_special_rows_of_an_application(dtype):
    print(f"[linear special rows] {dtype}", flush=True)
    dt = DT[dtype]
    for counts, n_in, n_out in (([2000], 264, 3577), ([1100, 700, 200], 320, 3584)):
        bounds, offsets = bounds_of(counts)
        x, w = rand((2000, n_in), 5, dt), rand((len(counts), n_out, n_in), 6, dt)
        gy = rand((2000, n_out), 7, dt)
        plain = orth.orth_linear_apply(x, w, offsets)
        plain_t = orth.orth_linear_apply(gy, w, offsets, transposed=True)
        at = [3, 128, 1000, 1999]
        rest = [r for r in range(2000) if r not in at]
        x[3, 5], x[128, 7], x[1000], x[1999] = NAN, INF, 0.0, -INF
        gy[3, 5], gy[128, 7], gy[1000], gy[1999] = NAN, INF, 0.0, -INF
        for a, tr, want in ((x, False, plain), (gy, True, plain_t)):
            y = orth.orth_linear_apply(a, w, offsets, transposed=tr)
            assert torch.equal(y[rest], want[rest])
            assert torch.all(torch.isnan(y[3])) and torch.all(y[1000] == 0)
            for r in (128, 1999):
                g = max(i for i, b in enumerate(bounds[:-1]) if b <= r)
                m = w[g].double() if tr else w[g].double().t().contiguous()
                ref = torch.mv(m.t().contiguous(), a[r].double())
                assert torch.equal(torch.isnan(y[r]), torch.isnan(ref))
                assert torch.equal(y[r][torch.isinf(ref)].double(), ref[torch.isinf(ref)])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_special_columns_of_a_gradient(dtype):
    """A NaN in dy reaches its row of dW only, one in x its column, and those of
    one group not the next."""
    print(f"[linear special gradient] {dtype}", flush=True)
    dt = DT[dtype]
    bounds, offsets = bounds_of([900, 800, 0, 700])
    x, gy = rand((2400, 520), 8, dt), rand((2400, 1032), 9, dt)
    plain = orth.orth_linear_grad_weight(gy, x, offsets, dtype=torch.float32)
    gy[1000, 77], x[1650, 301] = NAN, INF
    gw = orth.orth_linear_grad_weight(gy, x, offsets, dtype=torch.float32)
    for g in (0, 2, 3):
        assert torch.equal(gw[g], plain[g])
    rows, cols = [r for r in range(1032) if r != 77], [c for c in range(520) if c != 301]
    assert torch.all(torch.isnan(gw[1, 77])) and not torch.isfinite(gw[1, :, 301]).any()
    assert torch.equal(gw[1][rows][:, cols], plain[1][rows][:, cols])


def ranges(offsets, rows):
    """The ranges that offsets stand for: each clamped to [0, rows] and to the
    largest before it."""
    out, top = [], 0
    at = [min(max(o, 0), rows) for o in offsets]
    for a, b in zip(at[:-1], at[1:]):
        top = max(top, a)
        out.append((top, max(top, b)))
        top = out[-1][1]
    return out


def malformed(kind):
    g = torch.Generator().manual_seed(11)
    if kind == "few":       # decreasing, negative, too large
        return [-5, 900, 300, 1700, 100000], 2300
    if kind == "all behind":
        return [2 ** 31 - 1, -2 ** 31, 5, 2300, 7], 2300
    at = torch.randint(-2000, 16000, (101,), generator=g)      # 100 groups, mostly disordered
    at[::3] = torch.sort(torch.randint(0, 12000, (len(at[::3]),), generator=g))[0]
    return at.tolist(), 12000


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["few", "all behind", "many"])
def test_malformed_offsets(kind, dtype):
    at, rows = malformed(kind)
    print(f"[linear malformed offsets] {kind} {dtype}", flush=True)
    dt, n_in, n_out = DT[dtype], 136, 264
    groups = len(at) - 1
    offsets = torch.tensor(at, dtype=torch.int64).to(torch.int32).to(DEV)
    x, w, gy = rand((rows, n_in), 12, dt), rand((groups, n_out, n_in), 13, dt), rand((rows, n_out), 14, dt)
    for a, tr, n, k in ((x, False, n_out, n_in), (gy, True, n_in, n_out)):
        out = torch.full((rows, n), 7.0, dtype=dt, device=DEV)
        orth.orth_linear_apply(a, w, offsets, transposed=tr, out=out)
        seen = torch.zeros(rows, dtype=torch.bool, device=DEV)
        for g, (b, e) in enumerate(ranges(at, rows)):
            m = w[g].double() if tr else w[g].double().t().contiguous()
            check(out[b:e], torch.mm(a[b:e].double(), m), torch.mm(a[b:e].double().abs(), m.abs()), k, dt)
            assert not seen[b:e].any()
            seen[b:e] = True
        assert torch.all(out[~seen] == 7.0)
    gw = orth.orth_linear_grad_weight(gy, x, offsets, dtype=torch.float32)
    for g, (b, e) in enumerate(ranges(at, rows)):
        m = gy[b:e].double().t().contiguous()
        check(gw[g], torch.mm(m, x[b:e].double()), torch.mm(m.abs(), x[b:e].double().abs()), max(e - b, 1), torch.float32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("features", [264, 261])
def test_rows_without_a_target_that_hold_anything(features, dtype):
    """NaN, infinities and the largest values in rows without a target, of x and
    of grad_loss, through the staged loss, dz and both gradients."""
    print(f"[xent special rows] {features} {dtype}", flush=True)
    dt = DT[dtype]
    x, w = rand((700, features), 15, dt), rand((4001, features), 16, dt, features ** -0.5)
    t, gl = targets_of(700, 4001, 17), rand((700,), 18, torch.float32)
    free = torch.nonzero((t < 0) | (t >= 4001))[:, 0]
    rest = torch.nonzero((t >= 0) & (t < 4001))[:, 0]
    loss, lse = orth.orth_linear_xent(x, w, t)
    clean = orth.orth_linear_xent_vjp(x, w, t, lse, gl, piece=1504)
    x[free[0]], x[free[1], 3], x[free[2]], gl[free[3]] = NAN, INF, torch.finfo(dt).max, NAN
    loss2, lse2 = orth.orth_linear_xent(x, w, t)
    assert torch.equal(loss2, loss) and torch.equal(lse2[rest], lse[rest])
    gx, gw = orth.orth_linear_xent_vjp(x, w, t, lse2, gl, piece=1504)
    assert torch.equal(gx, clean[0]) and torch.equal(gw, clean[1])
    assert torch.all(gx[free] == 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_classes_of_no_weight(dtype):
    """Classes whose logits are -inf in every row (masked by their weights),
    whole column tiles of them among them, and logits of +-1e4."""
    print(f"[xent masked classes] {dtype}", flush=True)
    dt = DT[dtype]
    x, w = rand((600, 128), 19, dt).abs() + 0.25, rand((3000, 128), 20, dt, 0.05)
    off = torch.zeros(3000, dtype=torch.bool, device=DEV)
    off[256:1024], off[5], off[2999] = True, True, True
    w[off] = -INF
    w[7], w[9] = 80.0, -80.0
    t = targets_of(600, 3000, 21)
    t[off[t.clamp(0, 2999)]] = 7
    t[0], t[1] = 7, 2
    loss, lse = orth.orth_linear_xent(x, w, t)
    keep = torch.nonzero(~off)[:, 0]
    where = torch.full((3001,), -1, device=DEV)
    where[keep] = torch.arange(len(keep), device=DEV)
    t2 = where[torch.where((t < 0) | (t >= 3000), 3000, t)]
    r_loss, r_lse, _, _, z = definition(x, w[keep], t2, 1.0, torch.ones(600, device=DEV))
    # a logit's error and the result's rounding, both of the largest logit
    tol = (128 + 20) * 2.0 ** -23 * z.abs().amax(1)
    assert torch.all((lse.double() - r_lse).abs() <= tol) and torch.all((loss.double() - r_loss).abs() <= tol)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,features,classes", [(5, 64, 300), (6, 128, 70000), (700, 264, 4001)])
def test_infinite_logits(rows, features, classes, dtype):
    """lse of a row with a logit of +inf is +inf, of -inf ones and +inf ones too;
    all of -inf give -inf, and one NaN gives NaN.  The other rows are as without."""
    print(f"[xent infinite logits] {rows} {features} {classes} {dtype}", flush=True)
    dt = DT[dtype]
    x, w = rand((rows, features), 29, dt), rand((classes, features), 30, dt, features ** -0.5)
    w[:, 0] = w[:, 0].abs() + 2.0 ** -9
    plain = orth.orth_linear_xent(x, w, torch.full((rows,), 3, device=DEV))
    x[0, 0], x[1, 0], x[2, 1], x[3, 0], x[3, 1] = INF, -INF, INF, INF, NAN
    t = torch.full((rows,), 3, device=DEV)
    loss, lse = orth.orth_linear_xent(x, w, t)
    z = torch.mm(x.double(), w.double().t().contiguous())
    want = torch.logsumexp(z, 1)
    assert want[0] == INF and want[1] == -INF and want[2] == INF and torch.isnan(want[3])
    assert torch.equal(lse[:3].double(), want[:3]) and torch.isnan(lse[3])
    assert torch.isnan(loss[0]) and torch.isnan(loss[1]) and torch.isnan(loss[3])       # inf - inf
    assert loss[2] == INF if z[2, 3] == -INF else torch.isnan(loss[2])
    assert torch.equal(lse[4:], plain[1][4:]) and torch.equal(loss[4:], plain[0][4:])


@pytest.mark.parametrize("counts,n_in,n_out", [([2000, 100, 1500], 264, 3577), ([4096], 256, 4096), ([200, 0, 30, 9] * 60, 64, 136),
                                               ([700], 1000, 90), ([64] * 20, 90, 256)])
def test_fp32_products_keep_24_bits(counts, n_in, n_out):
    """The relative 2-norm error of fp32 products.  A step of 16 k's is rounded
    once, by 2^-24 / sqrt(3) of a partial sum that grows as the root of its
    steps: 2^-24 sqrt(K / 96) in all, 3.9e-7 at K = 4096, and with the products'
    own 2^-24 / sqrt(3) and the result's below 5e-7.  A middle piece is 2^-9 of
    its value or so (2^-8 at most, uniform) and a low one 2^-18, so that one of
    the six products left out costs 2.4e-6 and more."""
    print(f"[linear 24 bits] {len(counts)} {n_in}->{n_out}", flush=True)
    bounds, offsets = bounds_of(counts)
    x, w = rand((bounds[-1], n_in), 22, torch.float32), rand((len(counts), n_out, n_in), 23, torch.float32)
    gy = rand((bounds[-1], n_out), 24, torch.float32)
    y = orth.orth_linear_apply(x, w, offsets)
    gx = orth.orth_linear_apply(gy, w, offsets, transposed=True)
    gw = orth.orth_linear_grad_weight(gy, x, offsets)
    ry, rx, rw = torch.empty_like(y, dtype=torch.float64), torch.empty_like(gx, dtype=torch.float64), torch.zeros_like(gw, dtype=torch.float64)
    for g, (a, b) in enumerate(zip(bounds[:-1], bounds[1:])):
        ry[a:b] = torch.mm(x[a:b].double(), w[g].double().t())
        rx[a:b] = torch.mm(gy[a:b].double(), w[g].double())
        rw[g] = torch.mm(gy[a:b].double().t(), x[a:b].double())
    for got, ref in ((y, ry), (gx, rx), (gw, rw)):
        rel = float(torch.linalg.vector_norm(got.double() - ref) / torch.linalg.vector_norm(ref))
        assert rel <= 5e-7, rel


@pytest.mark.parametrize("rows,d,classes", [(9, 200, 2011), (200, 264, 520), (700, 1000, 3001)])
def test_fp32_head_gradients_keep_24_bits(rows, d, classes):
    """As above: products within 5e-7, and dz's exponentials off by the logits'
    errors (below 3e-7 absolute here, with |z| < 8) and their own 2^-22."""
    print(f"[xent 24 bits] {rows} {d} {classes}", flush=True)
    x, w = rand((rows, d), 25, torch.float32), rand((classes, d), 26, torch.float32, d ** -0.5)
    t, gl = targets_of(rows, classes, 27), rand((rows,), 28, torch.float32)
    lse = orth.orth_linear_xent(x, w, t)[1]
    gx, gw = orth.orth_linear_xent_vjp(x, w, t, lse, gl)
    dz = definition(x, w, t, 1.0, gl)[2]
    for got, ref in ((gx, torch.mm(dz, w.double())), (gw, torch.mm(dz.t(), x.double()))):
        rel = float(torch.linalg.vector_norm(got.double() - ref) / torch.linalg.vector_norm(ref))
        assert rel <= 1.2e-6, rel
