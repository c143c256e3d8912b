"""GPU parity of the gradients' global norm and clipping
(orth_grad_norm_batched, orth_grad_clip_batched) with the formula in 64 bits.

Tolerances: squares are summed in fp64 (errors far below fp32's), so the norm
is off by its one rounding to fp32 (2^-24 relative); a clipped value by the
factor's rounding and the product's (2^-24 each) and the rounding to its type
(eps / 2)."""

import pytest
import torch

from paper_2601_13776_amd import orth

from gpu_util import DEV

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def rand(shape, seed, dtype, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).to(DEV)


def norm_of(grads):
    return torch.stack([g.double().square().sum() for g in grads]).sum().sqrt()


def check_clip(grads, outs, norm, max_norm, eps=1e-6):
    ref = norm_of(grads)
    assert abs(float(norm) - float(ref)) <= 2.0 ** -23 * float(ref)
    factor = min(1.0, max_norm / (float(ref) + eps))
    for g, o in zip(grads, outs):
        want = g.double() * factor
        tol = (torch.finfo(g.dtype).eps / 2 + 3 * 2.0 ** -24) * want.abs() + torch.finfo(g.dtype).tiny
        assert torch.all((o.double() - want).abs() <= tol)


LISTS = [
    [((1,), F32)], [((3, 5), BF16)], [((16, 16), F32)] + [((16, 8), F32)] * 4, [((1023,), BF16), ((8193,), F32)],
    [((64, 64), F32), ((7, 3), BF16), ((0, 5), F32), ((0,), BF16), ((2, 3, 4), F32), ((), F32)],
    [((512, 256), F32)] * 56, [((32, 32), BF16)] * 57, [((17, 9), F32), ((33,), BF16)] * 700,
    [((1000, 2048), BF16), ((1,), F32)] + [((31,), F32)] * 70 + [((2048, 2048), BF16)],
    # past what is kept in the caches; a few vectors around the one-launch limit
    [((8192, 4100), F32), ((333,), BF16)], [((16383,), F32)], [((16384,), F32), ((1,), F32)],
]


@pytest.mark.parametrize("case", range(len(LISTS)))
@pytest.mark.parametrize("max_norm", [0.5, 1e6])
def test_clip(case, max_norm):
    print(f"[grad clip] list {case} max_norm {max_norm}", flush=True)
    grads = [rand(s, i, dt) for i, (s, dt) in enumerate(LISTS[case])]
    outs = [torch.full_like(g, 9.0) for g in grads]
    norm = orth.orth_grad_clip_batched(orth.orth_grad_list(grads, outs), max_norm)
    check_clip(grads, outs, norm, max_norm)
    assert torch.equal(orth.orth_grad_norm_batched(grads), norm)
    again = [torch.empty_like(g) for g in grads]
    orth.orth_grad_clip_batched(orth.orth_grad_list(grads, again), max_norm)
    assert all(torch.equal(a, b) for a, b in zip(outs, again))
    # in place, and with a norm that is given
    mine = [g.clone() for g in grads]
    orth.orth_grad_clip_batched(mine, max_norm)
    assert all(torch.equal(a, b) for a, b in zip(outs, mine))
    given = torch.tensor([2 * max_norm], device=DEV)
    orth.orth_grad_clip_batched(orth.orth_grad_list(grads, outs), max_norm, eps=0.0, norm=given, norm_given=True)
    assert float(given) == 2 * max_norm
    for g, o in zip(grads, outs):
        assert torch.equal(o, (g.float() * 0.5).to(g.dtype))


def test_strided_tensors():
    """Column slices (odd offsets and widths), 1-D strides, outputs strided
    another way; nothing beside them is written."""
    print("[grad clip strides]", flush=True)
    a, b, c = rand((50, 100), 1, BF16), rand((70, 33), 2, F32), rand((64, 2), 3, F32)
    grads = [a[:, 3:90], a[:, 91:92], b[:, :31], c[:, 1], b[1:2, 32:33]]
    bufs = [torch.full((50, 130), 5.0, dtype=BF16, device=DEV), torch.full((50, 4), 5.0, dtype=BF16, device=DEV),
            torch.full((70, 31), 5.0, device=DEV), torch.full((64, 3), 5.0, device=DEV),
            torch.full((3, 3), 5.0, device=DEV)]
    outs = [bufs[0][:, 41:128], bufs[1][:, 2:3], bufs[2], bufs[3][:, 0], bufs[4][1:2, 1:2]]
    norm = orth.orth_grad_clip_batched(orth.orth_grad_list(grads, outs), 1.0)
    check_clip(grads, outs, norm, 1.0)
    for buf, o in zip(bufs, outs):
        assert int((buf == 5.0).sum()) >= buf.numel() - o.numel()


def test_extreme_and_non_finite_values():
    print("[grad clip extremes]", flush=True)
    big = [torch.full((300,), 3e38, device=DEV), torch.full((40,), 1e-30, device=DEV)]
    outs = [torch.empty_like(g) for g in big]
    norm = orth.orth_grad_clip_batched(orth.orth_grad_list(big, outs), 1.0)
    assert torch.isinf(norm).all()            # past fp32's range; the factor is not
    assert torch.allclose(outs[0].double(), torch.full((300,), 300 ** -0.5, dtype=torch.float64, device=DEV), rtol=1e-6)
    tiny = [torch.full((256,), 1e-30, device=DEV)]
    assert abs(float(orth.orth_grad_norm_batched(tiny)) / 16e-30 - 1) < 1e-6
    for bad, rest in ((float("nan"), float("nan")), (float("inf"), 0.0)):
        g = [rand((100,), 4, F32), rand((10, 10), 5, BF16)]
        g[0][17] = bad
        outs = [torch.empty_like(t) for t in g]
        norm = orth.orth_grad_clip_batched(orth.orth_grad_list(g, outs), 1.0)
        assert torch.isnan(norm).all() if rest != rest else torch.isinf(norm).all()
        assert torch.isnan(outs[0][17])
        assert torch.all(torch.isnan(outs[1])) if rest != rest else torch.all(outs[1] == 0)
    zero = [torch.zeros(50, device=DEV)]
    assert float(orth.orth_grad_clip_batched(zero, 1.0)) == 0.0 and torch.all(zero[0] == 0)


def test_zero_norm_and_no_epsilon():
    zero = [torch.zeros(50, device=DEV), torch.zeros(3, 7, dtype=BF16, device=DEV)]
    assert float(orth.orth_grad_clip_batched(zero, 0.0, eps=0.0)) == 0.0
    assert all(torch.all(z == 0) for z in zero)


def test_tensor_of_more_than_2_31_values():
    """One tensor past 32 bits beside small ones."""
    print("[grad clip past 2^31]", flush=True)
    n = 2 ** 31 + 4099
    big = torch.zeros(n, dtype=BF16, device=DEV)
    big[:5], big[2 ** 31 - 3:2 ** 31 + 5], big[-3:] = 3.0, -2.0, 1.0
    small = rand((700,), 6, F32)
    out = [torch.full_like(big, 9.0), torch.empty_like(small)]
    norm = orth.orth_grad_clip_batched(orth.orth_grad_list([big, small], out), 1.0)
    ref = (5 * 9.0 + 8 * 4.0 + 3 * 1.0 + float(small.double().square().sum())) ** 0.5
    assert abs(float(norm) / ref - 1) <= 2.0 ** -22
    for sl in (slice(0, 8), slice(2 ** 31 - 8, 2 ** 31 + 8), slice(n - 8, n)):
        want = big[sl].double() / (ref + 1e-6)
        assert torch.all((out[0][sl].double() - want).abs() <= 2.0 ** -8 * 1.01 * want.abs())
    assert int(torch.count_nonzero(out[0])) == 16


def test_captured_clip_and_long_lists():
    """A list that fits the kernel arguments is captured and replayed with
    other gradients; a longer one is refused."""
    print("[grad clip graph]", flush=True)
    grads = [rand((40, 30), i, F32) for i in range(20)]
    lst = orth.orth_grad_list(grads, [torch.empty_like(g) for g in grads])
    many = orth.orth_grad_list([torch.ones(4, device=DEV) for _ in range(57)])
    norm = torch.zeros(1, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        orth.orth_grad_clip_batched(lst, 1.0, norm=norm)
        with pytest.raises(orth.OrthError) as e:
            orth.orth_grad_clip_batched(many, 1.0)
        assert e.value.code == orth.ORTH_EUNSUPPORTED
    for i in range(4):
        for k, g in enumerate(grads):
            g.copy_(rand((40, 30), 100 * i + k, F32))
        graph.replay()
        torch.cuda.synchronize()
        check_clip(grads, lst.tensors[1], norm, 1.0)


@pytest.mark.parametrize("apart", [False, True])
def test_kept_list_follows_its_tensors(apart):
    """A kept list whose tensors got other memory since it was made: replaced
    .data, resized beyond their storage and within it, storage given up."""
    print(f"[grad clip moved] {apart}", flush=True)
    grads = [rand((64, 30), 1, F32), rand((200,), 2, BF16), rand((9, 9), 3, F32)]
    outs = [torch.empty_like(g) for g in grads] if apart else None
    lst = orth.orth_grad_list(grads, outs)
    kept = [g.clone() for g in grads]

    def check():
        before = [g.clone() for g in grads]
        norm = orth.orth_grad_clip_batched(lst, 0.5)
        check_clip(before, outs if apart else grads, norm, 0.5)
        assert torch.equal(orth.orth_grad_norm_batched(before), norm)

    check()
    old = grads[0].data
    grads[0].data = rand((64, 30), 4, F32)
    was = old.clone()
    check()
    assert torch.equal(old, was)               # nothing is written where the tensor was
    grads[1].data = rand((70, 80), 5, BF16)    # another shape
    if apart:
        with pytest.raises(ValueError):
            orth.orth_grad_clip_batched(lst, 0.5)
        with pytest.raises(ValueError):        # (and again: the list is not taken for read)
            orth.orth_grad_norm_batched(lst)
        outs[1].data = torch.empty(70, 80, dtype=BF16, device=DEV)
    check()
    for size in ((300, 300), (2, 3)):          # past the storage, within it
        for t in (grads[2], *(outs[2:] if apart else ())):
            t.resize_(size)
        grads[2].copy_(rand(size, 6, F32))
        if size == (2, 3):
            lst.refresh()                      # (where it was: the list cannot see it)
        check()
    if apart:
        outs[0].data = torch.empty(64, 30, device=DEV)
        check()
    grads[0].untyped_storage().resize_(0)
    with pytest.raises(RuntimeError):
        orth.orth_grad_clip_batched(lst, 0.5)
    grads[0].untyped_storage().resize_(64 * 30 * 4)
    grads[0].copy_(kept[0])
    check()
    slices = [rand((40, 50), 7, F32)[:, 3:20]]   # (an address of 12 is no memory either)
    kept_slices = orth.orth_grad_list(slices)
    slices[0].untyped_storage().resize_(0)
    with pytest.raises(RuntimeError):
        orth.orth_grad_norm_batched(kept_slices)
