"""What the row-grouped products, the head's loss and the gradient clipping
refuse, and the sizes of their workspaces: host checks that run before
anything is enqueued.  No compute call is made here (pointers are made up)."""

import ctypes
import math
import os

import pytest
import torch

from paper_2601_13776_amd import orth

OK, EINVAL, EWORKSPACE = orth.ORTH_OK, orth.ORTH_EINVAL, orth.ORTH_EWORKSPACE
BIG = 2 ** 31 - 1


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(orth._LIB_PATH):
        from paper_2601_13776_amd import build
        build.build(verbose=False)
    return orth.lib()


def linear(**kw):
    f = dict(x=1 << 40, w=2 << 40, y=3 << 40, offsets=4 << 40, rows=100, groups=4, in_features=64, out_features=32,
             ld_x=64, ld_w=64, stride_w=2048, ld_y=32, dtype=1, grad_dtype=0, transposed=0)
    f.update(kw)
    return orth.orth_linear_args(**f)


LINEAR = [dict(x=None), dict(w=None), dict(y=None), dict(offsets=None), dict(rows=-1), dict(rows=BIG), dict(groups=0),
          dict(in_features=0), dict(out_features=0), dict(in_features=BIG, ld_x=BIG, ld_w=BIG), dict(ld_x=63),
          dict(ld_w=63), dict(ld_y=31), dict(stride_w=2047), dict(ld_x=2 ** 60), dict(ld_y=2 ** 44), dict(ld_w=2 ** 50, stride_w=2 ** 60),
          dict(stride_w=2 ** 60), dict(dtype=2), dict(dtype=-1), dict(grad_dtype=2)]


@pytest.mark.parametrize("kw", LINEAR + [dict(transposed=2), dict(transposed=1), dict(y=1 << 40), dict(y=2 << 40),
                                         dict(y=(2 << 40) + 4 * 2048 * 2 - 2)])
def test_apply_refusals(L, kw):
    # (transposed: ld_x and ld_y now bound the other sizes, ld_y = 32 < 64)
    assert L.orth_linear_apply(ctypes.byref(linear(**kw)), None) == EINVAL
    assert L.orth_last_error()


def test_apply_null_and_nothing_to_do(L):
    assert L.orth_linear_apply(None, None) == EINVAL
    assert L.orth_linear_apply(ctypes.byref(linear(rows=0, x=None, y=None)), None) == OK


@pytest.mark.parametrize("kw", LINEAR + [dict(w=1 << 40), dict(w=(3 << 40) + 10)])
def test_grad_weight_refusals(L, kw):
    assert L.orth_linear_grad_weight(ctypes.byref(linear(**kw)), 1 << 50, 1 << 40, None) == EINVAL


def test_grad_weight_workspace(L):
    n = ctypes.c_size_t(7)
    assert L.orth_linear_grad_weight_workspace_size(ctypes.byref(linear()), None) == EINVAL
    assert L.orth_linear_grad_weight_workspace_size(ctypes.byref(linear()), ctypes.byref(n)) == OK


def xent(**kw):
    f = dict(x=1 << 40, w=2 << 40, targets=4 << 40, rows=100, features=64, classes=1000, ld_x=64, ld_w=64, scale=1.0,
             dtype=1, piece=0)
    f.update(kw)
    return orth.orth_linear_xent_args(**f)


XENT = [dict(x=None), dict(w=None), dict(targets=None), dict(rows=-1), dict(rows=BIG), dict(features=0),
        dict(classes=0), dict(classes=BIG), dict(ld_x=63), dict(ld_w=63), dict(ld_x=2 ** 60), dict(ld_w=2 ** 40), dict(scale=math.inf), dict(scale=math.nan),
        dict(dtype=2), dict(piece=-1)]


@pytest.mark.parametrize("kw", XENT)
def test_xent_refusals(L, kw):
    n = ctypes.c_size_t()
    a = ctypes.byref(xent(**kw))
    assert L.orth_linear_xent_workspace_size(a, ctypes.byref(n)) == EINVAL
    assert L.orth_linear_xent_vjp_workspace_size(a, ctypes.byref(n)) == EINVAL
    assert L.orth_linear_xent(a, 1 << 45, 2 << 45, 1 << 50, 1 << 40, None) == EINVAL
    assert L.orth_linear_xent_vjp(a, 1 << 45, 2 << 45, 5 << 45, 64, 6 << 45, 64, 1 << 50, 1 << 40, None) == EINVAL


def test_xent_pointers_and_workspace(L):
    a = ctypes.byref(xent())
    n, m = ctypes.c_size_t(), ctypes.c_size_t()
    assert L.orth_linear_xent_workspace_size(a, ctypes.byref(n)) == OK
    assert L.orth_linear_xent_vjp_workspace_size(a, ctypes.byref(m)) == OK
    # no logits: far below rows x classes for the loss, one piece of dz for
    # the gradients
    assert 0 < n.value < 100 * 1000 * 2 and m.value >= 100 * 1000 * 2
    few = ctypes.c_size_t()
    assert L.orth_linear_xent_vjp_workspace_size(ctypes.byref(xent(rows=4096, classes=131072, piece=1000)),
                                                 ctypes.byref(few)) == OK
    # dz, the rows, dx's sum, and where dW's few tiles take the rows in slices
    # the sums of at most 512 tiles and one row of tiles more
    assert few.value < 4096 * (1000 * 2 + 64 * 2 + 64 * 4) + (512 + 8) * 128 * 128 * 4 + 4096
    assert L.orth_linear_xent(a, None, 2 << 45, 1 << 50, n.value, None) == EINVAL
    for loss, lse in ((2 << 45, 2 << 45), ((2 << 45) + 396, 2 << 45), ((1 << 40) + 100, 2 << 45), (1 << 45, 2 << 40),
                      ((4 << 40) + 796, 2 << 45)):
        assert L.orth_linear_xent(a, loss, lse, 1 << 50, n.value, None) == EINVAL
    assert L.orth_linear_xent(a, 1 << 45, 2 << 45, None, 0, None) == EWORKSPACE
    assert L.orth_linear_xent(a, 1 << 45, 2 << 45, (1 << 50) + 16, n.value, None) == EWORKSPACE
    assert L.orth_linear_xent(a, 1 << 45, 2 << 45, 1 << 50, n.value - 1, None) == EWORKSPACE

    def vjp(lse=1 << 45, gl=2 << 45, gx=5 << 45, lx=64, gw=6 << 45, lw=64, ws=1 << 50, nb=m.value):
        return L.orth_linear_xent_vjp(a, lse, gl, gx, lx, gw, lw, ws, nb, None)

    assert vjp(lse=None) == EINVAL and vjp(gl=None) == EINVAL and vjp(gx=None, gw=None) == EINVAL
    assert vjp(lx=63) == EINVAL and vjp(lw=63) == EINVAL
    assert vjp(lx=2 ** 60) == EINVAL and vjp(lw=2 ** 50) == EINVAL
    assert vjp(gx=(1 << 45) + 396) == EINVAL and vjp(gw=2 << 45) == EINVAL and vjp(gx=4 << 40) == EINVAL
    assert vjp(gx=1 << 40) == EINVAL and vjp(gw=2 << 40) == EINVAL and vjp(gx=6 << 45) == EINVAL
    assert vjp(ws=None) == EWORKSPACE and vjp(ws=(1 << 50) + 1) == EWORKSPACE and vjp(nb=m.value - 1) == EWORKSPACE
    assert L.orth_linear_xent(ctypes.byref(xent(rows=0, x=None, targets=None)), None, None, None, 0, None) == OK


def grads(n=3, **kw):
    arr = (orth.orth_grad * n)()
    for i in range(n):
        f = dict(grad=(1 << 40) + (i << 30), out=(2 << 40) + (i << 30), rows=4, cols=8, ld_grad=8, ld_out=8, dtype=0)
        if i == n - 1:
            f.update(kw)
        arr[i] = orth.orth_grad(**f)
    return arr


@pytest.mark.parametrize("kw", [dict(grad=None), dict(out=None), dict(rows=-1), dict(cols=-1), dict(ld_grad=7),
                                dict(ld_out=7), dict(dtype=2), dict(out=2 << 40),
                                dict(out=(1 << 40) + (2 << 30), ld_out=9)])
def test_clip_refusals(L, kw):
    o = orth.orth_clip_opts(1.0, 1e-6, 0)
    assert L.orth_grad_clip_batched(grads(**kw), 3, ctypes.byref(o), 1 << 45, 1 << 50, 1 << 30, None) == EINVAL


@pytest.mark.parametrize("o", [(-1.0, 0.0, 0), (math.nan, 0.0, 0), (math.inf, 0.0, 0), (1.0, -1.0, 0),
                               (1.0, math.nan, 0), (1.0, 0.0, 2)])
def test_clip_option_refusals(L, o):
    assert L.orth_grad_clip_batched(grads(), 3, ctypes.byref(orth.orth_clip_opts(*o)), 1 << 45, 1 << 50, 1 << 30,
                                    None) == EINVAL


def test_norm_refusals_and_workspace(L):
    n = ctypes.c_size_t()
    assert L.orth_grad_norm_workspace_size(grads(), 3, ctypes.byref(n)) == OK and 0 < n.value < 1 << 16
    assert L.orth_grad_norm_workspace_size(grads(), -1, ctypes.byref(n)) == EINVAL
    assert L.orth_grad_norm_workspace_size(None, 3, ctypes.byref(n)) == EINVAL
    assert L.orth_grad_norm_workspace_size(grads(), 3, None) == EINVAL
    # (outputs are not looked at by the norm)
    assert L.orth_grad_norm_workspace_size(grads(out=None, ld_out=0), 3, ctypes.byref(n)) == OK
    assert L.orth_grad_norm_batched(grads(), 3, None, 1 << 50, 1 << 30, None) == EINVAL
    assert L.orth_grad_norm_batched(grads(), 3, 1 << 45, None, 0, None) == EWORKSPACE
    assert L.orth_grad_norm_batched(grads(), 3, 1 << 45, (1 << 50) + 8, 1 << 30, None) == EWORKSPACE
    assert L.orth_grad_norm_batched(grads(), 3, 1 << 45, 1 << 50, 16, None) == EWORKSPACE
    assert L.orth_grad_clip_batched(grads(), 3, None, 1 << 45, 1 << 50, 1 << 30, None) == EINVAL


def test_binding_refusals():
    """What the Python functions check before the library is called."""
    x, w = torch.zeros(4, 8), torch.zeros(2, 3, 8)
    off = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        orth.orth_linear_apply(x, w, off)                          # not on the GPU
    with pytest.raises(ValueError):
        orth.orth_linear_apply(x[:, :7], w, off)
    with pytest.raises(ValueError):
        orth.orth_linear_apply(x, w, off, out=torch.zeros(4, 4))
    with pytest.raises(TypeError):
        orth.orth_linear_apply(x.bfloat16(), w, off)
    with pytest.raises(ValueError):
        orth.orth_linear_grad_weight(torch.zeros(5, 3), x)
    with pytest.raises(TypeError):
        orth.orth_linear_grad_weight(torch.zeros(4, 3).bfloat16(), x)
    with pytest.raises(ValueError):
        orth.orth_linear_xent(x, torch.zeros(10, 8), torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError):
        orth.orth_linear_xent(x, torch.zeros(10, 7), torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError):
        orth.orth_grad_list([])
    with pytest.raises(ValueError):
        orth.orth_grad_list([x], [x, x])
    with pytest.raises(ValueError):
        orth.orth_grad_clip_batched([x], 1.0, norm_given=True)


def test_vjp_rows(L):
    """bf16 gradients hold dz in two rows each: up to 2^29 rows; the loss and
    fp32 gradients 2^30."""
    n = ctypes.c_size_t()
    most = 2 ** 30
    for dtype, rows, want in ((1, most // 2, OK), (1, most // 2 + 1, EINVAL), (0, most, OK)):
        a = ctypes.byref(xent(dtype=dtype, rows=rows))
        assert L.orth_linear_xent_vjp_workspace_size(a, ctypes.byref(n)) == want
        assert L.orth_linear_xent_workspace_size(a, ctypes.byref(n)) == OK
        if want != OK:
            assert L.orth_linear_xent_vjp(a, 1 << 45, 2 << 45, 5 << 45, 64, 6 << 45, 64, 1 << 50, 1 << 40, None) == want


@pytest.mark.parametrize("groups", [2 ** 20 + 1, 2 ** 30, BIG])
def test_too_many_groups(L, groups):
    """The device counts groups in 32 bits, 64 offsets at a time in every
    workgroup: more groups than that can be read in milliseconds are refused
    (with one matrix for all, which no bound on stride_w reaches)."""
    n = ctypes.c_size_t()
    a = ctypes.byref(linear(groups=groups, stride_w=0))
    assert L.orth_linear_apply(a, None) == EINVAL
    a = ctypes.byref(linear(groups=groups))
    assert L.orth_linear_grad_weight_workspace_size(a, ctypes.byref(n)) == EINVAL
    assert L.orth_linear_grad_weight(a, 1 << 50, 1 << 40, None) == EINVAL
    a = ctypes.byref(linear(groups=2 ** 20))
    assert L.orth_linear_grad_weight_workspace_size(a, ctypes.byref(n)) == OK


IN, OUT = 1 << 40, 2 << 40


@pytest.mark.parametrize("kw,want", [
    # (the last of three tensors, 4 x 8 float32: IN + 2^31 and OUT + 2^31 are its places)
    (dict(out=IN + (2 << 30) + 4), EINVAL), (dict(out=IN + (2 << 30) - 124), EINVAL),
    (dict(grad=IN, out=IN + 32, ld_grad=16, ld_out=16), OK), (dict(grad=IN, out=IN + 28, ld_grad=16, ld_out=16), EINVAL),
    (dict(grad=IN + 32, out=IN, ld_grad=16, ld_out=16), OK), (dict(grad=IN, out=IN + 96, ld_grad=16, ld_out=16), OK),
    (dict(grad=IN, out=IN + 40, ld_grad=16, ld_out=16), EINVAL), (dict(grad=IN, out=IN + 32, ld_grad=16, ld_out=17), EINVAL),
    (dict(out=OUT + 124), EINVAL), (dict(out=OUT + 128), OK), (dict(out=OUT + (1 << 30) - 4), EINVAL),
    # rows with gaps may hold another output in them
    (dict(out=OUT - 32, ld_out=64), OK),
    (dict(ld_grad=2 ** 47), EINVAL), (dict(ld_out=2 ** 47), EINVAL), (dict(rows=BIG, cols=BIG, ld_grad=2 ** 62, ld_out=2 ** 62), EINVAL)])
def test_clip_outputs_that_overlap(L, kw, want):
    """Outputs that share a part of their gradient or of each other.  (A small
    workspace refuses what is accepted otherwise, before anything is enqueued.)"""
    o = orth.orth_clip_opts(1.0, 1e-6, 0)
    rc = L.orth_grad_clip_batched(grads(**kw), 3, ctypes.byref(o), 1 << 45, 1 << 50, 16, None)
    assert rc == (EWORKSPACE if want == OK else want)
