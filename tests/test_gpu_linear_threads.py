"""The row-grouped products, the head's loss and the clipping from several host
threads at once, each on a stream and with tensors of its own: every result
is the same, bit for bit, as of the call made alone (the long gradient list
takes its table through the library's shared staging buffers)."""

import threading

import pytest
import torch

from paper_2601_13776_amd import orth

from gpu_util import DEV
from test_gpu_linear import bounds_of, rand
from test_gpu_xent import targets_of

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def job_layers(dt, seed):
    x, w, gy = rand((900, 264), seed, dt), rand((3, 520, 264), seed + 1, dt), rand((900, 520), seed + 2, dt)
    offsets = bounds_of([500, 0, 400])[1]
    return lambda: [orth.orth_linear_apply(x, w, offsets), orth.orth_linear_apply(gy, w, offsets, transposed=True),
                    orth.orth_linear_grad_weight(gy, x, offsets)]


def job_head(dt, seed):
    x, w = rand((600, 128), seed, dt), rand((3001, 128), seed + 1, dt, 128 ** -0.5)
    t, gl = targets_of(600, 3001, seed + 2), rand((600,), seed + 3, F32)

    def call():
        loss, lse = orth.orth_linear_xent(x, w, t)
        return [loss, lse, *orth.orth_linear_xent_vjp(x, w, t, lse, gl, piece=1000)]
    return call


def job_clip(n, seed):
    grads = [rand((17 + i % 5, 31), seed + i, (F32, BF16)[i % 2]) for i in range(n)]
    outs = [torch.empty_like(g) for g in grads]
    lst = orth.orth_grad_list(grads, outs)
    return lambda: [orth.orth_grad_clip_batched(lst, 1.0), *[o.clone() for o in outs]]


def test_concurrent_callers_match_single_calls():
    print("[linear threads]", flush=True)
    jobs = [job_layers(F32, 1), job_layers(BF16, 11), job_head(F32, 21), job_head(BF16, 31), job_clip(20, 41),
            job_clip(300, 100)]
    alone = [j() for j in jobs]
    torch.cuda.synchronize()
    results, errors = [[] for _ in jobs], []
    start = threading.Barrier(len(jobs))

    def worker(k):
        try:
            s = torch.cuda.Stream()
            start.wait(timeout=30)
            with torch.cuda.stream(s):
                for _ in range(4):
                    results[k].append(jobs[k]())
            s.synchronize()
        except Exception as e:  # noqa: BLE001 (reported below)
            errors.append((k, e))

    threads = [threading.Thread(target=worker, args=(k,)) for k in range(len(jobs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join(timeout=60)
    assert not errors, errors
    for want, runs in zip(alone, results):
        assert len(runs) == 4
        for got in runs:
            assert all(torch.equal(a, b) for a, b in zip(want, got))
