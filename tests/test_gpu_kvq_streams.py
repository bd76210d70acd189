"""Memory that the handles of the 8-bit cache allocate for the library's work:
dropped while another stream still uses it, it is not given out again before
that stream is done."""
import numpy as np
import pytest
import torch

from test_gpu_kvq_attend import Case
from test_gpu_pool import Pair

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


def busy(side, ms=60):
    """Tens of milliseconds of products on a stream; returns an event after them."""
    a = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(ms):
            b = a @ a
        b.record_stream(side)
        a.record_stream(side)
        done = torch.cuda.Event()
        done.record(side)
    return done


def given_out(shape, dtype, n=4):
    """Addresses that the allocator gives out for tensors of a size."""
    keep = [torch.empty(shape, dtype=dtype, device="cuda") for _ in range(n)]
    return [t.data_ptr() for t in keep], keep


def test_a_plan_dropped_while_a_side_stream_runs_it():
    c = Case("bf16", 8, 2, 128, [3000, 900], [20, 64], seed=21)
    plan, q = c.plan(), c.q_t.cuda()
    want = plan(0, q).float().cpu().numpy()
    out = torch.zeros_like(q)
    side = torch.cuda.Stream()
    done = busy(side)
    with torch.cuda.stream(side):
        plan(0, q, out)
    size, at = plan.workspace.shape, plan.workspace.data_ptr()
    keep = (plan.cache, plan._keep)     # the caller's own tensors live on
    assert size[0] > 1 << 20            # (several splits: the partials are there)
    del plan
    early = not done.query()
    ptrs, hold = given_out(size, torch.uint8)
    for t in hold:
        t.fill_(0xFF)                   # NaN partials, if they were the same memory
    assert early, "the side stream was done before the plan was dropped"
    assert at not in ptrs
    side.synchronize()
    assert np.array_equal(out.float().cpu().numpy(), want)
    del keep, hold


def test_a_pool_dropped_while_a_side_stream_forks_it():
    p = Pair(6, 5, 1 << 16, caches=False)
    p.grow([33, 16, 40])
    length = p.i32([33, 16, 40, 0, 0, 0])
    side = torch.cuda.Stream()
    done = busy(side)
    with torch.cuda.stream(side):
        p.pool.fork([0, 2], [4, 5], length)
    size, at = p.pool.scratch.shape, p.pool.scratch.data_ptr()
    p.ref.fork([0, 2], [4, 5], [33, 16, 40, 0, 0, 0])
    refs, held = p.pool.refs, p.pool.held
    p.pool = None
    early = not done.query()
    ptrs, hold = given_out(size, torch.int32)
    assert early, "the side stream was done before the pool was dropped"
    assert at not in ptrs
    side.synchronize()
    np.testing.assert_array_equal(held.cpu().numpy(), p.ref.held)
    np.testing.assert_array_equal(refs.cpu().numpy(), p.ref.refs)
    del hold
