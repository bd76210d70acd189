"""read_cache and write_cache of a runtime with an 8-bit target cache: what they
return is the cache that verification reads, or they refuse."""
import dataclasses

import numpy as np
import pytest
import torch

import synth
from gpu_harness import host, models, runtime
from test_gpu_kvq_runtime import accept_deepest, cache_values, workload

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


def step(rt, w, seqs):
    for m in range(1, w.M + 1):
        rt.expand(m)
    rt.verify()
    rt.accept()
    accept_deepest(rt, seqs)
    rt.commit()
    torch.cuda.synchronize()


def check8(rt, seq):
    n = int(rt.T[seq])
    for got, want in zip(rt.read_cache("target8", seq, n), cache_values(rt, seq, n)):
        # (a code times a power of two is exact in fp32)
        np.testing.assert_array_equal(got, np.stack(want))
    lo = max(0, n - 7)
    for got, want in zip(rt.read_cache("target8", seq, n - lo, lo), cache_values(rt, seq, n)):
        np.testing.assert_array_equal(got, np.stack(want)[:, lo:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_reads_follow_the_8_bit_cache(dtype):
    w = dataclasses.replace(workload(dtype, 4, 50, 30), n_seqs=4)
    weights, _, _ = models(w)
    rt = runtime(w, weights, max_pages=10, kvq=True)
    rt.prefill(synth.prompts(w))
    torch.cuda.synchronize()
    n0 = [int(t) for t in rt.T]
    first = [rt.read_cache("target", s, n0[s]) for s in range(4)]
    # pages that move under it do not change what a prefill left
    rt.pool.release([0])
    rt.pool.compact()
    for s in range(1, 4):
        for a, b in zip(rt.read_cache("target", s, n0[s]), first[s]):
            np.testing.assert_array_equal(a, b)
        check8(rt, s)
    with pytest.raises(ValueError, match="target8"):
        rt.read_cache("target", 1, n0[1] + 1)       # past its prompt
    with pytest.raises(ValueError, match="no pages"):
        rt.read_cache("target8", 0, 1)
    rt.prefill(synth.prompts(w))
    step(rt, w, range(4))
    with pytest.raises(ValueError, match="target8"):
        rt.read_cache("target", 0, 1)
    for s in range(4):
        assert int(rt.T[s]) > n0[s] + 1
        check8(rt, s)
    rt.fork([0], [2])
    rt.pool.compact()
    torch.cuda.synchronize()
    for s in range(4):
        check8(rt, s)
    n = int(rt.T[0])
    for a, b in zip(rt.read_cache("target8", 0, n), rt.read_cache("target8", 2, n)):
        np.testing.assert_array_equal(a, b)


def test_reads_and_writes_that_are_refused():
    w = workload("f32", 2, 20, 17)
    weights, _, _ = models(w)
    rt = runtime(w, weights, max_pages=10, kvq=True)
    with pytest.raises(ValueError, match="target8"):
        rt.read_cache("target", 0, 1)               # nothing prefilled
    rt.prefill(synth.prompts(w))
    k, v = rt.read_cache("target", 0, 17)
    with pytest.raises(ValueError, match="kvq.store"):
        rt.write_cache("target", 0, k, v)
    dk, dv = rt.read_cache("drafter", 0, 10)
    rt.write_cache("drafter", 0, dk, dv, 3)         # (the drafter's as ever)
    np.testing.assert_array_equal(rt.read_cache("drafter", 0, 10, 3)[0], dk)
    with pytest.raises(ValueError, match="no pages"):
        rt.read_cache("drafter", 0, 60)
    rt.fork([0], [1])
    with pytest.raises(ValueError, match="target8"):
        rt.read_cache("target", 1, 1)
    plain = runtime(w, weights, max_pages=10)
    with pytest.raises(ValueError, match="8-bit"):
        plain.read_cache("target8", 0, 1)
    plain.prefill(synth.prompts(w))
    plain.write_cache("target", 0, k, v, 5)
    np.testing.assert_array_equal(plain.read_cache("target", 0, 17, 5)[1], v)
    assert host(plain.T).min() >= 17
