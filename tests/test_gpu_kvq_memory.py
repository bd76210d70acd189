"""The device memory of a runtime with an 8-bit target cache: no element-type
cache beside it, but for a prefill's prompts until the first commit or fork."""
import dataclasses
import gc

import numpy as np
import pytest
import torch

import synth
from gpu_harness import host, models, runtime
from test_gpu_kvq_runtime import SMALL, cache_values, workload

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


def allocated():
    gc.collect()
    torch.cuda.synchronize()
    return torch.cuda.memory_allocated()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_half_the_bytes_or_less(dtype):
    w = dataclasses.replace(workload(dtype, 4, 100, 60), target=SMALL, n_seqs=4)
    es, pages = (2 if dtype == "bf16" else 4), 4 * 512
    page = 2 * SMALL.n_layers * SMALL.n_kv_heads * 16 * SMALL.head_dim   # values
    at = allocated()
    plain = runtime(w, None, max_pages=512)
    plain_bytes = allocated() - at
    at = allocated()
    rt = runtime(w, None, max_pages=512, kvq=True)
    slack = 1 << 20             # (tables, counts, rounding of the allocator)
    want = plain_bytes - pages * page * es + pages * page * 17 // 16
    assert allocated() - at <= want + slack
    at = allocated()
    prompts = synth.prompts(w)
    staged = sum((len(p) + 15) // 16 for p in prompts) * page * es
    for leave in ("commit", "fork"):
        rt.prefill(prompts)
        assert staged <= allocated() - at <= staged + slack
        rt.prefill(prompts)     # (the earlier one's go)
        assert allocated() - at <= staged + slack
        if leave == "commit":
            rt.iteration()
        else:
            rt.fork([0], [1])
        assert allocated() - at <= slack, leave
    del plain


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompts_that_fill_their_tables(dtype):
    """Prompts of one entry and of all that a table holds but one, prefilled
    again over what was there: what is stored is what each prefill computed."""
    w = workload(dtype, 3, 79, 1)
    weights, _, _ = models(w)
    rt = runtime(w, weights, max_pages=5, kvq=True)
    plain = runtime(w, weights, max_pages=5)
    rng = np.random.default_rng(4)
    for lens in ((79, 1, 16), (1, 79, 17), (64, 65, 79)):
        prompts = [[int(t) for t in rng.integers(0, w.target.vocab, n)] for n in lens]
        for r in (rt, plain):
            r.prefill(prompts)
        torch.cuda.synchronize()
        assert host(rt.root).tolist() == host(plain.root).tolist()
        for s, n in enumerate(lens):
            for a, b, c in zip(rt.read_cache("target", s, n), plain.read_cache("target", s, n),
                               cache_values(rt, s, n)):
                np.testing.assert_array_equal(a, b)
                top = np.abs(a).max()
                assert (np.abs(np.stack(c) - a)
                        <= 2.0 ** -4 * np.abs(a) + 2.0 ** -17 * top).all()
        rt.iteration()
    assert int(rt.pool.refused[0]) == 0


def test_prompts_that_memory_does_not_hold():
    """An allocation that fails in a prefill leaves the sequences their pages."""
    w = workload("bf16", 2, 40, 30)
    weights, _, _ = models(w)
    rt = runtime(w, weights, max_pages=10, kvq=True)
    rt.prefill(synth.prompts(w))
    rt.iteration()
    state = [host(t).copy() for t in (rt.pool.page_table, rt.pool.held, rt.pool.refs, rt.T)]

    def no_room(lens):
        raise torch.OutOfMemoryError("no room")

    stage, rt._stage = rt._stage, no_room
    with pytest.raises(torch.OutOfMemoryError):
        rt.prefill(synth.prompts(w))
    rt._stage = stage
    for t, was in zip((rt.pool.page_table, rt.pool.held, rt.pool.refs, rt.T), state):
        np.testing.assert_array_equal(host(t), was)
