"""Prompts that a prefill refuses leave the sequences of a runtime with an 8-bit
target cache as they are: their pages, their caches and their next steps."""
import numpy as np
import pytest
import torch

import synth
from gpu_harness import host, models, runtime
from paper_2605_07243_amd import binding as B
from test_gpu_kvq_runtime import workload

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_refused_prompts_change_nothing(dtype):
    w = workload(dtype, 3, 60, 30)
    weights, _, _ = models(w)
    prompts = [list(p) for p in synth.prompts(w)]
    bad = [[prompts[0], [], prompts[2]],            # an empty prompt
           prompts[:2],                             # one missing
           [prompts[0], [1] * 160, prompts[2]],     # longer than its table
           prompts + prompts[:1]]                   # one too many
    a, b = (runtime(w, weights, max_pages=10, kvq=True) for _ in range(2))
    for rt in (a, b):
        rt.prefill(prompts)
        rt.iteration()
    for p in bad:
        state = [host(t).copy() for t in (a.pool.page_table, a.pool.held, a.pool.refs,
                                          a.pool.refused, a.T, a.root)]
        with pytest.raises((B.SBError, IndexError)):
            a.prefill(p)
        torch.cuda.synchronize()
        for t, was in zip((a.pool.page_table, a.pool.held, a.pool.refs, a.pool.refused,
                           a.T, a.root), state):
            np.testing.assert_array_equal(host(t), was)
        for rt in (a, b):
            rt.iteration()
        torch.cuda.synchronize()
        for s in range(3):
            n = int(b.T[s])
            assert int(a.T[s]) == n and int(a.root[s]) == int(b.root[s])
            for x, y in zip(a.read_cache("target8", s, n), b.read_cache("target8", s, n)):
                np.testing.assert_array_equal(x, y)
    a.prefill(prompts)                              # and one that is taken
    assert host(a.T).tolist() == [len(p) for p in prompts]
