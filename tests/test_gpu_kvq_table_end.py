"""Commits of a runtime with an 8-bit target cache near the end of a page-table
row: ``refused`` counts only what found no page or no room."""
import pytest
import torch

import synth
from gpu_harness import host, models, runtime
from test_gpu_kvq_runtime import accept_deepest, workload

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_commits_up_to_the_end_of_a_table(dtype):
    """Tables of 48 entries, prompts that leave six: commits that fit are not
    refused, whatever they might have added; the first that does not is."""
    w = workload(dtype, 2, 42, 42)
    weights, _, _ = models(w)
    rt = runtime(w, weights, max_pages=3, kvq=True)
    rt.prefill(synth.prompts(w))
    end = 48
    assert w.M * w.K + 1 > end - 42
    # entry by entry, then both sequences past the end in the last commit
    for step in range(8):
        for m in range(1, w.M + 1):
            rt.expand(m)
        rt.verify()
        rt.accept()
        rt.aout["n_accepted"].zero_()           # (the root alone)
        if step == 0:
            accept_deepest(rt, [1])             # and a path of sequence 1
            a = int(rt.aout["n_accepted"][1])
            assert a > 1
        rt.commit()
        torch.cuda.synchronize()
        T = host(rt.T).tolist()
        assert T == [43 + step, 43 + a + step]
        print("[table end]", step, T, int(rt.pool.refused[0]), flush=True)
        want = sum(max(0, 43 + step + d - end) for d in (0, a))
        assert int(rt.pool.refused[0]) == want
        assert host(rt.pool.held).tolist() == [min(3, (t + 15) // 16) for t in T]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_commit_takes_the_pages_of_what_it_adds(dtype):
    w = workload(dtype, 3, 40, 20)
    weights, _, _ = models(w)
    rt = runtime(w, weights, max_pages=12, kvq=True)
    rt.prefill(synth.prompts(w))
    for step in range(6):
        for m in range(1, w.M + 1):
            rt.expand(m)
        rt.verify()
        rt.accept()
        if step % 2:
            accept_deepest(rt, range(3))
        rt.commit()
        torch.cuda.synchronize()
        assert host(rt.pool.held).tolist() == [(t + 15) // 16 for t in host(rt.T).tolist()]
    assert int(rt.pool.refused[0]) == 0
