"""Sequences without the pages that they ask for: nothing of what they would
store reaches a page of another sequence, in the 8-bit cache, the element-type
caches and the drafter's."""
import dataclasses

import numpy as np
import pytest
import torch

import synth
from gpu_harness import host, models, runtime
from paper_2605_07243_amd import binding as B
from test_gpu_kvq_runtime import accept_deepest, workload
from test_gpu_pool import Pair

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


def kc():
    from paper_2605_07243_amd import kvcache
    return kvcache


def test_table_entries_past_what_is_held_name_no_page():
    S, mp = 10, 6
    p = Pair(S, mp, 30, caches=False)
    p.pool.reset()
    rng = np.random.default_rng(5)
    for step in range(40):
        op = rng.choice(["grow", "fork", "release", "compact"], p=[.4, .3, .2, .1])
        length = rng.integers(0, 16 * mp, S)
        if op == "grow":
            p.grow(length[:rng.integers(1, S + 1)], int(rng.integers(0, 20)))
        elif op == "release":
            p.release([int(s) for s in rng.permutation(S)[:3]])
        elif op == "compact":
            p.compact()
        else:
            order = [int(s) for s in rng.permutation(S)]
            n = int(rng.integers(1, S))
            p.fork([int(rng.choice(order[n:])) for _ in range(n)], order[:n], length)
        p.check()
        past = np.arange(mp) >= p.ref.held[:, None]
        assert (host(p.pool.page_table)[past] == -1).all(), (step, op)
    assert p.ref.refused > 0


@pytest.mark.parametrize("dtype,Hkv,hd", [("bf16", 2, 128), ("f32", 3, 64)])
def test_store_past_a_refused_grow(dtype, Hkv, hd):
    """A pool with pages for some of what three sequences store: the rest is
    dropped, as if the lengths had been cut to the pages."""
    S, mp, L, n = 3, 4, 2, 7
    shape = kc().Shape(Hkv, Hkv, hd, dtype, S, mp)
    g = torch.Generator().manual_seed(7)
    val = lambda *s: torch.randn(s, generator=g).to(shape.elem).cuda()  # noqa: E731
    table = torch.arange(S * mp, dtype=torch.int32).view(S, mp).cuda()
    src = kc().PagedKV(shape, val(L, S * mp, Hkv, 16, hd), val(L, S * mp, Hkv, hd, 16), table)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32).cuda()  # noqa: E731
    lens = [40, 50, 60]                     # 3 + 4 + none of 4 pages

    def run(last):
        pool = kc().PagePool.empty(shape, n)
        cache = kc().QuantKV.empty(shape, L, n, pool.page_table)
        for t in (cache.k, cache.v, cache.k_exp, cache.v_exp):
            t.fill_(0x5A)
        pool.grow(i32(lens))
        cache.store(src, i32([0, 0, 0]), i32(last), 64)
        torch.cuda.synchronize()
        assert int(pool.refused[0]) == 1 and host(pool.held).tolist() == [3, 4, 0]
        return [host(t) for t in (cache.k, cache.v, cache.k_exp, cache.v_exp)]

    for a, b in zip(run(lens), run([40, 50, 0])):
        np.testing.assert_array_equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("deepest", [False, True])
def test_commit_without_pages(dtype, deepest):
    """A commit whose new entries have no page: the target's 8-bit cache and the
    drafter's keep every byte, the debug word reports it, and a sequence that
    has its pages commits as ever."""
    w = workload(dtype, 2, 32, 32)
    weights, _, _ = models(w)
    print("[pages] commit", dtype, deepest, flush=True)

    def run(missing):
        rt = runtime(w, weights, max_pages=6, kvq=True)
        rt.set_debug(True)
        rt.prefill(synth.prompts(w))
        for m in range(1, w.M + 1):
            rt.expand(m)
        rt.verify()
        rt.accept()
        if deepest:
            accept_deepest(rt, range(2))
        rt.device_check()
        # both prompts end with their second page; sequence 0 holds page 0
        assert host(rt.pool.held).tolist() == [2, 2] and int(rt.tpt[0, 0]) == 0
        mem = [rt.kvq.k, rt.kvq.v, rt.kvq.k_exp, rt.kvq.v_exp, rt.dk, rt.dv]
        before = [t.clone() for t in mem]
        if missing:                     # (none for sequence 1 either way)
            rt.pool.grow = lambda *a, **kw: None
        rt.commit()
        torch.cuda.synchronize()
        if missing:
            with pytest.raises(B.SBError) as e:
                rt.device_check()
            assert e.value.code == B.SB_EDEVICE and "page" in str(e.value)
            for t, was in zip(mem, before):
                assert torch.equal(t.view(torch.uint8), was.view(torch.uint8))
        else:
            rt.device_check()
            assert any(not torch.equal(t.view(torch.uint8), was.view(torch.uint8))
                       for t, was in zip(mem, before))

    run(True)
    run(False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_element_type_caches_without_a_page(dtype):
    """sb_prefill and sb_commit through a negative page-table entry leave page 0
    to the sequence that has it."""
    w = dataclasses.replace(workload(dtype, 2, 40, 40), n_seqs=2)
    weights, _, _ = models(w)
    print("[pages] prefill", dtype, flush=True)
    first = []
    for missing in (False, True):
        rt = runtime(w, weights, max_pages=6)
        for pt in (rt.tpt, rt.dpt):     # page j of sequence s: 6 s + j
            pt.copy_(torch.arange(12, dtype=torch.int32).view(2, 6))
            if missing:
                pt[1, 2:] = -1
        rt.prefill(synth.prompts(w))
        for m in range(1, w.M + 1):
            rt.expand(m)
        rt.verify()
        rt.accept()
        accept_deepest(rt, [0, 1])
        rt.commit()
        torch.cuda.synchronize()
        first.append([host(t[:, :6].float()) for t in (rt.tk, rt.tv, rt.dk, rt.dv)])
        n = int(rt.T[0])
        assert n > 41
        if missing:                     # what sequence 1 could not store is nowhere
            for t in (rt.tk, rt.tv, rt.dk, rt.dv):
                assert not t[:, 8:].any()
    for a, b in zip(*first):
        np.testing.assert_array_equal(a, b)
