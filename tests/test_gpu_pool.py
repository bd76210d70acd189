"""The page pool (sb_pool_*) against its rules, one call at a time: tables,
counts, refusals and every byte of the caches' pages."""
import numpy as np
import pytest
import torch

import kvq_ref as ref

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


def kc():
    from paper_2605_07243_amd import kvcache
    return kvcache


class Pair:
    """A pool on the device with both caches, and the same on the host."""

    def __init__(self, S, mp, n_pages, Hkv=2, hd=64, layers=2, seed=0, dtype="bf16",
                 caches=True):
        self.shape = kc().Shape(Hkv, Hkv, hd, dtype, S, mp)
        self.pool = kc().PagePool.empty(self.shape, n_pages)
        self.ref = ref.PoolRef(S, mp, n_pages)
        self.mem = []
        if caches:
            g = torch.Generator().manual_seed(seed)
            byte = lambda *n: torch.randint(0, 256, n, generator=g,  # noqa: E731
                                            dtype=torch.int32).to(torch.uint8).cuda()
            es = 2 if dtype == "bf16" else 4
            el = self.shape.elem
            k = byte(1, n_pages, Hkv, 16, hd * es).view(el)
            v = byte(1, n_pages, Hkv, hd, 16 * es).view(el)
            kv = kc().PagedKV(self.shape, k, v, self.pool.page_table)
            kvq = kc().QuantKV(self.shape, byte(layers, n_pages, Hkv, 16 * hd),
                               byte(layers, n_pages, Hkv, 16 * hd),
                               byte(layers, n_pages, Hkv), byte(layers, n_pages, Hkv),
                               self.pool.page_table)
            self.pool.attach([kv, kvq])
            self.dev_mem = [k.view(torch.uint8), v.view(torch.uint8), kvq.k, kvq.v,
                            kvq.k_exp, kvq.v_exp]
            self.mem = [t.cpu().numpy().copy() for t in self.dev_mem]

    def i32(self, a):
        return torch.tensor(list(a), dtype=torch.int32).cuda()

    def check(self):
        torch.cuda.synchronize()
        r, p = self.ref, self.pool
        np.testing.assert_array_equal(p.held.cpu().numpy(), r.held)
        np.testing.assert_array_equal(p.refs.cpu().numpy(), r.refs)
        assert int(p.refused[0]) == r.refused
        t = p.page_table.cpu().numpy()
        for s in range(len(r.held)):
            np.testing.assert_array_equal(t[s, :r.held[s]], r.table[s, :r.held[s]],
                                          err_msg=str(s))
        for a, b in zip(self.mem, self.dev_mem if self.mem else []):
            np.testing.assert_array_equal(b.cpu().numpy(), a)

    def grow(self, length, extra=0):
        self.pool.grow(self.i32(length), extra)
        self.ref.grow(length, extra)

    def release(self, seqs):
        self.pool.release(seqs)
        self.ref.release(seqs)

    def _move(self, moves):
        for m in self.mem:
            src = [m[:, a].copy() for a, _ in moves]
            for (_, b), x in zip(moves, src):
                m[:, b] = x

    def fork(self, parents, children, length):
        self.pool.fork(parents, children, self.i32(length))
        self._move(self.ref.fork(parents, children, length))

    def compact(self):
        self.pool.compact()
        self._move(self.ref.compact())


def test_calls_in_turn():
    p = Pair(6, 5, 20)
    p.check()
    p.grow([33, 16, 0, 1])
    p.check()
    p.grow([33, 17, 0, 1], extra=15)
    p.check()
    p.fork([0, 0, 1], [2, 4, 5], [33, 17, 0, 1, 0, 0])
    p.check()
    p.release([0, 3])
    p.check()
    p.compact()
    p.check()
    p.grow([80, 0, 0, 70])
    p.check()
    p.pool.reset()
    p.ref = ref.PoolRef(6, 5, 20)
    p.check()


def test_lengths_at_page_borders_and_beyond_what_is_held():
    p = Pair(5, 4, 20)
    p.grow([48])
    # a whole number of pages: nothing is copied; past what the parent holds;
    # none at all, below zero
    for n in (48, 32, 64, 1000, 2 ** 31 - 1, 0, -5, 1, 15, 17):
        p.fork([0], [3], [n, 0, 0, 0, 0])
        p.check()


def test_chains_and_shared_pages_released_in_either_order():
    p = Pair(4, 6, 40)
    p.grow([70])
    p.fork([0], [1], [70, 0, 0, 0])
    p.fork([1], [2], [0, 68, 0, 0])
    p.grow([70, 68, 68], extra=20)
    p.check()
    p.release([0])
    p.check()
    p.release([2, 1])
    p.check()
    assert (p.ref.refs == 0).all()


def test_a_pool_that_runs_out():
    p = Pair(5, 8, 7)
    p.grow([40, 40, 40, 5])             # 3 + 3 + 1 of 3, none of 1
    p.check()
    assert p.ref.refused == 2
    p.fork([0, 1], [3, 4], [40, 39, 0, 0, 0])   # no page for the copies
    p.check()
    p.release([2])
    p.fork([0, 1], [3, 4], [40, 39, 0, 0, 0])   # one for the first
    p.check()
    p.grow([1, 1, 1, 2 ** 31 - 1, 2 ** 31 - 1], extra=2 ** 31 - 1)
    p.check()


def test_tables_that_run_out():
    p = Pair(2, 3, 20)
    p.grow([49, 48])
    p.check()
    assert p.ref.refused == 1


@pytest.mark.parametrize("dtype,Hkv,hd", [("bf16", 1, 64), ("f32", 3, 128), ("bf16", 8, 128)])
def test_random_calls(dtype, Hkv, hd):
    rng = np.random.default_rng([Hkv, hd])
    S, mp = 12, 7
    p = Pair(S, mp, 60, Hkv, hd, layers=3, dtype=dtype)
    for step in range(30):
        op = rng.choice(["grow", "fork", "release", "compact"], p=[.4, .3, .2, .1])
        length = rng.integers(0, 16 * mp, S)
        if op == "grow":
            p.grow(length[:rng.integers(1, S + 1)], int(rng.integers(0, 20)))
        elif op == "release":
            p.release(list(rng.permutation(S)[:rng.integers(1, S + 1)]))
        elif op == "compact":
            p.compact()
        else:
            order = list(rng.permutation(S))
            n = int(rng.integers(1, S))
            children, rest = order[:n], order[n:]
            p.fork([int(rng.choice(rest)) for _ in range(n)], children, length)
        print("[pool]", step, op, flush=True)
        p.check()


@pytest.mark.parametrize("n_pages", [8191, 8192, 8193, 70000])
def test_many_pages(n_pages):
    """Pools of several walks of 8192 pages (bookkeeping alone)."""
    S, mp = 64, 2048
    p = Pair(S, mp, n_pages, caches=False)
    rng = np.random.default_rng(n_pages)
    # (the rule, in whole-array form: the lowest free pages in order)
    p.pool.grow(p.i32(rng.integers(1, 16 * (n_pages // S + 200), S)))
    p.pool.release([int(s) for s in rng.permutation(S)[:40]])
    held = p.pool.held.cpu().numpy()
    refs = p.pool.refs.cpu().numpy()
    table = p.pool.page_table.cpu().numpy()
    want = np.zeros(n_pages, np.int64)
    for s in range(S):
        want[table[s, :held[s]]] += 1
    np.testing.assert_array_equal(refs, want)
    n = int((refs > 0).sum())
    p.pool.compact()
    torch.cuda.synchronize()
    refs2 = p.pool.refs.cpu().numpy()
    assert (refs2[:n] > 0).all() and (refs2[n:] == 0).all()
    to = np.arange(n_pages)
    src, dst = np.nonzero(refs > 0)[0], np.nonzero(refs[:n] == 0)[0]
    to[src[src >= n]] = dst
    t2 = p.pool.page_table.cpu().numpy()
    for s in range(S):
        np.testing.assert_array_equal(t2[s, :held[s]], to[table[s, :held[s]]])
    # the next pages are the lowest free ones, in order of sequence
    grow = np.where(held == 0, 16 * rng.integers(0, 3, S), 0)
    p.pool.grow(p.i32(grow))
    t3, nxt = p.pool.page_table.cpu().numpy(), n
    for s in range(S):
        k = int(min(grow[s] // 16, n_pages - nxt)) if held[s] == 0 else 0
        np.testing.assert_array_equal(t3[s, :k], np.arange(nxt, nxt + k))
        nxt += k


def test_calls_in_a_graph():
    """grow, fork, release and compact captured once and replayed from the same
    state."""
    p = Pair(6, 5, 24)
    p.grow([33, 16, 40, 1])
    p.check()
    length = p.i32([33, 16, 40, 1, 0, 0])
    state = [p.pool.page_table, p.pool.held, p.pool.refs, p.pool.refused] + p.dev_mem
    keep = [t.clone() for t in state]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.pool.fork([0, 2], [4, 5], length)
        p.pool.release([1, 2])
        p.pool.grow(length[:1], 30)
        p.pool.compact()
    p._move(p.ref.fork([0, 2], [4, 5], [33, 16, 40, 1, 0, 0]))
    p.ref.release([1, 2])
    p.ref.grow([33], 30)
    p._move(p.ref.compact())
    for _ in range(3):
        for t, was in zip(state, keep):
            t.copy_(was)
        graph.replay()
        p.check()
