"""Attention over the 8-bit cache in each way that a call can be laid out: the
eight-wave workgroups, split prefixes of 64-wide heads, and waves that take
more tiles than they hold page numbers for (32 of the 16-query kernel, 64 of the
32-query one).  Every case states the plan that it is there for, so that a
change of the rule shows.  Values against float64 with test_gpu_kvq_attend's
tolerances."""
import ctypes as C

import numpy as np
import pytest
import torch

import kvq_ref as ref
from paper_2605_07243_amd import binding as B
from test_gpu_kvq_attend import Case

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


class Plan(C.Structure):
    """sb::QPlan"""
    _fields_ = [(n, C.c_int) for n in ("n_split", "split_tokens", "width", "n_waves")]


def plan_of(c, max_prefix=None):
    fn = B.load()._ZN2sb13kvq_attn_planEiiiiiiiii
    fn.restype, fn.argtypes = Plan, [C.c_int] * 9
    return fn(c.S, max(c.rows), max_prefix or max(c.T), c.window, c.sinks, c.H, c.Hkv,
              2 if c.dtype == "bf16" else 4, 64)


def check(c, width, n_waves, splits, rows=None):
    p = plan_of(c)
    print("[plan]", c.dtype, c.H, c.Hkv, c.hd, c.T, c.rows, "window", c.window, "->",
          p.n_split, p.split_tokens, p.width, p.n_waves, flush=True)
    assert (p.width, p.n_waves) == (width, n_waves)
    assert p.n_split > 1 if splits else p.n_split == 1
    got = c.run()
    c.check(got, rows=rows)
    assert np.array_equal(c.run(), got)
    return got, p


HEADS = [(8, 2, 128), (8, 8, 64), (5, 1, 64), (32, 4, 128)]


@pytest.mark.parametrize("H,Hkv,hd", HEADS)
@pytest.mark.parametrize("T,rows", [
    ([1024], [20]), ([1025], [17]), ([1151], [33]), ([1279], [21]),
    ([1279, 37, 0, 1040], [18, 33, 5, 1]), ([1263, 0], [64, 19])])
def test_eight_waves(H, Hkv, hd, T, rows):
    """More than 16 query vectors over prefixes that are not split."""
    check(Case("bf16", H, Hkv, hd, T, rows, seed=30), 32, 8, False)


@pytest.mark.parametrize("H,Hkv,hd", HEADS[:2])
def test_eight_waves_over_long_splits(H, Hkv, hd):
    n = {2: 40, 8: 60}[Hkv]
    c = Case("bf16", H, Hkv, hd, [9000, 4100, 11], [n, 23, 2], seed=31)
    check(c, 32, 8, True, rows=[0, 1, n // 2, n - 1, n, n + 22, n + 23, n + 24])


@pytest.mark.parametrize("H,Hkv,hd", HEADS[:2])
@pytest.mark.parametrize("window,sinks", [(1060, 4), (1000, 0), (1024, 17)])
def test_eight_waves_and_a_window(H, Hkv, hd, window, sinks):
    c = Case("bf16", H, Hkv, hd, [5003, 700, 1030], [33, 20, 1], seed=32, window=window,
             sinks=sinks)
    check(c, 32, 8, False, rows=list(range(0, 54, 3)) + [32, 52, 53])


@pytest.mark.parametrize("hd", [128, 64])
def test_hidden_entries_of_eight_waves(hd):
    """NaN codes past the prefix, NaN and infinities in slots that a row does not
    see, and in one that some rows do."""
    c = Case("bf16", 8, 2, hd, [1100], [40], seed=33)
    clean, _ = check(c, 32, 8, False)
    p, t = 1100 // 16, 1100 % 16
    for codes, is_v in ((c.k, False), (c.v, True)):
        for h in range(c.Hkv):
            pg = c.table[0, p]
            x = (ref.v_from_page(codes[0, pg, h], hd) if is_v
                 else codes[0, pg, h].reshape(16, hd)).copy()
            x[t:] = 0x7F
            codes[0, pg, h] = ref.v_to_page(x) if is_v else x.reshape(-1)
        codes[0, c.table[0, p + 1:]] = 0xFF
    c.sk_t[0, 2, :, 8:] = float("nan")          # slots 40 .. 47: no node
    c.sv_t[0, 2, :, :, 8:] = float("-inf")
    assert np.array_equal(c.run(), clean)
    c.sv_t[0, 0, :, 9, 6] = float("inf")
    got = c.run()
    for i in range(40):
        want = clean[i].copy()
        if (int(c.vis[i, 0]) >> 6) & 1:
            want[:, 9] = np.inf
        assert np.array_equal(got[i], want), i


def test_eight_waves_in_a_graph():
    c = Case("bf16", 8, 2, 128, [9000, 4100, 11], [40, 23, 2], seed=34)
    assert plan_of(c).n_waves == 8 and plan_of(c).n_split > 1
    first = c.run()
    plan, q = c.plan(), c.q_t.cuda()
    out = torch.zeros_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan(0, q, out)
    other = c.plan()
    for _ in range(3):
        out.zero_()
        other(0, q)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(out.float().cpu().numpy(), first)


@pytest.mark.parametrize("H,Hkv,T,rows", [(8, 8, [3000], [40]), (8, 8, [1290, 2600, 5], [17, 2, 70]),
                                          (5, 1, [2047, 1281], [9, 4])])
def test_split_prefixes_of_64_wide_heads(H, Hkv, T, rows):
    c = Case("bf16", H, Hkv, 64, T, rows, seed=35)
    check(c, 32, 4, True)


@pytest.mark.parametrize("dtype,H,Hkv,T,rows", [("bf16", 5, 1, [1281, 2000], [3, 1]),
                                                ("bf16", 8, 8, [4500], [16]),
                                                ("f32", 8, 8, [1300, 1290], [3, 33])])
def test_split_prefixes_of_64_wide_heads_in_16(dtype, H, Hkv, T, rows):
    check(Case(dtype, H, Hkv, 64, T, rows, seed=36), 16, 4, True)


@pytest.mark.parametrize("dtype,hd,most", [("bf16", 64, 5003), ("bf16", 128, 4300),
                                           ("f32", 64, 4225)])
def test_more_than_32_tiles_a_wave(dtype, hd, most):
    """A full chip of single tokens: prefixes past 4096 entries in one split."""
    T = [most, 4097, 4128] + [5 * i for i in range(14)]
    c = Case(dtype, 8, 8, hd, T, [1] * 17, seed=37)
    _, p = check(c, 16, 4, False)
    assert p.split_tokens > 4 * 32 * 32


@pytest.mark.parametrize("H,Hkv,hd,window,n_waves", [
    (8, 2, 128, 40, 4), (8, 8, 64, 40, 4), (8, 2, 128, 1060, 8), (8, 8, 64, 1060, 8)])
def test_more_than_64_tiles_a_wave(H, Hkv, hd, window, n_waves):
    """Rows far from the end of their prefix: windows that reach over most of
    it, in a call that is laid out for short ones."""
    c = Case("bf16", H, Hkv, hd, [20011, 50], [21, 20], seed=38, window=window, sinks=3)
    c.pos[:21] = 1200 + np.arange(21) * 7
    check(c, 32, n_waves, False, rows=[0, 10, 20, 21, 40])


@pytest.mark.parametrize("dtype,H,Hkv,hd", [("bf16", 8, 2, 128), ("f32", 4, 4, 64)])
def test_more_than_32_tiles_a_wave_of_windows(dtype, H, Hkv, hd):
    c = Case(dtype, H, Hkv, hd, [9005], [4], seed=39, window=30, sinks=0)
    c.pos[:] = [100, 117, 140, 4000]
    check(c, 16, 4, False)


@pytest.mark.parametrize("H,Hkv,hd", HEADS[:2])
def test_rows_of_one_tree_at_widely_spread_positions(H, Hkv, hd):
    """The first and the last row of a group of query vectors see next to nothing
    in common: most tiles are whole for some rows alone."""
    c = Case("bf16", H, Hkv, hd, [6000], [40], seed=40, window=64, sinks=20)
    c.pos[:] = np.linspace(0, 6100, 40).astype(np.int32)
    check(c, 32, 4, False)
