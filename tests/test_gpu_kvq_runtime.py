"""The decoding loop over an 8-bit target cache with pooled pages: every
verification against the oracle on the values the cache holds, the committed
entries against the oracle's K/V, forks and compaction inside the loop.

Tolerances: fp32 logits 1e-4 and bf16 2e-2 relative (the suite's, see
test_gpu_tiny / test_gpu_bf16); a stored value is off by half an e4m3 step of
the oracle's K/V (2^-4 relative, 2^-10 of the page's scale below the least
normal code) plus those bounds on the K/V themselves."""
import dataclasses

import numpy as np
import pytest
import torch

import kvq_ref as ref
import synth
from gpu_harness import host, models, rel_err, runtime
from paper_2605_07243_amd import binding as B

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(600)]

SMALL = synth.ModelShape(2, 512, 8, 2, 128, 1024, 1024)


def workload(dtype, n_seqs, hi, lo=None):
    t = synth.TINY if dtype == "f32" else SMALL
    return synth.Workload("kvq-" + dtype, dtype, t, 1, K=3, M=2, B_max=4, budget=24,
                          n_seqs=n_seqs, prompt_len=(lo or hi, hi))


def cache_values(rt, seq, n):
    """What the 8-bit cache holds: ([layer] -> [n][Hkv][hd]) for K and V."""
    c, hd = rt.kvq, rt.w.target.head_dim
    table = host(rt.tpt)[seq]
    k, v, ke, ve = (host(t) for t in (c.k, c.v, c.k_exp, c.v_exp))
    return ([ref.entries(k[l], ke[l], table, n, hd, False) for l in range(k.shape[0])],
            [ref.entries(v[l], ve[l], table, n, hd, True) for l in range(k.shape[0])])


def oracle_verify(rt, tgt, seq):
    """The oracle's forward over the device's tree and the cache's values."""
    t = rt.tree
    n, T = int(t["n_nodes"][seq]), int(rt.T[seq])
    parent, depth, token = (host(t[f])[seq, :n] for f in ("parent", "depth", "token"))
    anc = []
    for i in range(n):
        anc.append(([] if parent[i] < 0 else anc[parent[i]]) + [i])
    prefix = tgt.new_prefix()
    k, v = cache_values(rt, seq, T)
    prefix.k, prefix.v = list(k), list(v)
    seg = tgt.new_segment(n)
    logits, _ = tgt.forward(token, T + depth, np.arange(n), anc, prefix, seg)
    return logits, seg, (k, v), T


def accept_deepest(rt, seqs):
    """Every sequence accepts the path to its lowest deepest node, as if the
    target had chosen it (random weights hardly ever do)."""
    t = rt.tree
    for s in seqs:
        n = int(t["n_nodes"][s])
        depth, parent = host(t["depth"])[s, :n], host(t["parent"])[s, :n]
        node, path = int(depth.argmax()), []
        while node > 0:
            path.insert(0, node)
            node = int(parent[node])
        rt.aout["path"][s, :len(path)] = torch.tensor(path, dtype=torch.int32)
        rt.aout["n_accepted"][s] = len(path)


def check_iteration(rt, tgt, tol, seqs, deepest=False):
    w = rt.w
    for m in range(1, w.M + 1):
        rt.expand(m)
    rt.verify(want_logits=True)
    torch.cuda.synchronize()
    want = {s: oracle_verify(rt, tgt, s) for s in seqs}
    rows = host(rt.tree["n_nodes"])
    at = np.concatenate([[0], np.cumsum(rows)])
    lg = host(rt.vout["logits"])
    for s in seqs:
        z = want[s][0]
        err = rel_err(lg[at[s]:at[s] + rows[s]], z).max()
        assert err < tol, (s, err)
        # greedy tokens: the oracle's best up to the tolerance
        a = host(rt.vout["argmax"])[s, :rows[s]]
        short = z.max(1) - z[np.arange(rows[s]), a]
        assert (short <= 2 * tol * np.abs(z).max(1)).all()
    rt.accept()
    if deepest:
        accept_deepest(rt, seqs)
        assert int(rt.aout["n_accepted"].max()) > 1
    rt.commit()
    torch.cuda.synchronize()
    for s in seqs:
        _, seg, before, T = want[s]
        n = int(rt.aout["n_accepted"][s])
        keep = [0] + host(rt.aout["path"])[s, :n].tolist()
        assert int(rt.T[s]) == T + n + 1
        k, v = cache_values(rt, s, T + n + 1)
        for got, old, src in ((k, before[0], seg.k), (v, before[1], seg.v)):
            for l in range(len(got)):
                x = np.stack([src[l][i] for i in keep])
                page = np.abs(got[l]).max()
                slack = 2.0 ** -4 * np.abs(x) + 2.0 ** -16 * page + 2 * tol * np.abs(x).max()
                assert (np.abs(got[l][T:] - x) <= slack).all()
                # held entries move by half a step at most where a scale rose
                assert (np.abs(got[l][:T] - old[l]) <= 2.0 ** -16 * page).all()


@pytest.mark.parametrize("dtype,tol", [("f32", 1e-4), ("bf16", 2e-2)])
@pytest.mark.parametrize("hi,lo", [(130, 17), (1, 1)])
def test_loop_over_the_8_bit_cache(dtype, tol, hi, lo):
    w = workload(dtype, 3, hi, lo)
    weights, tgt, _ = models(w)
    rt = runtime(w, weights, max_pages=(hi + 90) // 16, kvq=True)
    print("[kvq loop]", dtype, hi, flush=True)
    rt.prefill(synth.prompts(w))
    torch.cuda.synchronize()
    # the stored prompt: within half a step of the element-type cache
    for s in range(w.n_seqs):
        n = int(rt.T[s])
        for got, x in zip(cache_values(rt, s, n), rt.read_cache("target", s, n)):
            x = np.asarray(x, np.float64)
            top = np.abs(x).max()
            assert (np.abs(np.stack(got) - x)
                    <= 2.0 ** -4 * np.abs(x) + 2.0 ** -17 * top).all()
    for i in range(6):
        check_iteration(rt, tgt, tol, range(w.n_seqs), deepest=i != 1)
    assert int(rt.pool.refused[0]) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_window_that_holds_everything_and_one_that_does_not(dtype):
    """A window past the longest position changes nothing, one of 16 entries
    and 2 sinks does, and a later full verification is as before."""
    w = workload(dtype, 2, 100, 60)
    weights, _, _ = models(w)
    rt = runtime(w, weights, max_pages=12, kvq=True)
    rt.prefill(synth.prompts(w))
    for m in range(1, w.M + 1):
        rt.expand(m)
    rows = int(rt.tree["n_nodes"].sum())

    def logits(window, sinks):
        rt.window, rt.sinks = window, sinks
        rt.verify(want_logits=True)
        torch.cuda.synchronize()
        return host(rt.vout["logits"])[:rows].copy()

    full = logits(0, 0)
    assert np.array_equal(logits(100000, 0), full)
    near = logits(16, 2)
    assert not np.array_equal(near, full) and np.isfinite(near).all()
    assert np.array_equal(logits(0, 0), full)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forks_decode_as_their_parent(dtype):
    """Children of one parent, forked in the middle of a page, then a
    compaction: every continuation takes the parent's steps, bit for bit."""
    w = dataclasses.replace(workload(dtype, 4, 90, 40), n_seqs=4)
    weights, _, _ = models(w)
    rt = runtime(w, weights, max_pages=14, kvq=True)
    rt.prefill(synth.prompts(w))
    rt.iteration()
    rt.fork([0, 0], [2, 3])
    torch.cuda.synchronize()
    assert (host(rt.T)[[2, 3]] == host(rt.T)[0]).all()
    shared = host(rt.pool.refs).max()
    assert shared == 3
    for step in range(4):
        if step == 2:
            rt.pool.compact()
        rt.iteration()
        torch.cuda.synchronize()
        T = host(rt.T)
        for f in ("n_accepted", "bonus", "path"):
            a = host(rt.aout[f])
            assert np.array_equal(a[2], a[0]) and np.array_equal(a[3], a[0]), (step, f)
        assert T[2] == T[0] and T[3] == T[0]
        base = cache_values(rt, 0, int(T[0]))
        for s in (2, 3):
            for a, b in zip(cache_values(rt, s, int(T[0])), base):
                assert np.array_equal(np.stack(a), np.stack(b))
    refs, held = host(rt.pool.refs), host(rt.pool.held)
    live = int((refs > 0).sum())
    assert live < held.sum() and int(rt.pool.refused[0]) == 0


def test_the_element_type_cache_is_as_it_was():
    """The same prompts without the 8-bit cache: prefill alike, and the loop's
    first drafts too (they read the drafter's cache alone)."""
    w = workload("f32", 2, 70, 30)
    weights, _, _ = models(w)
    a = runtime(w, weights, max_pages=10)
    b = runtime(w, weights, max_pages=10, kvq=True)
    for rt in (a, b):
        rt.prefill(synth.prompts(w))
        for m in range(1, w.M + 1):
            rt.expand(m)
    torch.cuda.synchronize()
    assert np.array_equal(host(a.root), host(b.root))
    for s in range(2):
        for x, y in zip(a.read_cache("target", s, 30), b.read_cache("target", s, 30)):
            assert np.array_equal(x, y)
        n = int(a.tree["n_nodes"][s])
        assert np.array_equal(host(a.tree["token"])[s, :n], host(b.tree["token"])[s, :n])


def test_out_of_range_pages_are_reported():
    """With debug on, verification and commit report page-table entries that
    they clamped; with valid ones nothing."""
    w = workload("bf16", 2, 70, 40)
    weights, _, _ = models(w)
    rt = runtime(w, weights, max_pages=10, kvq=True)
    rt.set_debug(True)
    rt.prefill(synth.prompts(w))
    rt.iteration()
    rt.device_check()
    for m in range(1, w.M + 1):
        rt.expand(m)
    saved = rt.tpt.clone()
    rt.tpt[0, 0] = rt.kvq.k.shape[1] + 5
    rt.tpt[1, 1] = -1
    print("[debug] verify over out-of-range page-table entries", flush=True)
    rt.verify()
    with pytest.raises(B.SBError) as e:
        rt.device_check()
    assert e.value.code == B.SB_EDEVICE and "page" in str(e.value)
    rt.tpt.copy_(saved)
    rt.verify()
    rt.accept()
    rt.commit()
    rt.device_check()


def test_forks_need_the_8_bit_cache():
    w = workload("f32", 2, 20, 17)
    weights, _, _ = models(w)
    with pytest.raises(ValueError, match="8-bit"):
        runtime(w, weights, max_pages=10).fork([0], [1])
