"""Host-side checks of the 8-bit cache's and the page pool's entry points: what
is refused, with which code and message, before anything is enqueued.  No GPU."""
import ctypes as C
import types

import pytest
import torch

from paper_2605_07243_amd import binding as B
from paper_2605_07243_amd import kvcache
from paper_2605_07243_amd.runtime import Runtime
from test_abi import Fake, bound, cfg, lib  # noqa: F401


def shape(**kw):
    v = dict(n_heads=8, n_kv_heads=2, head_dim=64, dtype=B.SB_BF16, max_seqs=4,
             max_pages=10)
    v.update(kw)
    return B.CacheShape(**v)


def kvq(f, **kw):
    v = dict(k=f.at(), v=f.at(), k_exp=f.at(1), v_exp=f.at(3), page_table=f.at(4),
             n_layers=2, n_pages=40)
    v.update(kw)
    return B.KVQ(**v)


def kv(f, **kw):
    v = dict(k=f.at(), v=f.at(), page_table=f.at(4), n_layers=2, n_pages=40)
    v.update(kw)
    return B.KV(**v)


def rows(f, **kw):
    v = dict(n_seqs=2, n_rows=9, rows_per_seq=5, max_prefix=100, vis_words=1,
             seg_pages=1, row_off=f.at(), pos=f.at(), prefix_len=f.at(),
             seg_len=f.at(), vis=f.at(), seg_k=f.at(), seg_v=f.at())
    v.update(kw)
    return B.AttnRows(**v)


def pool(f, **kw):
    v = dict(page_table=f.at(4), held=f.at(), refs=f.at(), refused=f.at(),
             scratch=f.at(), n_pages=40)
    v.update(kw)
    return B.Pool(**v)


BAD_SHAPES = [(dict(dtype=3), B.SB_EDTYPE), (dict(head_dim=96), B.SB_ESHAPE),
              (dict(n_heads=7), B.SB_ESHAPE), (dict(n_heads=0), B.SB_ESHAPE),
              (dict(n_heads=66, n_kv_heads=66), B.SB_ESHAPE),
              (dict(n_kv_heads=0), B.SB_ESHAPE), (dict(n_kv_heads=-2), B.SB_ESHAPE),
              (dict(max_seqs=0), B.SB_ESHAPE), (dict(max_seqs=65), B.SB_ESHAPE),
              (dict(max_pages=0), B.SB_ESHAPE), (dict(max_pages=16385), B.SB_ESHAPE)]


def says(lib, call):  # noqa: F811
    assert lib.sb_last_error(None).decode().startswith(call + ": ")


@pytest.mark.parametrize("kw,code", BAD_SHAPES)
def test_shapes(lib, kw, code):  # noqa: F811
    f = Fake()
    s, p = shape(**kw), pool(f)
    i = (C.c_int32 * 1)(0)
    assert lib.sb_kvq_store(s, 1, kv(f), f.at(), f.at(), 1, kvq(f), None) == code
    says(lib, "sb_kvq_store")
    assert lib.sb_kvq_attend_workspace(s, rows(f), 0, 0) == 0
    assert lib.sb_kvq_attend(s, kvq(f), 0, rows(f), f.at(), 0, 0, f.at(1 << 15),
                             f.at(), 1 << 30, None) == code
    says(lib, "sb_kvq_attend")
    for rc in (lib.sb_pool_reset(s, p, None), lib.sb_pool_grow(s, p, 1, f.at(), 0, None),
               lib.sb_pool_release(s, p, 1, i, None),
               lib.sb_pool_fork(s, p, 1, i, i, f.at(), None, None, None),
               lib.sb_pool_compact(s, p, None, None, None)):
        assert rc == code
    assert lib.sb_pool_compact(None, p, None, None, None) == B.SB_EINVAL


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), B.SB_EINVAL), (dict(v=None), B.SB_EINVAL),
    (dict(k_exp=None), B.SB_EINVAL), (dict(v_exp=None), B.SB_EINVAL),
    (dict(page_table=None), B.SB_EINVAL), (dict(n_pages=0), B.SB_EINVAL),
    (dict(n_layers=0), B.SB_ESHAPE), (dict(n_layers=70000), B.SB_ESHAPE)])
def test_caches(lib, kw, code):  # noqa: F811
    f, s = Fake(), shape()
    assert lib.sb_kvq_store(s, 1, kv(f), f.at(), f.at(), 1, kvq(f, **kw), None) == code
    assert lib.sb_kvq_attend(s, kvq(f, **kw), 0, rows(f), f.at(), 0, 0, f.at(1 << 15),
                             f.at(), 1 << 30, None) == code
    assert lib.sb_pool_compact(s, pool(f), None, kvq(f, **kw), None) == code
    kw = {n: x for n, x in kw.items() if not n.endswith("_exp")}
    if kw:
        assert lib.sb_kvq_store(s, 1, kv(f, **kw), f.at(), f.at(), 1, kvq(f), None) == code
        assert lib.sb_pool_compact(s, pool(f), kv(f, **kw), None, None) == code


def test_store(lib):  # noqa: F811
    f, s = Fake(), shape()
    run = lambda **k: lib.sb_kvq_store(  # noqa: E731
        s, k.get("n", 1), kv(f), k.get("first", f.at()), k.get("last", f.at()),
        k.get("most", 1), k.get("dst", kvq(f)), None)
    assert run(n=0) == B.SB_ESHAPE and run(n=5) == B.SB_ESHAPE
    assert run(first=None) == B.SB_EINVAL and run(last=f.at(2)) == B.SB_EINVAL
    assert run(most=0) == B.SB_EINVAL and run(most=-1) == B.SB_EINVAL
    assert run(dst=kvq(f, n_layers=3)) == B.SB_ESHAPE
    assert run(dst=kvq(f, k=f.at(8))) == B.SB_EINVAL
    assert lib.sb_kvq_store(s, 1, None, f.at(), f.at(), 1, kvq(f), None) == B.SB_EINVAL
    assert lib.sb_kvq_store(s, 1, kv(f), f.at(), f.at(), 1, None, None) == B.SB_EINVAL


@pytest.mark.parametrize("kw,code", [
    (dict(n_seqs=0), B.SB_ESHAPE), (dict(n_seqs=5), B.SB_ESHAPE),
    (dict(n_rows=0), B.SB_ESHAPE), (dict(n_rows=(1 << 22) + 1), B.SB_ESHAPE),
    (dict(rows_per_seq=0), B.SB_ESHAPE), (dict(rows_per_seq=16385), B.SB_ESHAPE),
    (dict(max_prefix=-1), B.SB_EINVAL), (dict(vis_words=17), B.SB_ESHAPE),
    (dict(vis_words=-1), B.SB_ESHAPE), (dict(seg_pages=33), B.SB_ESHAPE),
    (dict(seg_pages=-1), B.SB_ESHAPE)])
def test_rows_host_values(lib, kw, code):  # noqa: F811
    f, s = Fake(), shape()
    assert lib.sb_kvq_attend_workspace(s, rows(f, **kw), 0, 0) == 0
    says(lib, "sb_kvq_attend_workspace")
    assert lib.sb_kvq_attend(s, kvq(f), 0, rows(f, **kw), f.at(), 0, 0, f.at(1 << 15),
                             f.at(), 1 << 30, None) == code


def test_attend(lib):  # noqa: F811
    f, s = Fake(), shape()
    n = 9 * 8 * 64 * 2

    def run(**k):
        return lib.sb_kvq_attend(
            s, kvq(f), k.get("layer", 0), k.get("rows", rows(f)), k.get("q", f.at()),
            k.get("window", 0), k.get("sinks", 0), k.get("out", f.at(1 << 15)),
            k.get("ws", f.at()), k.get("bytes", 1 << 30), None)

    assert run(layer=-1) == B.SB_EINVAL and run(layer=2) == B.SB_EINVAL
    assert run(window=-1) == B.SB_EINVAL and run(sinks=-1) == B.SB_EINVAL
    assert lib.sb_kvq_attend_workspace(s, rows(f), -1, 0) == 0
    assert run(q=None) == B.SB_EINVAL and run(q=f.at(8)) == B.SB_EINVAL
    assert run(out=None) == B.SB_EINVAL and run(out=f.at(4)) == B.SB_EINVAL
    assert run(out=f.at()) == B.SB_EINVAL and run(out=f.at(n - 16)) == B.SB_EINVAL
    says(lib, "sb_kvq_attend")
    assert run(ws=None) == B.SB_EINVAL and run(ws=f.at(16)) == B.SB_EINVAL
    need = lib.sb_kvq_attend_workspace(s, rows(f), 0, 0)
    assert need >= 256 and need % 256 == 0
    assert run(bytes=need - 1) == B.SB_EBUDGET
    assert run(rows=None) == B.SB_EINVAL
    for name in ("row_off", "prefix_len", "seg_len", "vis", "seg_k", "seg_v"):
        assert run(rows=rows(f, **{name: None})) == B.SB_EINVAL, name
    assert run(rows=rows(f, vis_words=0)) == B.SB_EINVAL
    assert run(rows=rows(f, pos=None), window=3) == B.SB_EINVAL
    assert run(rows=rows(f, seg_k=f.at(8))) == B.SB_EINVAL


def test_workspace_grows_with_the_splits(lib):  # noqa: F811
    f = Fake()
    s = shape(max_pages=16384)
    short = lib.sb_kvq_attend_workspace(s, rows(f, max_prefix=100), 0, 0)
    long = lib.sb_kvq_attend_workspace(s, rows(f, max_prefix=200000), 0, 0)
    capacity = lib.sb_kvq_attend_workspace(s, rows(f, max_prefix=0), 0, 0)
    windowed = lib.sb_kvq_attend_workspace(s, rows(f, max_prefix=200000), 64, 4)
    assert 256 <= short <= long <= capacity and windowed < long
    # device pointers are not looked at
    null = {n: None for n in ("row_off", "pos", "prefix_len", "seg_len", "vis",
                              "seg_k", "seg_v")}
    assert lib.sb_kvq_attend_workspace(s, rows(f, max_prefix=100, **null), 0, 0) == short


def test_pool(lib):  # noqa: F811
    f, s = Fake(), shape()
    ok = (C.c_int32 * 4)(0, 1, 2, 3)
    arr = lambda *v: (C.c_int32 * len(v))(*v)  # noqa: E731
    for name in ("page_table", "held", "refs", "refused", "scratch"):
        for p in (None, f.at(2)):
            assert lib.sb_pool_reset(s, pool(f, **{name: p}), None) == B.SB_EINVAL
    assert lib.sb_pool_reset(s, None, None) == B.SB_EINVAL
    for n in (0, -1, (1 << 20) + 1):
        assert lib.sb_pool_reset(s, pool(f, n_pages=n), None) == B.SB_ESHAPE
        assert lib.sb_pool_scratch_ints(n) == 0
    assert lib.sb_pool_scratch_ints(40) >= 80
    p = pool(f)
    assert lib.sb_pool_grow(s, p, 0, f.at(), 0, None) == B.SB_ESHAPE
    assert lib.sb_pool_grow(s, p, 5, f.at(), 0, None) == B.SB_ESHAPE
    assert lib.sb_pool_grow(s, p, 1, None, 0, None) == B.SB_EINVAL
    assert lib.sb_pool_grow(s, p, 1, f.at(), -1, None) == B.SB_EINVAL
    for n, a, code in ((0, ok, B.SB_ESHAPE), (5, ok, B.SB_ESHAPE), (1, None, B.SB_EINVAL),
                       (1, arr(4), B.SB_EINVAL), (1, arr(-1), B.SB_EINVAL),
                       (2, arr(1, 1), B.SB_EINVAL)):
        assert lib.sb_pool_release(s, p, n, a, None) == code
    for pa, ch in ((arr(0, 1), arr(2, 2)), (arr(0, 1), arr(1, 2)), (arr(0), arr(0)),
                   (arr(0, 4), arr(1, 2)), (arr(0, 0), arr(1, -1))):
        assert lib.sb_pool_fork(s, p, len(pa), pa, ch, f.at(), None, None,
                                None) == B.SB_EINVAL
    one = arr(0), arr(1)
    assert lib.sb_pool_fork(s, p, 1, *one, None, None, None, None) == B.SB_EINVAL
    assert lib.sb_pool_fork(s, p, 1, None, arr(1), f.at(), None, None, None) == B.SB_EINVAL
    other = [kv(f, n_pages=41), kv(f, page_table=f.at(8))]
    for c in other:
        assert lib.sb_pool_fork(s, p, 1, *one, f.at(), c, None, None) == B.SB_EINVAL
        says(lib, "sb_pool_fork")
    for c in (kvq(f, n_pages=41), kvq(f, page_table=f.at(8))):
        assert lib.sb_pool_compact(s, p, None, c, None) == B.SB_EINVAL


def test_verify_and_commit(bound):  # noqa: F811
    """sb_tree_verify_kvq and sb_commit_kvq refuse what the element-type calls
    refuse, and windows below zero."""
    lib, ctx, f = bound  # noqa: F811
    sq, t = B.Seqs(1, f.at(), f.at(), f.at()), B.Tree(*[f.at()] * len(B.TREE_FIELDS))
    out, acc = B.VerifyOut(f.at(), f.at(), None), B.AcceptOut(f.at(), f.at(), f.at(), None)
    q = kvq(f)
    run = lambda c=q, w=0, s=0, o=out: lib.sb_tree_verify_kvq(  # noqa: E731
        ctx, C.byref(sq), C.byref(t), c, w, s, o, None)
    assert run(w=-1) == B.SB_EINVAL and run(s=-1) == B.SB_EINVAL
    assert run(c=None) == B.SB_EINVAL and run(o=None) == B.SB_EINVAL
    assert run(c=kvq(f, n_layers=3)) == B.SB_ESHAPE
    assert run(c=kvq(f, k_exp=None)) == B.SB_EINVAL
    assert lib.sb_tree_verify_kvq(None, C.byref(sq), C.byref(t), q, 0, 0, out,
                                  None) == B.SB_EINVAL
    go = lambda c, d: lib.sb_commit_kvq(  # noqa: E731
        ctx, C.byref(sq), C.byref(t), out, acc, c, d, None)
    d = kv(f, n_layers=1)
    assert go(None, d) == B.SB_EINVAL and go(q, None) == B.SB_EINVAL
    assert go(kvq(f, n_layers=1), d) == B.SB_ESHAPE
    assert go(q, kv(f, n_layers=2)) == B.SB_ESHAPE
    assert lib.sb_commit_kvq(None, C.byref(sq), C.byref(t), out, acc, q, d,
                             None) == B.SB_EINVAL


def test_unbound_context(lib):  # noqa: F811
    f = Fake()
    ctx = C.c_void_p()
    assert lib.sb_create(C.byref(cfg()), C.byref(ctx)) == B.SB_OK
    sq = B.Seqs(1, f.at(), f.at(), f.at())
    t = B.Tree(*[f.at()] * len(B.TREE_FIELDS))
    out = B.VerifyOut(f.at(), f.at(), None)
    assert lib.sb_tree_verify_kvq(ctx, C.byref(sq), C.byref(t), kvq(f), 0, 0,
                                  C.byref(out), None) == B.SB_ESTATE
    acc = B.AcceptOut(f.at(), f.at(), f.at(), None)
    assert lib.sb_commit_kvq(ctx, C.byref(sq), C.byref(t), C.byref(out), C.byref(acc),
                             kvq(f), kv(f, n_layers=1), None) == B.SB_ESTATE
    lib.sb_destroy(ctx)


PAST = [2 ** 31, 2 ** 32, -1]


@pytest.mark.parametrize("name", ["window", "sinks", "max_prefix", "n_rows", "rows_per_seq"])
@pytest.mark.parametrize("value", PAST)
def test_handles_refuse_what_int32_does_not_hold(name, value):
    """Values that would reach the library as their low 32 bits."""
    sh = kvcache.Shape(8, 2, 64, "bf16", 4, 10)
    cache = types.SimpleNamespace(shape=sh, device=torch.device("cpu"))
    z = torch.zeros(3, dtype=torch.int32)
    args = dict(n_rows=1, rows_per_seq=1, max_prefix=0, window=0, sinks=0)
    args[name] = value
    with pytest.raises(ValueError, match=name):
        kvcache.Attention(cache, z, None, z[:2], **args)


@pytest.mark.parametrize("value", PAST)
def test_stores_and_grows_refuse_what_int32_does_not_hold(value):
    z = torch.zeros(2, dtype=torch.int32)
    store = kvcache.QuantKV.__new__(kvcache.QuantKV)
    with pytest.raises(ValueError, match="max_entries"):
        store.store(None, z, z, value)
    pool = kvcache.PagePool.__new__(kvcache.PagePool)
    with pytest.raises(ValueError, match="extra"):
        pool.grow(z, value)


@pytest.mark.parametrize("left_out", ["seg_len", "vis", "seg_k", "seg_v"])
def test_a_segment_is_given_whole(left_out):
    sh = kvcache.Shape(8, 2, 64, "bf16", 4, 10)
    cache = types.SimpleNamespace(shape=sh, device=torch.device("cpu"))
    z = torch.zeros(3, dtype=torch.int32)
    seg = dict(seg_len=z, vis=z, seg_k=z, seg_v=z)
    seg[left_out] = None
    with pytest.raises(ValueError, match="segment"):
        kvcache.Attention(cache, z, None, z[:2], n_rows=1, rows_per_seq=1, **seg)


def test_a_window_needs_the_8_bit_cache():
    for kw in (dict(window=8), dict(sinks=2)):
        with pytest.raises(ValueError, match="8-bit"):
            Runtime(None, **kw)
    with pytest.raises(ValueError, match="window"):
        Runtime(None, kvq=True, window=2 ** 32)


def test_layers_and_sequences_that_int32_does_not_hold():
    plan = kvcache.Attention.__new__(kvcache.Attention)
    plan._layers = 3
    for layer in (-1, 3, 2 ** 32):
        with pytest.raises(ValueError, match="layer"):
            plan(layer, None)
    pool = kvcache.PagePool.__new__(kvcache.PagePool)
    for s in PAST:
        with pytest.raises(ValueError, match="sequence"):
            pool.release([0, s])
        with pytest.raises(ValueError, match="sequence"):
            pool.fork([0], [s], None)
        with pytest.raises(ValueError, match="sequence"):
            pool.fork([s], [1], None)
