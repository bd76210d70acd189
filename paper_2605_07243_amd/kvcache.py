"""The 8-bit K/V cache and the page pool of libspecblock.so over torch tensors.

Thin handles around the ``sb_kvq_*`` and ``sb_pool_*`` calls: they check the
tensors they are given (type, shape, layout, device), keep them alive and
marshal arguments; every step runs in the library's HIP kernels on the current
stream of the tensors' device.  Nothing here waits for the device.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import binding as B


def _tensor(t, name, dtype, shape, device=None):
    """The tensor's address, after checking what the kernels rely on."""
    if (not isinstance(t, torch.Tensor) or t.dtype != dtype
            or tuple(t.shape) != tuple(shape) or not t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape "
                         f"{tuple(shape)}")
    if not t.is_cuda or (device is not None and t.device != device):
        raise ValueError(f"{name} must be on the GPU of the other tensors")
    return C.c_void_p(t.data_ptr())


def int32(x, name, least=0):
    """x as an int32 argument (ctypes would cut it to its low bits)."""
    x = int(x)
    if not least <= x < 1 << 31:
        raise ValueError(f"{name} must be in {least} .. 2^31 - 1")
    return x


def _seqs(seqs):
    """A host list of sequences."""
    return (C.c_int32 * max(1, len(seqs)))(*(int32(s, "a sequence") for s in seqs))


# handle of the current stream of a device (the integer alone: building a
# torch.cuda.Stream for it costs as much as the rest of a call)
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda i: torch.cuda.current_stream(i).cuda_stream)


def _call(device, fn, *args):
    """fn(*args, stream) with the tensors' device current; raises SBError."""
    if torch.cuda.current_device() == device.index:
        rc = fn(*args, _stream(device.index))
    else:
        with torch.cuda.device(device):
            rc = fn(*args, _stream(device.index))
    if rc != B.SB_OK:
        B.check(B.load(), None, rc)


class _Scratch:
    """Device memory that a handle allocates for the library's work, on the
    stream that is current then."""

    def __init__(self, n, dtype, device):
        self.t = torch.empty(n, dtype=dtype, device=device)
        self.home = _stream(device.index)

    def used(self):
        """After a call that uses it on the current stream: when the handle is
        dropped, the memory waits for that stream too."""
        if _stream(self.t.device.index) != self.home:
            self.t.record_stream(torch.cuda.current_stream(self.t.device))


class Shape:
    """sb_cache_shape: heads, element type ("bf16" or "f32") and page tables."""

    def __init__(self, n_heads, n_kv_heads, head_dim, dtype, max_seqs, max_pages):
        if dtype not in ("bf16", "f32"):
            raise ValueError('dtype must be "bf16" or "f32"')
        self.n_heads, self.n_kv_heads, self.head_dim = n_heads, n_kv_heads, head_dim
        self.max_seqs, self.max_pages, self.dtype = max_seqs, max_pages, dtype
        self.elem = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.c = B.CacheShape(n_heads, n_kv_heads, head_dim,
                              B.SB_BF16 if dtype == "bf16" else B.SB_F32,
                              max_seqs, max_pages)


class PagedKV:
    """sb_kv over tensors: k [layers][pages][Hkv][16][hd], v [..][hd][16]."""

    def __init__(self, shape, k, v, page_table):
        self.shape, self.k, self.v, self.page_table = shape, k, v, page_table
        L, n = k.shape[:2]
        hkv, hd, dev = shape.n_kv_heads, shape.head_dim, k.device
        self.device = dev
        self.c = B.KV(_tensor(k, "k", shape.elem, (L, n, hkv, 16, hd)),
                      _tensor(v, "v", shape.elem, (L, n, hkv, hd, 16), dev),
                      _tensor(page_table, "page_table", torch.int32,
                              (shape.max_seqs, shape.max_pages), dev), L, n)


class QuantKV:
    """sb_kvq over tensors: codes uint8 [layers][pages][Hkv][16 hd], scale
    bytes uint8 [layers][pages][Hkv]."""

    def __init__(self, shape, k, v, k_exp, v_exp, page_table):
        self.lib = B.load()
        self.shape, self.page_table = shape, page_table
        self.k, self.v, self.k_exp, self.v_exp = k, v, k_exp, v_exp
        L, n = k.shape[:2]
        hkv, dev = shape.n_kv_heads, k.device
        codes = (L, n, hkv, 16 * shape.head_dim)
        u8 = torch.uint8
        self.device = dev
        self.c = B.KVQ(_tensor(k, "k", u8, codes), _tensor(v, "v", u8, codes, dev),
                       _tensor(k_exp, "k_exp", u8, (L, n, hkv), dev),
                       _tensor(v_exp, "v_exp", u8, (L, n, hkv), dev),
                       _tensor(page_table, "page_table", torch.int32,
                               (shape.max_seqs, shape.max_pages), dev), L, n)

    @classmethod
    def empty(cls, shape, n_layers, n_pages, page_table):
        """A cache of n_pages pages (codes 0, scale 1) for the page table."""
        dev = page_table.device
        n = (n_layers, n_pages, shape.n_kv_heads)
        z = lambda: torch.zeros(*n, 16 * shape.head_dim, dtype=torch.uint8,  # noqa: E731
                                device=dev)
        e = lambda: torch.full(n, 127, dtype=torch.uint8, device=dev)  # noqa: E731
        return cls(shape, z(), z(), e(), e(), page_table)

    def store(self, src, first, last, max_entries):
        """Entries first[s] .. last[s] - 1 of ``src`` (a PagedKV) into this
        cache; first, last: int32 tensors [n_seqs]."""
        n, most = first.shape[0], int32(max_entries, "max_entries", 1)
        if src.shape.dtype != self.shape.dtype or src.device != self.device or (
                src.shape.n_kv_heads, src.shape.head_dim, src.shape.max_seqs,
                src.shape.max_pages) != (self.shape.n_kv_heads, self.shape.head_dim,
                                         self.shape.max_seqs, self.shape.max_pages):
            raise ValueError("the caches differ in shape or device")
        a = _tensor(first, "first", torch.int32, (n,), self.device)
        z = _tensor(last, "last", torch.int32, (n,), self.device)
        _call(self.device, self.lib.sb_kvq_store, self.shape.c, n, src.c, a, z,
              most, self.c)


class Attention:
    """sb_kvq_attend for one description of rows (sb_attn_rows) and one
    workspace: ``plan(layer, q, out)`` for every layer of a forward.  A plan
    runs on one stream at a time; captured graphs that may run at the same
    time need a plan each, which has to live as long as its graph.
    max_prefix bounds prefix_len (0: the page table's capacity) and sets how
    the work is split: the nearer to the lengths, the faster."""

    def __init__(self, cache, row_off, pos, prefix_len, seg_len=None, vis=None,
                 seg_k=None, seg_v=None, *, n_rows, rows_per_seq, max_prefix=0,
                 window=0, sinks=0):
        sh, dev = cache.shape, cache.device
        self.lib, self.cache, self.device = B.load(), cache, dev
        self.n_rows = n_rows = int32(n_rows, "n_rows", 1)
        self.window, self.sinks = int32(window, "window"), int32(sinks, "sinks")
        rows_per_seq = int32(rows_per_seq, "rows_per_seq", 1)
        max_prefix = int32(max_prefix, "max_prefix")
        given = [t is not None for t in (seg_len, vis, seg_k, seg_v)]
        if any(given) and not all(given):
            raise ValueError("a segment needs seg_len, vis, seg_k and seg_v")
        n = row_off.shape[0] - 1
        i32 = torch.int32
        null = C.c_void_p(0)
        words = pages = 0
        sl = vs = sk = sv = null
        if seg_k is not None:
            words, pages = vis.shape[1], seg_k.shape[1]
            hkv, hd = sh.n_kv_heads, sh.head_dim
            sl = _tensor(seg_len, "seg_len", i32, (n,), dev)
            vs = _tensor(vis, "vis", i32, (n_rows, words), dev)
            sk = _tensor(seg_k, "seg_k", sh.elem, (n, pages, hkv, 16, hd), dev)
            sv = _tensor(seg_v, "seg_v", sh.elem, (n, pages, hkv, hd, 16), dev)
        self.rows = B.AttnRows(
            n, n_rows, rows_per_seq, max_prefix, words, pages,
            _tensor(row_off, "row_off", i32, (n + 1,), dev),
            null if pos is None else _tensor(pos, "pos", i32, (n_rows,), dev),
            _tensor(prefix_len, "prefix_len", i32, (n,), dev), sl, vs, sk, sv)
        self._keep = (row_off, pos, prefix_len, seg_len, vis, seg_k, seg_v)
        nbytes = self.lib.sb_kvq_attend_workspace(sh.c, self.rows, self.window, self.sinks)
        if nbytes == 0:
            raise B.SBError(B.SB_ESHAPE, self.lib.sb_last_error(None).decode())
        self._scratch = _Scratch(nbytes, torch.uint8, dev)
        self.workspace = self._scratch.t
        self._ws = C.c_void_p(self.workspace.data_ptr())
        self._rows_shape = torch.Size((n_rows, sh.n_heads, sh.head_dim))
        self._nbytes, self._layers = nbytes, cache.c.n_layers
        self._attend = self.lib.sb_kvq_attend

    def _fits(self, t):
        return (t.dtype is self.cache.shape.elem and t.shape == self._rows_shape
                and t.device == self.device and t.is_contiguous())

    def __call__(self, layer, q, out=None):
        """Attention outputs of the rows, [n_rows][n_heads][head_dim]."""
        if not 0 <= layer < self._layers:
            raise ValueError(f"layer must be in 0 .. {self._layers - 1}")
        if (q.requires_grad or (out is not None and out.requires_grad)
                ) and torch.is_grad_enabled():
            raise ValueError("attention over the 8-bit cache has no backward pass: "
                             "call it under torch.no_grad() or on q.detach()")
        if out is None:
            out = torch.empty_like(q)
        if not (self._fits(q) and self._fits(out)):
            raise ValueError(
                f"q and out must be contiguous {self.cache.shape.elem} tensors of "
                f"shape {tuple(self._rows_shape)} on {self.device}")
        _call(self.device, self._attend, self.cache.shape.c, self.cache.c, layer,
              self.rows, q.data_ptr(), self.window, self.sinks, out.data_ptr(),
              self._ws, self._nbytes)
        self._scratch.used()
        return out


class PagePool:
    """sb_pool over tensors, with the caches whose pages it shares and moves
    (at most one PagedKV and one QuantKV, with the pool's page table).
    page_table entries at and past held[s] are -1 (no page): what a store or a
    commit would put there is dropped.  ``refused`` counts the requests for
    which there was no page; a caller that may run out looks at it."""

    def __init__(self, shape, page_table, held, refs, refused, caches=()):
        self.lib, self.shape, self.device = B.load(), shape, page_table.device
        dev, i32 = self.device, torch.int32
        self.page_table, self.held, self.refs, self.refused = page_table, held, refs, refused
        n = refs.shape[0]
        ints = self.lib.sb_pool_scratch_ints(n)
        if ints == 0:
            raise ValueError("a pool has 1 .. 2^20 pages")
        self._scratch = _Scratch(ints, i32, dev)
        self.scratch = self._scratch.t
        self.c = B.Pool(
            _tensor(page_table, "page_table", i32, (shape.max_seqs, shape.max_pages)),
            _tensor(held, "held", i32, (shape.max_seqs,), dev),
            _tensor(refs, "refs", i32, (n,), dev),
            _tensor(refused, "refused", i32, (1,), dev),
            C.c_void_p(self.scratch.data_ptr()), n)
        self.attach(caches)

    @classmethod
    def empty(cls, shape, n_pages, device="cuda"):
        """A pool of n_pages free pages with tables of its own."""
        z = lambda *n: torch.zeros(*n, dtype=torch.int32, device=device)  # noqa: E731
        return cls(shape, z(shape.max_seqs, shape.max_pages) - 1, z(shape.max_seqs),
                   z(n_pages), z(1))

    def attach(self, caches):
        """The caches that fork and compact copy from now on."""
        kv = [c for c in caches if isinstance(c, PagedKV)]
        kvq = [c for c in caches if isinstance(c, QuantKV)]
        if len(kv) > 1 or len(kvq) > 1 or len(kv) + len(kvq) != len(caches):
            raise ValueError("a pool takes at most one PagedKV and one QuantKV")
        for c in caches:
            if c.page_table.data_ptr() != self.page_table.data_ptr():
                raise ValueError("the cache goes through another page table")
            if (c.shape.n_kv_heads, c.shape.head_dim, c.shape.dtype,
                    c.shape.max_seqs, c.shape.max_pages) != (
                    self.shape.n_kv_heads, self.shape.head_dim, self.shape.dtype,
                    self.shape.max_seqs, self.shape.max_pages):
                raise ValueError("the cache has another shape")
        self._caches = list(caches)
        self._kv = kv[0].c if kv else None
        self._kvq = kvq[0].c if kvq else None

    def reset(self):
        _call(self.device, self.lib.sb_pool_reset, self.shape.c, self.c)

    def grow(self, length, extra=0):
        """Pages for length[s] + extra entries of sequences 0 .. n - 1
        (length: int32 tensor [n]); what there are of them, and refused counts
        the sequence, when the pool or the table runs out."""
        n, extra = length.shape[0], int32(extra, "extra")
        _call(self.device, self.lib.sb_pool_grow, self.shape.c, self.c, n,
              _tensor(length, "length", torch.int32, (n,), self.device), extra)

    def release(self, seqs):
        """The listed sequences return what they hold."""
        arr = _seqs(seqs)
        _call(self.device, self.lib.sb_pool_release, self.shape.c, self.c,
              len(seqs), arr)

    def fork(self, parents, children, length):
        """children[i] continues parents[i] after length[parents[i]] entries
        (length: int32 tensor [max_seqs]).  A child that refused counts holds
        the full pages alone: its length is 16 held."""
        n = len(parents)
        if len(children) != n:
            raise ValueError("as many children as parents")
        pa, ch = _seqs(parents), _seqs(children)
        _call(self.device, self.lib.sb_pool_fork, self.shape.c, self.c, n, pa, ch,
              _tensor(length, "length", torch.int32, (self.shape.max_seqs,),
                      self.device), self._kv, self._kvq)
        self._scratch.used()

    def compact(self):
        """Moves the pages in use to the front of the pool."""
        _call(self.device, self.lib.sb_pool_compact, self.shape.c, self.c,
              self._kv, self._kvq)
        self._scratch.used()
