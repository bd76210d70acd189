"""Measured cases of the 8-bit K/V cache: attention over it, storing into it, and its page pool.

Three operators, each in a plain form (elementary torch operations in 32 bits)
and, with ``own`` true, through this package's entry points
(``paper_2605_07243_amd.kvcache``):

* ``attend``: rows (nodes of draft trees, single tokens) of several sequences
  against a paged cache held as e4m3 codes with one power-of-two scale per
  page of 16 entries, KV head and K / V, plus a bf16 or fp32 segment of the
  rows' own keys under visibility bits; optionally only the first ``sinks``
  entries and a ``window`` of the last ones;
* ``store``: entries of a paged bf16 / fp32 cache into the 8-bit one;
* ``fork`` and ``compact``: sequences that share pages, and live pages moved
  to the front of their pool.

Layouts: K page ``[Hkv][16][hd]`` (both caches), V page ``[Hkv][hd][16]``
(elem cache and segment); 8-bit V page ``[Hkv][4][16][hd/16][4]``: entry
4 a + d, column 16 c + r at ``[a][r][c][d]``.
"""
import math

import numpy as np
import torch

own = False

F8 = torch.float8_e4m3fn


# ---------------------------------------------------------------- cases
def _attend(name, dtype, H, Hkv, hd, seqs, lo, hi, rows, window=0, sinks=0):
    return dict(name=name, op="attend", dtype=dtype, H=H, Hkv=Hkv, hd=hd,
                seqs=seqs, lo=lo, hi=hi, rows=rows, window=window, sinks=sinks)


def _store(name, dtype, Hkv, hd, layers, seqs, lo, hi, new):
    return dict(name=name, op="store", dtype=dtype, Hkv=Hkv, hd=hd,
                layers=layers, seqs=seqs, lo=lo, hi=hi, new=new)


def listed():
    return [
        # one token of one sequence after a prompt of 1024 (8B heads)
        _attend("decode-1", "bf16", 32, 8, 128, 1, 1024, 1024, 1),
        # the tree of the default benchmark: 60 nodes, 1024 committed entries
        _attend("tree-8b", "bf16", 32, 8, 128, 1, 1024, 1024, 60),
        # 16 ragged sequences, trees of up to 64 nodes
        _attend("tree-8b-batch16", "bf16", 32, 8, 128, 16, 512, 2048, 64),
        # 70B heads: 4 trees of 96 nodes over 2048 entries
        _attend("tree-70b-batch4", "bf16", 64, 8, 128, 4, 2048, 2048, 96),
        # a full house of long sequences, a token each
        _attend("decode-64-long", "bf16", 32, 8, 128, 64, 4096, 32768, 1),
        # trees over very long streams that see 4 sinks and the last 4096
        _attend("window-long", "bf16", 32, 8, 128, 8, 40000, 100000, 33, 4096, 4),
        # a tree at the budget's limit over a long prompt
        _attend("tree-512", "bf16", 32, 8, 128, 1, 8192, 8192, 512),
        # the toy fp32 model: 64-wide heads, no grouping
        _attend("tree-tiny-fp32", "f32", 4, 4, 64, 1, 128, 128, 32),
        # a batch of prompts into the 8-bit cache, 8 layers
        _store("store-prompts", "bf16", 8, 128, 8, 16, 512, 2048, 0),
        # the entries that one iteration adds (1 to 9) to pages in use
        _store("store-append", "bf16", 8, 128, 32, 16, 512, 2048, 9),
        # one prompt of 1003 entries shared by 15 continuations
        dict(name="fork-15", op="fork", Hkv=8, hd=128, layers=32, seqs=16,
             pages=80, lo=1003, hi=1003),
        # half of 64 sequences have left: the others' pages move up
        dict(name="compact-64", op="compact", Hkv=8, hd=128, layers=8,
             seqs=64, pages=128, lo=700, hi=2000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "store", "fork", "compact"])
    hd = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 4, 8])
    if op == "attend":
        H = Hkv * rng.choice([1, 2, 4, 5, 8])
        seqs = _log(rng, 1, 64)
        rows = _log(rng, 1, 512)
        # at most 2^31 codes in all, and 2^27 (row, entry, head) products
        most = min(100000, (1 << 30) // (seqs * Hkv * hd),
                   (1 << 27) // (seqs * rows * H))
        hi = _log(rng, 1, max(1, most))
        lo = max(1, hi - _log(rng, 1, hi))
        window, sinks = 0, 0
        if rng.random() < 0.4:
            window, sinks = _log(rng, 1, 2 * hi), rng.choice([0, 1, 4, 17])
        return {k: v for k, v in _attend(
            "", rng.choice(["bf16", "bf16", "f32"]), H, Hkv, hd, seqs, lo, hi,
            rows, window, sinks).items() if k != "name"}
    if op == "store":
        seqs, layers = _log(rng, 1, 32), _log(rng, 1, 16)
        hi = _log(rng, 1, max(1, min(4096, (1 << 27) // (seqs * layers * Hkv * hd))))
        lo = max(1, hi - _log(rng, 1, hi))
        new = rng.choice([0, _log(rng, 1, 64)])
        return {k: v for k, v in _store(
            "", rng.choice(["bf16", "bf16", "f32"]), Hkv, hd, layers, seqs, lo,
            hi, new).items() if k != "name"}
    layers, seqs = _log(rng, 1, 8), rng.randint(2, 64)
    pages = _log(rng, 2, max(2, min(200, (1 << 29) // (seqs * layers * Hkv * hd * 32))))
    hi = rng.randint(1, 16 * pages - 1)
    lo = rng.randint(1, hi)
    return dict(op=op, Hkv=Hkv, hd=hd, layers=layers, seqs=seqs, pages=pages,
                lo=lo, hi=hi)


# ---------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + 17)
    return g


def _elem(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lens(case, rng):
    return rng.integers(case["lo"], case["hi"] + 1, case["seqs"]).astype(np.int32)


def _codes(shape, g):
    """Codes as a page quantised to its own largest value holds them."""
    out = torch.empty(shape, dtype=torch.uint8, device="cuda")
    flat = out.view(-1)
    step = 1 << 27
    for i in range(0, flat.numel(), step):
        n = min(step, flat.numel() - i)
        x = torch.randn(n, generator=g, device="cuda").mul_(90.0).clamp_(-448.0, 448.0)
        flat[i:i + n] = x.to(F8).view(torch.uint8)
    return out


def _exps(shape, g):
    """Scale bytes: values of a few units, pages of differing size."""
    return torch.randint(119, 123, shape, generator=g, device="cuda",
                         dtype=torch.int32).to(torch.uint8)


def _values(shape, g, dtype, hd_dim):
    """K / V values with a few large channels."""
    x = torch.randn(shape, generator=g, device="cuda")
    big = 1.0 + 7.0 * (torch.rand(shape[hd_dim], generator=g, device="cuda") < 0.05).float()
    view = [1] * len(shape)
    view[hd_dim] = shape[hd_dim]
    return x.mul_(big.view(view)).to(dtype)


def _table(rng, seqs, max_pages, n_pages):
    return torch.from_numpy(rng.permutation(n_pages)[:seqs * max_pages].astype(
        np.int32).reshape(seqs, max_pages)).cuda()


def _prepare_attend(case, seed):
    g, rng = _gen(seed), np.random.default_rng([seed, 1])
    S, R, H, Hkv, hd = (case[k] for k in ("seqs", "rows", "H", "Hkv", "hd"))
    T = _lens(case, rng)
    max_pages = (case["hi"] + R + 15) // 16
    n_pages = S * max_pages
    # tree sizes go with the case, so that every seed has as many rows
    rows = np.random.default_rng([R, S]).integers(max(1, R - R // 3), R + 1, S).astype(np.int32)
    words, seg_pages = (R + 31) // 32, (R + 15) // 16
    off = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    vis = np.zeros((off[-1], words), np.uint32)
    pos = np.zeros(off[-1], np.int32)
    for s in range(S):      # a random tree per sequence
        for i in range(rows[s]):
            a = off[s] + i
            pos[a] = T[s]
            if i:
                p = off[s] + int(rng.integers(max(0, i - 8), i))
                vis[a] = vis[p]
                pos[a] = pos[p] + 1
            vis[a, i // 32] |= np.uint32(1 << (i % 32))
    dt = _elem(case)
    n = int(off[-1])
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    s = dict(
        case=case, k=_codes((1, n_pages, Hkv, 16 * hd), g),
        v=_codes((1, n_pages, Hkv, 16 * hd), g), k_exp=_exps((1, n_pages, Hkv), g),
        v_exp=_exps((1, n_pages, Hkv), g),
        page_table=_table(rng, S, max_pages, n_pages), row_off=dev(off), pos=dev(pos),
        prefix_len=dev(T), seg_len=dev(rows), vis=dev(vis.view(np.int32)),
        q=(torch.randn(n, H, hd, generator=g, device="cuda") * 0.9).to(dt),
        seg_k=_values((S, seg_pages, Hkv, 16, hd), g, dt, 4),
        seg_v=_values((S, seg_pages, Hkv, hd, 16), g, dt, 3),
        out=torch.empty(n, H, hd, dtype=dt, device="cuda"), max_prefix=int(T.max()))
    if own:     # what a program keeps: the cache's handle and the plan of its rows
        from paper_2605_07243_amd import kvcache as kc
        shape = kc.Shape(H, Hkv, hd, case["dtype"], S, max_pages)
        cache = kc.QuantKV(shape, s["k"], s["v"], s["k_exp"], s["v_exp"], s["page_table"])
        s["attend"] = kc.Attention(
            cache, s["row_off"], s["pos"], s["prefix_len"], s["seg_len"], s["vis"],
            s["seg_k"], s["seg_v"], n_rows=n, rows_per_seq=int(rows.max()),
            max_prefix=s["max_prefix"], window=case["window"], sinks=case["sinks"])
    return s


def _prepare_store(case, seed):
    g, rng = _gen(seed), np.random.default_rng([seed, 2])
    S, L, Hkv, hd = (case[k] for k in ("seqs", "layers", "Hkv", "hd"))
    T = _lens(case, rng)
    new = rng.integers(1, case["new"] + 1, S).astype(np.int32) if case["new"] else T
    max_pages = (case["hi"] + case["new"] + 15) // 16
    n_pages = S * max_pages
    first = T if case["new"] else np.zeros_like(T)
    dt = _elem(case)
    s = dict(
        case=case, src_k=_values((L, n_pages, Hkv, 16, hd), g, dt, 4),
        src_v=_values((L, n_pages, Hkv, hd, 16), g, dt, 3),
        src_table=_table(rng, S, max_pages, n_pages),
        k=_codes((L, n_pages, Hkv, 16 * hd), g), v=_codes((L, n_pages, Hkv, 16 * hd), g),
        k_exp=_exps((L, n_pages, Hkv), g), v_exp=_exps((L, n_pages, Hkv), g),
        page_table=_table(rng, S, max_pages, n_pages),
        first=torch.from_numpy(first).cuda(), last=torch.from_numpy(first + new).cuda(),
        most=int(new.max()))
    if own:
        from paper_2605_07243_amd import kvcache as kc
        shape = kc.Shape(Hkv, Hkv, hd, case["dtype"], S, max_pages)
        s["src"] = kc.PagedKV(shape, s["src_k"], s["src_v"], s["src_table"])
        s["dst"] = kc.QuantKV(shape, s["k"], s["v"], s["k_exp"], s["v_exp"], s["page_table"])
    return s


def _prepare_pool(case, seed):
    g, rng = _gen(seed), np.random.default_rng([seed, 3])
    S, L, Hkv, hd, mp = (case[k] for k in ("seqs", "layers", "Hkv", "hd", "pages"))
    n_pages = S * mp
    T = _lens(case, rng)
    table = np.zeros((S, mp), np.int32)
    held = np.zeros(S, np.int32)
    perm = rng.permutation(n_pages)
    if case["op"] == "fork":
        live = [0]              # sequence 0 holds its prompt's pages
    else:                       # sequences that are still there
        live = [s for s in range(S) if rng.random() < 0.5] or [0]
    at = 0
    refs = np.zeros(n_pages, np.int32)
    for s in live:
        held[s] = (T[s] + 15) // 16
        table[s, :held[s]] = perm[at:at + held[s]]
        at += held[s]
        refs[table[s, :held[s]]] = 1
    if case["op"] == "compact" and len(live) > 1:   # a shared prompt among them
        a, b = live[0], live[1]
        n = min(held[a], held[b]) // 2
        refs[table[b, :n]] -= 1
        table[b, :n] = table[a, :n]
        refs[table[a, :n]] += 1
    meta = np.concatenate([table.ravel(), held, refs, np.zeros(1, np.int32)])
    s = dict(
        case=case, k=_codes((L, n_pages, Hkv, 16 * hd), g),
        v=_codes((L, n_pages, Hkv, 16 * hd), g), k_exp=_exps((L, n_pages, Hkv), g),
        v_exp=_exps((L, n_pages, Hkv), g), before=torch.from_numpy(meta).cuda(),
        lens=torch.from_numpy(T).cuda())
    s["meta"] = s["before"].clone()
    m, i = s["meta"], 0
    for name, n in (("table", S * mp), ("held", S), ("refs", n_pages), ("refused", 1)):
        s[name] = m[i:i + n]
        i += n
    s["table"] = s["table"].view(S, mp)
    s["children"] = list(range(1, S))
    if own:
        from paper_2605_07243_amd import kvcache as kc
        shape = kc.Shape(Hkv, Hkv, hd, "bf16", S, mp)
        cache = kc.QuantKV(shape, s["k"], s["v"], s["k_exp"], s["v_exp"], s["table"])
        s["pool"] = kc.PagePool(shape, s["table"], s["held"], s["refs"], s["refused"],
                                [cache])
    return s


def prepare(case, seed):
    if case["op"] == "attend":
        return _prepare_attend(case, seed)
    if case["op"] == "store":
        return _prepare_store(case, seed)
    return _prepare_pool(case, seed)


# ---------------------------------------------------------------- plain forms
def _plain_attend(s):
    c = s["case"]
    S, H, Hkv, hd = (c[k] for k in ("seqs", "H", "Hkv", "hd"))
    q, dt = s["q"], s["q"].dtype
    N, G = q.shape[0], H // Hkv
    off = s["row_off"].long()
    row = torch.arange(N, device="cuda")
    seq = torch.searchsorted(off[1:], row, right=True)
    at = row - off[seq]
    R = c["rows"]
    qp = torch.zeros(S, R, H, hd, device="cuda")
    qp[seq, at] = q.float()
    qp = qp.view(S, R, Hkv, G, hd).permute(0, 2, 3, 1, 4).reshape(S, Hkv, G * R, hd)
    P = (s["max_prefix"] + 15) // 16
    pages = s["page_table"][:, :P].long()
    scale = lambda e: torch.exp2(e.float() - 127.0)  # noqa: E731
    k = s["k"][0][pages].view(F8).float() * scale(s["k_exp"][0][pages])[..., None]
    k = k.view(S, P, Hkv, 16, hd).permute(0, 2, 1, 3, 4).reshape(S, Hkv, P * 16, hd)
    v = s["v"][0][pages].view(F8).float() * scale(s["v_exp"][0][pages])[..., None]
    v = v.view(S, P, Hkv, 4, 16, hd // 16, 4).permute(0, 2, 1, 3, 6, 5, 4)
    v = v.reshape(S, Hkv, P * 16, hd)
    n_seg = s["seg_k"].shape[1] * 16
    sk = s["seg_k"].float().permute(0, 2, 1, 3, 4).reshape(S, Hkv, n_seg, hd)
    sv = s["seg_v"].float().permute(0, 2, 1, 4, 3).reshape(S, Hkv, n_seg, hd)
    # what each row sees
    pos = torch.zeros(S, R, dtype=torch.int64, device="cuda")
    pos[seq, at] = s["pos"].long()
    e = torch.arange(P * 16, device="cuda")
    ok = (e < s["prefix_len"][:, None])[:, None, :]
    if c["window"]:
        ok = ok & ((e < c["sinks"]) | (e > pos[..., None] - c["window"]))
    else:
        ok = ok.expand(S, R, P * 16)
    slot = torch.arange(n_seg, device="cuda")
    word = (slot // 32).clamp(max=s["vis"].shape[1] - 1)
    bits = torch.zeros(S, R, n_seg, dtype=torch.bool, device="cuda")
    bits[seq, at] = ((s["vis"][:, word] >> (slot % 32)) & 1).bool()
    bits &= (slot < s["seg_len"][:, None])[:, None, :]
    sc = torch.cat([qp @ k.transpose(2, 3), qp @ sk.transpose(2, 3)], 3)
    see = torch.cat([ok, bits], 2)[:, None, None].expand(S, Hkv, G, R, -1)
    see = see.reshape(S, Hkv, G * R, -1)
    sc = (sc * (1.0 / math.sqrt(hd))).masked_fill_(~see, float("-inf"))
    m = sc.amax(3, keepdim=True).clamp(min=-3e38)
    p = torch.exp(sc - m)
    o = (p[..., :P * 16] @ v + p[..., P * 16:] @ sv) / p.sum(3, keepdim=True).clamp(min=1e-30)
    o = o.view(S, Hkv, G, R, hd).permute(0, 3, 1, 2, 4).reshape(S, R, H, hd)
    s["out"].copy_(o[seq, at].to(dt))
    return s["out"]


def _requant(x, new, held_codes, held, held_exp):
    """Codes and scale byte of a page: x, new and held over its entries in the
    last axis but one ([..., 16, hd]); held_exp [...]."""
    x = x.float()
    fine = new & torch.isfinite(x)
    amax = torch.where(fine, x.abs(), 0.0).amax((-1, -2))
    mant, ex = torch.frexp(amax)
    need = torch.where(amax > 0, ex - 8 - (mant <= 0.875).int(), -126).clamp(min=-126)
    any_held = held.any(-1).any(-1)
    e = torch.where(any_held, torch.maximum(need, held_exp.int() - 127), need)
    y = torch.ldexp(x, -e[..., None, None])
    y = torch.where(torch.isfinite(x), y, float("nan")).to(F8).view(torch.uint8)
    old = held_codes.view(F8).float()
    moved = torch.ldexp(old, (held_exp.int() - 127 - e).clamp(min=-60)[..., None, None])
    old = moved.to(F8).view(torch.uint8)
    codes = torch.where(new, y, torch.where(held, old, held_codes))
    return codes, (e + 127).to(torch.uint8)


def _plain_store(s):
    c = s["case"]
    S, L, Hkv, hd = (c[k] for k in ("seqs", "layers", "Hkv", "hd"))
    first, last = s["first"].long(), s["last"].long()
    P = (s["most"] + 15) // 16 + 1
    page = first[:, None] // 16 + torch.arange(P, device="cuda")
    seq, j = torch.nonzero(page * 16 < last[:, None], as_tuple=True)
    page = page[seq, j]
    n = seq.numel()
    src, dst = s["src_table"][seq, page].long(), s["page_table"][seq, page].long()
    entry = page[:, None] * 16 + torch.arange(16, device="cuda")
    new = (entry >= first[seq][:, None]) & (entry < last[seq][:, None])
    new, held = new[:, None, :, None], (entry < first[seq][:, None])[:, None, :, None]
    k, e = _requant(s["src_k"][:, src], new, s["k"][:, dst].view(L, n, Hkv, 16, hd), held,
                    s["k_exp"][:, dst])
    s["k"][:, dst] = k.reshape(L, n, Hkv, 16 * hd)
    s["k_exp"][:, dst] = e
    old = s["v"][:, dst].view(L, n, Hkv, 4, 16, hd // 16, 4).permute(0, 1, 2, 3, 6, 5, 4)
    v, e = _requant(s["src_v"][:, src].transpose(3, 4), new, old.reshape(L, n, Hkv, 16, hd),
                    held, s["v_exp"][:, dst])
    v = v.view(L, n, Hkv, 4, 4, hd // 16, 16).permute(0, 1, 2, 3, 6, 5, 4)
    s["v"][:, dst] = v.reshape(L, n, Hkv, 16 * hd)
    s["v_exp"][:, dst] = e
    return _cache_out(s)


def _cache_out(s):
    return {"k": s["k"].view(F8), "v": s["v"].view(F8), "k_exp": s["k_exp"],
            "v_exp": s["v_exp"]}


def _pool_out(s):
    return {**_cache_out(s), "table": s["table"], "held": s["held"], "refs": s["refs"],
            "refused": s["refused"]}


def _plain_fork(s):
    table, held, refs = s["table"], s["held"], s["refs"]
    col = torch.arange(table.shape[1], device="cuda")
    child = torch.tensor(s["children"], device="cuda")
    # the children's own pages go back first
    gone = table[child].long()[col < held[child][:, None]]
    refs.index_add_(0, gone, torch.full_like(gone, -1, dtype=torch.int32))
    n_full, part = s["lens"][0] // 16, (s["lens"][0] % 16 != 0).long()
    full = col < n_full
    table[child[:, None], col] = torch.where(full, table[0], table[child])
    refs.index_add_(0, table[0].long(), full.int() * child.numel())
    free = torch.nonzero(refs == 0).flatten()
    rank = torch.arange(child.numel(), device="cuda")
    got = (rank < free.numel()) & (part > 0)
    new = free[rank.clamp(max=free.numel() - 1)]
    c2, n2 = child[got], new[got]
    src = table[0][n_full.long()].long().expand(c2.numel())
    table[c2, n_full.long()] = n2.int()
    refs[n2] = 1
    held[child] = (n_full + got.int()).int()
    s["refused"] += ((part > 0) & ~got).sum().int()
    for t in (s["k"], s["v"], s["k_exp"], s["v_exp"]):
        t[:, n2] = t[:, src]
    return _pool_out(s)


def _plain_compact(s):
    table, held, refs = s["table"], s["held"], s["refs"]
    n = refs.numel()
    page = torch.arange(n, device="cuda")
    n_live = (refs > 0).sum()
    src = torch.nonzero((refs > 0) & (page >= n_live)).flatten()
    dst = torch.nonzero((refs == 0) & (page < n_live)).flatten()
    for t in (s["k"], s["v"], s["k_exp"], s["v_exp"]):
        t[:, dst] = t[:, src]
    to = page.int()
    to[src] = dst.int()
    col = torch.arange(table.shape[1], device="cuda")
    table.copy_(torch.where(col < held[:, None], to[table.long()], table))
    refs[dst] = refs[src]
    refs[src] = 0
    return _pool_out(s)


def run(s):
    op = s["case"]["op"]
    if op == "attend":
        if own:
            return s["attend"](0, s["q"], s["out"])
        return _plain_attend(s)
    if op == "store":
        if own:
            s["dst"].store(s["src"], s["first"], s["last"], s["most"])
            return _cache_out(s)
        return _plain_store(s)
    s["meta"].copy_(s["before"])    # the sequences as they were
    if op == "fork":
        if own:
            s["pool"].fork([0] * len(s["children"]), s["children"], s["lens"])
            return _pool_out(s)
        return _plain_fork(s)
    if own:
        s["pool"].compact()
        return _pool_out(s)
    return _plain_compact(s)


# ---------------------------------------------------------------- work
def work(case):
    """Bytes read and written once, and operations, at the mean sizes."""
    op, hd, Hkv = case["op"], case["hd"], case["Hkv"]
    mean = (case["lo"] + case["hi"]) / 2.0
    if op == "attend":
        es = 2 if case["dtype"] == "bf16" else 4
        R = case["rows"] - (case["rows"] // 3) / 2.0
        seen = min(mean, case["window"] + case["sinks"]) if case["window"] else mean
        S, H = case["seqs"], case["H"]
        kv = S * Hkv * (seen * 2 * (hd + 1 / 16) + R * 2 * hd * es)
        return {"bytes": kv + S * R * H * hd * 2 * es,
                "flops": 4.0 * S * R * H * hd * (seen + R / 4)}
    page = Hkv * (32 * hd + 2)
    if op == "store":
        es = 2 if case["dtype"] == "bf16" else 4
        new = (1 + case["new"]) / 2.0 if case["new"] else mean
        return {"bytes": case["seqs"] * case["layers"] * Hkv * new * 2 * hd * (es + 1),
                "flops": 0}
    if op == "fork":
        moved = (case["seqs"] - 1) * (15 / 16 if case["lo"] != case["hi"]
                                      else float(case["lo"] % 16 != 0))
        shared = (case["seqs"] - 1) * mean / 16
        return {"bytes": 2.0 * moved * case["layers"] * page + 8 * shared
                + 4 * case["seqs"] * case["pages"] + 64, "flops": 0}
    live = case["seqs"] / 2.0 * (mean / 16 + 0.5)
    share = live / (case["seqs"] * case["pages"])
    return {"bytes": 2.0 * live * (1 - share) * case["layers"] * page
            + 8 * case["seqs"] * case["pages"], "flops": 0}


# ---------------------------------------------------------------- 64 bits
def _e4m3(x):
    """Nearest e4m3 value (ties to even) of float64 values within +-448."""
    a = x.abs()
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _values_of(codes, ex):
    return codes.view(F8).double() * torch.exp2(ex.double() - 127)[..., None]


def _exact_attend(s):
    c = s["case"]
    H, Hkv, hd = c["H"], c["Hkv"], c["hd"]
    G, off = H // Hkv, s["row_off"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b in range(c["seqs"]):
        T, n = int(s["prefix_len"][b]), int(s["seg_len"][b])
        pg = s["page_table"][b, :(T + 15) // 16].long()
        rows = slice(off[b], off[b + 1])
        pos = s["pos"][rows].long()
        e = torch.arange(T, device="cuda")
        see = torch.ones(len(pos), T, dtype=torch.bool, device="cuda")
        if c["window"]:
            see = (e < c["sinks"]) | (e >= pos[:, None] + 1 - c["window"])
        slot = torch.arange(n, device="cuda")
        see = torch.cat([see, ((s["vis"][rows][:, slot // 32] >> (slot % 32)) & 1) == 1], 1)
        used = torch.nonzero(see.any(0)).flatten()
        for h in range(Hkv):
            k = _values_of(s["k"][0, pg, h], s["k_exp"][0, pg, h]).view(-1, hd)[:T]
            v = _values_of(s["v"][0, pg, h], s["v_exp"][0, pg, h])
            v = v.view(-1, 4, 16, hd // 16, 4).permute(0, 1, 4, 3, 2).reshape(-1, hd)[:T]
            k = torch.cat([k, s["seg_k"][b, :, h].reshape(-1, hd)[:n].double()])[used]
            v = torch.cat([v, s["seg_v"][b, :, h].transpose(1, 2).reshape(-1, hd)[:n].double()])[used]
            for j in range(G):
                z = s["q"][rows, h * G + j].double() @ k.T / math.sqrt(hd)
                z = torch.where(see[:, used], z, -torch.inf)
                p = torch.nan_to_num(torch.softmax(z, 1), nan=0.0)
                out[rows, h * G + j] = p @ v
    return out


def _exact_store(s):
    """Every value that the caches hold afterwards, in the units of its page's
    scale: held codes stay where no larger value joins their page."""
    c = s["case"]
    hd = c["hd"]
    out = {n: s[n].view(F8).double() for n in ("k", "v")}
    for b in range(c["seqs"]):
        lo, hi = int(s["first"][b]), int(s["last"][b])
        for p in range(lo // 16, (hi + 15) // 16):
            src, dst = int(s["src_table"][b, p]), int(s["page_table"][b, p])
            a, z = max(lo - 16 * p, 0), min(hi - 16 * p, 16)
            for n in ("k", "v"):
                x = s["src_" + n][:, src].double()
                x = x if n == "k" else x.transpose(2, 3)        # [L, Hkv, 16, hd]
                x = x[:, :, a:z]
                top = x.abs().amax((2, 3))
                # the least power of two that brings the largest to 448
                e = torch.ceil(torch.log2(top / 448.0).clamp(min=-126.0))
                was = s[n + "_exp"][:, dst].double() - 127
                if a:
                    e = torch.maximum(e, was)
                e4 = e[:, :, None, None]
                page = out[n][:, dst]
                if n == "k":
                    page = page.view(*page.shape[:2], 16, hd)
                else:
                    page = page.view(*page.shape[:2], 4, 16, hd // 16, 4).permute(
                        0, 1, 2, 5, 4, 3).reshape(*page.shape[:2], 16, hd)
                page = page.clone()
                page[:, :, :a] = _e4m3(page[:, :, :a] * torch.exp2(was[:, :, None, None] - e4))
                page[:, :, a:z] = _e4m3(x * torch.exp2(-e4))
                if n == "v":
                    page = page.view(*page.shape[:2], 4, 4, hd // 16, 16).permute(
                        0, 1, 2, 5, 4, 3)
                out[n][:, dst] = page.reshape(*page.shape[:2], 16 * hd)
    return {"k": out["k"], "v": out["v"], "k_exp": None, "v_exp": None}


def exact(case, seed):
    if case["op"] == "attend":
        if case["seqs"] * case["hi"] * case["Hkv"] > 1 << 24:
            return None
        return _exact_attend(_prepare_attend(case, seed))
    if case["op"] == "store":
        if case["seqs"] * max(case["new"], case["hi"] * (not case["new"])) > 1 << 16:
            return None
        return _exact_store(_prepare_store(case, seed))
    return None                 # pages are moved: nothing is computed
