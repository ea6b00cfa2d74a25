"""The operators of the shared, paged key-value cache, and the cases they are measured on.

Four operators: attention of packed prompt rows over the paged cache (causal, grouped heads, with or
without a prefix that is already cached), writing new K/V rows to their pages, forking sequences (which
also frees, rolls back and extends them) and compacting the pool. The pool is the framework's:
bf16 [layers, pages, 2 (K, V), kv_heads, 16 positions, head_dim], with int32 tables of page ids.

The plain forms below are elementary torch operations in 32 bits; `exact` is the definition in 64 bits.
"""
import math
import random

import torch

own = False

PAGE = 16

# (heads, kv_heads, head_dim, layers) of the decoders this repository runs.
TINY = (4, 4, 64, 4)
TINY_DRAFTER = (2, 2, 64, 2)
LLAMA_8B = (32, 8, 128, 32)
LLAMA_1B = (32, 8, 64, 16)
QWEN_32B = (40, 8, 128, 64)
QWEN_05B = (14, 2, 64, 24)
SHAPES = (TINY, TINY_DRAFTER, LLAMA_8B, LLAMA_1B, QWEN_32B, QWEN_05B)


# ---------------------------------------------------------------------------------------- cases
def _attention(shape, seqs, rows, prefix, mix, **kw):
    return dict(op="attention", heads=shape[0], kv_heads=shape[1], head_dim=shape[2], seqs=seqs, rows_lo=rows[0],
                rows_hi=rows[1], prefix_lo=prefix[0], prefix_hi=prefix[1], mix=mix, **kw)


def _append(shape, seqs, rows, prefix, dtype, mix, **kw):
    return dict(op="append", heads=shape[0], kv_heads=shape[1], head_dim=shape[2], seqs=seqs, rows_lo=rows[0],
                rows_hi=rows[1], prefix_lo=prefix[0], prefix_hi=prefix[1], dtype=dtype, mix=mix, **kw)


def _fork(shape, layers, seqs, lens, children, grow, mix, **kw):
    return dict(op="fork", kv_heads=shape[1], head_dim=shape[2], layers=layers, seqs=seqs, len_lo=lens[0],
                len_hi=lens[1], children=children, grow=grow, mix=mix, **kw)


def _compact(shape, layers, pages, seqs, percent, mix, **kw):
    return dict(op="compact", kv_heads=shape[1], head_dim=shape[2], layers=layers, pages=pages, seqs=seqs,
                percent=percent, mix=mix, **kw)


def listed():
    return [
        # a short question to the tiny pair: all latency
        _attention(TINY, 1, (37, 37), (0, 0), 1, name="attn_tiny_37"),
        # the benchmark's prompt: one sequence of 512 tokens through an 8B-shaped layer
        _attention(LLAMA_8B, 1, (512, 512), (0, 0), 2, name="attn_8b_512"),
        # the longest prompt the repository runs, 16K tokens: compute-bound
        _attention(LLAMA_8B, 1, (16384, 16384), (0, 0), 3, name="attn_8b_16k"),
        # a batch of ragged prompts of a 1B-shaped drafter (heads of 64), from one token to 2.1K
        _attention(LLAMA_1B, 24, (1, 2100), (0, 0), 4, name="attn_1b_ragged"),
        # a chunk of each of four long prompts, the earlier chunks being cached (five heads per KV head)
        _attention(QWEN_32B, 4, (411, 777), (3001, 16001), 5, name="attn_32b_chunk"),
        # a few new rows on two long shared prompts: bound by the cache's bytes, few rows
        _attention(LLAMA_8B, 2, (6, 17), (60001, 65501), 6, name="attn_8b_suffix"),
        # the rows of a verification block of 16 sequences, bf16
        _append(LLAMA_1B, 16, (9, 9), (100, 1000), "bf16", 7, name="append_1b_block"),
        # a whole 16K prompt, f32 rows cut out of a fused q|k|v projection's output
        _append(LLAMA_8B, 1, (16384, 16384), (0, 0), "f32", 8, name="append_8b_16k"),
        # one prompt forked into four sampled continuations
        _fork(LLAMA_1B, 16, 1, (517, 517), 4, 17, 9, name="fork_1b_4"),
        # a batch of 32 sequences reordered into 128: shared, dropped, rolled back and grown
        _fork(LLAMA_8B, 32, 32, (60, 1300), 128, 20, 10, name="fork_8b_128"),
        # a small pool after some sequences have gone
        _compact(LLAMA_1B, 16, 203, 5, 60, 11, name="compact_1b_203"),
        # a pool of 4096 pages, 6 in 10 alive
        _compact(LLAMA_8B, 32, 4096, 48, 60, 12, name="compact_8b_4096"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _too_much(case):
    """More work than the 16K prompt (its plain form pads every sequence to the longest), or a cache over 4 GB."""
    rows, prefix = case["rows_hi"], case["prefix_hi"]
    if case["op"] == "append":
        scores, flops = 0, 16384 * 8 * 128 < case["seqs"] * rows * case["kv_heads"] * case["head_dim"]
    else:
        scores, flops = case["seqs"] * case["heads"] * rows * (rows + prefix), work(case)["flops"] > 2.19e12
    return flops or scores > 32 * 16384 * 16384 or case["seqs"] * (rows + prefix) * case["kv_heads"] * case["head_dim"] * 4 > 2 << 30


def draw(rng):
    kind = rng.choice(("attention", "attention", "attention", "append", "fork", "compact"))
    shape = rng.choice(SHAPES)
    mix = rng.randrange(1, 1 << 20)
    if kind in ("attention", "append"):
        seqs = _log(rng, 1, 64)
        hi = _log(rng, 1, 16384)
        lo = rng.choice((1, hi, max(1, hi // 3)))
        p_hi = rng.choice((0, 0, _log(rng, 16, 65000)))
        p_lo = rng.choice((0, p_hi, p_hi // 2))
        make = ((lambda: _attention(shape, seqs, (min(lo, hi), hi), (p_lo, p_hi), mix)) if kind == "attention" else  # noqa: E731
                (lambda: _append(shape, seqs, (min(lo, hi), hi), (p_lo, p_hi), dtype, mix)))  # noqa: E731
        dtype = rng.choice(("bf16", "f32"))
        while _too_much(make()):
            if seqs > 1:
                seqs //= 2
            else:
                hi //= 2
        return make()
    layers = rng.choice((1, shape[3], max(1, min(32, shape[3] // 2))))
    page_bytes = layers * 2 * shape[1] * PAGE * shape[2] * 2
    if kind == "fork":
        hi = _log(rng, 1, 4000)
        seqs = _log(rng, 1, 64)
        children = _log(rng, 1, 256)
        grow = rng.choice((0, 1, 6, 40))
        while seqs > 1 and (seqs * (hi // PAGE + 1) + children * (2 + grow // PAGE + 1)) * page_bytes > (6 << 30):
            seqs //= 2
        return _fork(shape, layers, seqs, (rng.choice((1, hi)), hi), children, grow, mix)
    pages = _log(rng, 16, 8192)
    while pages > 16 and pages * page_bytes > (7 << 30):
        pages //= 2
    return _compact(shape, layers, pages, min(pages, _log(rng, 1, 64)), rng.randrange(5, 96), mix)


# ---------------------------------------------------------------------------------------- inputs
def _spread(rng, n, lo, hi):
    """n lengths between lo and hi, spread over their logarithm; the first is hi."""
    if lo >= hi:
        return [hi] * n
    return [hi if i == 0 else _log(rng, max(1, lo), hi) if lo > 0 else rng.randrange(0, hi + 1) for i in range(n)]


def _lens(case):
    """(new rows, cached prefix) of every sequence: part of the case, whatever the seed."""
    r = random.Random(case["mix"])
    return (_spread(r, case["seqs"], case["rows_lo"], case["rows_hi"]),
            _spread(r, case["seqs"], case["prefix_lo"], case["prefix_hi"]))


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def _table(seed, pages, stride, n_pages):
    """A table giving every sequence `pages[s]` pages of its own, scattered over the pool; 0 elsewhere."""
    ids = random.Random(seed).sample(range(n_pages), sum(pages))
    rows, at = [], 0
    for n in pages:
        rows.append(ids[at:at + n] + [0] * (stride - n))
        at += n
    return _ints(rows)


def _rows_state(case, seed, layers, layer):
    rows, prefix = _lens(case)
    kv = [a + b for a, b in zip(rows, prefix)]
    pages = [-(-n // PAGE) for n in kv]
    stride, n_pages = max(pages) + 1, sum(pages) + 3
    cu = [0]
    for n in rows:
        cu.append(cu[-1] + n)
    g = _gen(seed)
    s = {"case": case, "layer": layer, "M": cu[-1], "max_rows": max(rows), "max_kv": max(kv), "cu": _ints(cu), "kv_len": _ints(kv),
         "table": _table(seed, pages, stride, n_pages), "cu_host": cu, "kv_host": kv,
         "pool": _normal(g, layers, n_pages, 2, case["kv_heads"], PAGE, case["head_dim"])}
    return s, g


def _fork_plan(case, seed):
    """Parents, kept lengths and the old lengths of a fork. Most children share a parent with others; some
    sequences have no child (their pages are released), some children are empty or rolled back."""
    r = random.Random(case["mix"])
    lens = _spread(r, case["seqs"], case["len_lo"], case["len_hi"])
    n, c = case["seqs"], case["children"]
    few = c <= 4
    parent = [0 if n == 1 else (-1 if not few and r.random() < 0.05 else r.randrange(max(1, (3 * n) // 4))) for _ in range(c)]
    keep = [0 if p < 0 else lens[p] if few or r.random() < 0.75 else max(0, lens[p] - r.randrange(0, 20)) for p in parent]
    return lens, parent, keep


def prepare(case, seed):
    op = case["op"]
    if op == "attention":
        s, g = _rows_state(case, seed, 2, 1)
        # queries whose scores have a spread of about 1.5, as trained heads have
        s["q"] = _normal(g, s["M"], case["heads"], case["head_dim"]) * 1.5
        return s
    if op == "append":
        s, g = _rows_state(case, seed, 2, 1)
        w = case["heads"] + 2 * case["kv_heads"]
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        qkv = _normal(g, s["M"], w, case["head_dim"], dtype=dt)   # a fused projection's output, k and v cut out of it
        s["k"] = qkv[:, case["heads"]:case["heads"] + case["kv_heads"]]
        s["v"] = qkv[:, case["heads"] + case["kv_heads"]:]
        return s
    g = _gen(seed)
    if op == "fork":
        lens, parent, keep = _fork_plan(case, seed)
        pages = [-(-n // PAGE) for n in lens]
        n_pages = sum(pages) + case["children"] * (1 + -(-case["grow"] // PAGE)) + 5
        stride = max(pages) + 2 + case["grow"] // PAGE
        pinned = [0] * n_pages
        table = _table(seed, pages, stride, n_pages)
        pinned[int(table[0, 0])] = 1                              # a page that a prefix cache holds too
        return {"case": case, "table": table, "length": _ints(lens), "parent": _ints(parent), "keep": _ints(keep),
                "grow": _ints([case["grow"]] * len(parent)), "pinned": _ints(pinned),
                "pool": _normal(g, case["layers"], n_pages, 2, case["kv_heads"], PAGE, case["head_dim"])}
    r = random.Random(seed)
    n_pages, n = case["pages"], case["seqs"]
    live = r.sample(range(n_pages), max(n, n_pages * case["percent"] // 100))
    pages = [len(live) // n + (1 if i < len(live) % n else 0) for i in range(n)]
    stride = max(pages) + 1
    rows, at, ref = [], 0, [0] * n_pages
    for i, m in enumerate(pages):
        own_pages = live[at:at + m]
        if i and m > 1:
            own_pages[0] = rows[0][0]                             # every sequence shares one prompt's first page
        rows.append(own_pages + [0] * (stride - m))
        for p in own_pages:
            ref[p] += 1
        at += m
    return {"case": case, "table": _ints(rows), "pages": _ints(pages), "ref": _ints(ref),
            "pool": _normal(g, case["layers"], n_pages, 2, case["kv_heads"], PAGE, case["head_dim"])}


# ---------------------------------------------------------------------------------------- one pass
def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2511_09844_gb300 import sd2
        if op == "attention":
            out, lse = sd2.attention_prompt(s["q"], s["pool"], s["table"], s["layer"], s["cu"], s["kv_len"],
                                            max_kv=s["max_kv"], return_lse=True)
            return {"out": out, "lse": lse}
        if op == "append":
            sd2.pages_append(s["k"], s["v"], s["pool"], s["table"], s["layer"], s["cu"], s["kv_len"])
            return {"pool": s["pool"].view(torch.int16)}
        if op == "fork":
            f = sd2.pages_fork(s["pool"], s["table"], s["length"], s["parent"], keep=s["keep"], grow=s["grow"],
                               pinned=s["pinned"])
            return {"table": f.table, "length": f.length, "pages": f.pages, "ref": f.ref, "pool": s["pool"].view(torch.int16)}
        c = sd2.pages_compact(s["pool"], s["table"], s["pages"], s["ref"])
        return {"table": c.table, "ref": c.ref, "map": c.map, "n_live": c.n_live, "pool": s["pool"].view(torch.int16)}
    return {"attention": _plain_attention, "append": _plain_append, "fork": _plain_fork, "compact": _plain_compact}[op](s)


def _plain_attention(s):
    q, pool, table, cu, kv_len = s["q"], s["pool"][s["layer"]], s["table"], s["cu"].long(), s["kv_len"].long()
    (M, H, hd), Hkv, n = q.shape, pool.shape[2], table.shape[0]
    Q, K = s["max_rows"], s["max_kv"]
    row = torch.arange(Q, device=q.device)
    pos = torch.arange(K, device=q.device)
    rows_of = cu[1:] - cu[:-1]
    # queries and keys padded to the longest sequence: [n, Hkv, G * Q, hd] and [n, Hkv, K, hd]
    x = q[(cu[:-1, None] + row).clamp(max=M - 1)].float().view(n, Q, Hkv, H // Hkv, hd).permute(0, 2, 3, 1, 4)
    page, off = table.long()[:, pos // PAGE], pos % PAGE
    k = pool[page, 0, :, off].float().permute(0, 2, 1, 3)
    v = pool[page, 1, :, off].float().permute(0, 2, 1, 3).masked_fill((pos >= kv_len[:, None])[:, None, :, None], 0.0)
    a = torch.matmul(x.reshape(n, Hkv, -1, hd), k.transpose(2, 3)).mul_(hd ** -0.5).view(n, Hkv, H // Hkv, Q, K)
    hidden = pos > (kv_len - rows_of)[:, None, None] + row[:, None]
    a.masked_fill_(hidden[:, None, None], float("-inf"))
    top = a.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    a.sub_(top).exp_()
    total = a.sum(-1, keepdim=True)
    o = torch.matmul(a.view(n, Hkv, -1, K), v).view(n, Hkv, H // Hkv, Q, hd) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (total.log() + top).squeeze(-1)
    at = torch.arange(M, device=q.device)
    seq = torch.searchsorted(cu[1:].contiguous(), at, right=True)
    i = at - cu[seq]
    return {"out": o.permute(0, 3, 1, 2, 4)[seq, i].reshape(M, H * hd).to(torch.bfloat16),
            "lse": lse.permute(0, 3, 1, 2)[seq, i].reshape(M, H)}


def _plain_append(s):
    cu, kv_len, M = s["cu"].long(), s["kv_len"].long(), s["M"]
    at = torch.arange(M, device=s["k"].device)
    seq = torch.searchsorted(cu[1:].contiguous(), at, right=True)
    pos = kv_len[seq] - cu[seq + 1] + at
    page = s["table"].long()[seq, pos // PAGE]
    pool = s["pool"][s["layer"]]
    pool[page, 0, :, pos % PAGE] = s["k"].to(torch.bfloat16)
    pool[page, 1, :, pos % PAGE] = s["v"].to(torch.bfloat16)
    return {"pool": s["pool"].view(torch.int16)}


def _plain_fork(s):
    pool, table = s["pool"], s["table"].long()
    stride, n_pages, b = table.shape[1], pool.shape[1], s["parent"].numel()
    dev = table.device
    parent = s["parent"].long()
    keep = torch.where(parent >= 0, torch.minimum(s["keep"].long().clamp(min=0), s["length"].long()[parent.clamp(min=0)]), 0)
    full, tail = keep // PAGE, keep % PAGE
    slot = torch.arange(stride, device=dev)
    old = table[parent.clamp(min=0)]
    shared = slot < full[:, None]
    count = torch.zeros(n_pages, dtype=torch.int64, device=dev)
    count.scatter_add_(0, old.reshape(-1), shared.reshape(-1).long())
    last = old.gather(1, full.clamp(max=stride - 1)[:, None])[:, 0]         # the page of the partial tail
    order = torch.arange(b, device=dev)
    first = torch.full((n_pages,), b, dtype=torch.int64, device=dev)
    first.scatter_reduce_(0, last, torch.where(tail > 0, order, b), "amin")
    stays = (tail > 0) & (count[last] == 0) & (s["pinned"].long()[last] == 0) & (first[last] == order)
    held = torch.clamp((keep + s["grow"].long().clamp(min=0) + PAGE - 1) // PAGE, max=stride)
    kept = full + stays.long()
    ref = count + s["pinned"].long()
    ref.scatter_add_(0, last, stays.long())
    free = torch.nonzero(ref == 0)[:, 0]
    want = held - kept
    start = want.cumsum(0) - want
    got = (free.numel() - start).clamp(min=0).minimum(want)
    fresh = (slot >= kept[:, None]) & (slot < (kept + got)[:, None])
    ids = torch.cat([free, free.new_zeros(1)])[torch.where(fresh, start[:, None] + slot - kept[:, None], 0).clamp(max=free.numel())]
    new = torch.where(shared | (stays[:, None] & (slot == full[:, None])), old, torch.where(fresh, ids, 0))
    ref.scatter_add_(0, new.reshape(-1), fresh.reshape(-1).long())
    copied = (tail > 0) & ~stays & (got > 0)
    length = torch.where((tail > 0) & ~stays & (got == 0), full * PAGE, keep)
    # the tail rows of every copied page, in all layers
    who, r = torch.nonzero(copied[:, None] & (slot.new_tensor(range(PAGE)) < tail[:, None]), as_tuple=True)
    rows = pool.permute(1, 4, 0, 2, 3, 5)
    rows[new.gather(1, full.clamp(max=stride - 1)[:, None])[who, 0], r] = rows[last[who], r]
    return {"table": new.int(), "length": length.int(), "pages": (kept + got).int(), "ref": ref.int(), "pool": pool.view(torch.int16)}


def _plain_compact(s):
    pool, table, ref = s["pool"], s["table"].long(), s["ref"].long()
    n_pages = pool.shape[1]
    live = ref > 0
    n_live = live.sum()
    ids = torch.arange(n_pages, device=ref.device)
    holes = torch.nonzero(~live & (ids < n_live))[:, 0]
    moved = torch.nonzero(live & (ids >= n_live))[:, 0]
    where = torch.where(live, ids, -1)
    where[moved] = holes
    new_ref = torch.where(ids < n_live, ref, 0)
    new_ref[holes] = ref[moved]
    held = torch.arange(table.shape[1], device=ref.device) < s["pages"].long()[:, None]
    pool[:, holes] = pool[:, moved]
    return {"table": torch.where(held, where[table], 0).int(), "ref": new_ref.int(), "map": where.int(),
            "n_live": n_live.int().reshape(1), "pool": pool.view(torch.int16)}


# ---------------------------------------------------------------------------------------- what a pass needs
def work(case):
    op, Hkv, hd = case["op"], case["kv_heads"], case["head_dim"]
    if op in ("attention", "append"):
        rows, prefix = _lens(case)
        M, H = sum(rows), case["heads"]
        if op == "append":
            e = 2 if case["dtype"] == "bf16" else 4
            return {"bytes": 2 * M * Hkv * hd * (e + 2), "flops": 0}
        pairs = sum(n * p + n * (n + 1) // 2 for n, p in zip(rows, prefix))
        kv = sum(rows) + sum(prefix)
        return {"bytes": 2 * 2 * M * H * hd + 4 * M * H + 2 * 2 * kv * Hkv * hd + 4 * kv // PAGE, "flops": 4 * hd * H * pairs}
    row = case["layers"] * 2 * Hkv * hd * 2                        # bytes of one position in all layers
    if op == "fork":
        lens, parent, keep = _fork_plan(case, 0)
        held = [-(-(k + case["grow"]) // PAGE) for k in keep]
        whole = {(p, i) for p, k in zip(parent, keep) for i in range(k // PAGE)}
        seen, rows = set(), 0
        for p, k in zip(parent, keep):
            page = (p, k // PAGE)
            if k % PAGE and (page in whole or page in seen or page == (0, 0)):
                rows += k % PAGE
            seen.add(page)
        pages = sum(-(-n // PAGE) for n in lens) + case["children"] * (1 + -(-case["grow"] // PAGE)) + 5
        return {"bytes": 2 * rows * row + 4 * 2 * sum(held) + 4 * 2 * pages + 4 * 6 * case["children"], "flops": 0}
    # 1 in (percent, 100 - percent) of the live pages lie beyond the first n_live ids
    live = max(case["seqs"], case["pages"] * case["percent"] // 100)
    moved = live * (case["pages"] - live) / case["pages"]
    return {"bytes": int(2 * moved * row * PAGE + 4 * (2 * live + 3 * case["pages"])), "flops": 0}


# ---------------------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    if case["op"] != "attention":
        return None                                                # copies and whole numbers only
    s = prepare(case, seed)
    H, Hkv, hd = case["heads"], case["kv_heads"], case["head_dim"]
    rows, prefix = _lens(case)
    if sum(n * (n + p) for n, p in zip(rows, prefix)) * H * hd * 4 > 9e12:
        return None
    layer = s["pool"][s["layer"]]
    outs, lses = [], []
    for i, (n, p) in enumerate(zip(rows, prefix)):
        ids = s["table"][i, : -(-(n + p) // PAGE)].long()
        kv = layer[ids].double()                                   # [pages, 2, Hkv, 16, hd]
        keys = kv[:, 0].transpose(0, 1).reshape(Hkv, -1, hd)[:, : n + p]
        vals = kv[:, 1].transpose(0, 1).reshape(Hkv, -1, hd)[:, : n + p]
        for a in range(0, n, 512):
            b = min(n, a + 512)
            last = p + b                                           # the block's rows see positions below this
            x = s["q"][s["cu_host"][i] + a:s["cu_host"][i] + b].double()
            z = torch.einsum("rhgd,hkd->rhgk", x.view(b - a, Hkv, H // Hkv, hd), keys[:, :last]) / math.sqrt(hd)
            z += torch.full((b - a, last), float("-inf"), dtype=z.dtype, device=z.device).triu(p + a + 1)[:, None, None]
            lse = torch.logsumexp(z, -1)
            o = torch.einsum("rhgk,hkd->rhgd", torch.exp(z - lse[..., None]), vals[:, :last])
            outs.append(o.reshape(b - a, H * hd))
            lses.append(lse.reshape(b - a, H))
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}
