"""Appending to, forking and compacting the shared paged cache against plain Python: whole numbers and
copied rows, so everything has to be equal."""
import random
import subprocess
import sys

import pytest
import torch

from conftest import ROOT
from paper_2511_09844_gb300 import sd2

pytestmark = pytest.mark.gpu

ERR_RANGE, ERR_PAGES = 4, 8


def _i(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _pool(L, n, Hkv, hd, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-30000, 30000, (L, n, 2, Hkv, 16, hd), generator=g, device="cuda",
                         dtype=torch.int16).view(torch.bfloat16)


def _bits(t):
    return t.view(torch.int16)


# ------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("Hkv,hd", [(8, 128), (8, 64), (2, 64), (1, 8), (3, 40)])
@pytest.mark.parametrize("rows,kv", [([1], [1]), ([0, 5, 0, 17, 1, 0], [0, 21, 3, 17, 33, 16]), ([700, 9], [700, 100]),
                                     ([4], [2])])
def test_append(dtype, Hkv, hd, rows, kv):
    """New rows land at the last positions of their sequences and nowhere else; rows whose position would be
    negative are skipped and reported."""
    n, stride, M = len(rows), max(1, (max(kv) + 15) // 16), sum(rows)
    n_blocks = n * stride + 2
    table = torch.randperm(n_blocks, generator=torch.Generator().manual_seed(1))[: n * stride].view(n, stride)
    pool = _pool(2, n_blocks, Hkv, hd)
    want = pool.clone()
    g = torch.Generator(device="cuda").manual_seed(2)
    qkv = torch.randn(M, 3 + 2 * Hkv, hd, generator=g, device="cuda").to(dtype)
    k, v = qkv[:, 3:3 + Hkv], qkv[:, 3 + Hkv:]
    cu = [0]
    for s in range(n):
        for r in range(rows[s]):
            pos = kv[s] - rows[s] + r
            if pos >= 0:
                want[1, int(table[s, pos // 16]), 0, :, pos % 16] = k[cu[-1] + r].to(torch.bfloat16)
                want[1, int(table[s, pos // 16]), 1, :, pos % 16] = v[cu[-1] + r].to(torch.bfloat16)
        cu.append(cu[-1] + rows[s])
    err = _i([0])
    sd2.pages_append(k, v, pool, table.int().cuda(), 1, _i(cu), _i(kv), err=err)
    assert torch.equal(_bits(pool), _bits(want))
    assert int(err) == (ERR_RANGE if rows == [4] else 0)


def test_append_skips_what_has_no_page():
    """Bad page ids and positions beyond the table's room: skipped, reported, everything else written."""
    pool = _pool(1, 4, 2, 64)
    want = pool.clone()
    k = torch.randn(40, 2, 64, device="cuda")
    for r in list(range(0, 16)):
        want[0, 3, 0, :, r] = k[r].bfloat16()
        want[0, 3, 1, :, r] = (-k[r]).bfloat16()
    err = _i([0])
    sd2.pages_append(k, -k, pool, _i([[3, 4]]), 0, _i([0, 40]), _i([40]), err=err)
    assert torch.equal(_bits(pool), _bits(want)) and int(err) == ERR_RANGE
    err.zero_()
    sd2.pages_append(k, -k, pool, _i([[-1, -7]]), 0, _i([0, 40]), _i([40]), err=err)
    assert torch.equal(_bits(pool), _bits(want)) and int(err) == ERR_RANGE


def test_append_rounds_to_nearest_even_and_keeps_specials():
    vals = torch.tensor([1.00390625, 1.01171875, -1.00390625, float("inf"), float("-inf"), 3.4e38, -0.0, 1e-40],
                        device="cuda")
    k = vals.view(1, 1, 8)
    pool = _pool(1, 1, 1, 8)
    sd2.pages_append(k, k, pool, _i([[0]]), 0, _i([0, 1]), _i([1]))
    assert torch.equal(_bits(pool[0, 0, 0, 0, 0]), _bits(vals.bfloat16()))


# ------------------------------------------------------------------------------------------ fork
def _fork_reference(pool, table, length, parent, keep, grow, pinned):
    """The rules, one sequence at a time."""
    n_blocks, stride = pool.shape[1], len(table[0])
    n, err = len(parent), 0
    held, tails, pages, lens = [], [], [], []
    whole, first = [0] * n_blocks, {}
    seqs = []
    for b in range(n):
        p = parent[b]
        if p >= len(table):
            p, err = -1, err | ERR_RANGE
        ln = min(max(length[p], 0), 16 * stride) if p >= 0 else 0
        kp = ln if keep is None else min(max(keep[b], 0), ln)
        full, tail = divmod(kp, 16)
        last = table[p][full] if tail else None
        for i in range(full):
            whole[table[p][i]] += 1
        if tail and last not in first:
            first[last] = b
        seqs.append((p, kp, full, tail, last))
    ref = [w + max(x, 0) for w, x in zip(whole, pinned or [0] * n_blocks)]
    stays = [t > 0 and whole[last] == 0 and (pinned is None or pinned[last] <= 0) and first[last] == b
             for b, (_, _, _, t, last) in enumerate(seqs)]
    for b in range(n):
        if stays[b]:
            ref[seqs[b][4]] += 1
    free = [x for x in range(n_blocks) if ref[x] == 0]
    out_table, out_len, out_pages, copies = [], [], [], []
    for b, (p, kp, full, tail, last) in enumerate(seqs):
        row = [table[p][i] for i in range(full)] + ([last] if stays[b] else [])
        room = min(max(grow[b], 0), 16 * stride) if grow is not None else 0
        want = min(-(-(kp + room) // 16), stride)
        if tail and not stays[b] and not free:
            kp = 16 * full
        for i in range(len(row), want):
            if not free:
                err |= ERR_PAGES
                break
            x = free.pop(0)
            ref[x] += 1
            if i == full and tail and not stays[b]:
                copies.append((last, x, tail))
            row.append(x)
        out_pages.append(len(row))
        out_len.append(kp)
        out_table.append(row + [0] * (stride - len(row)))
    want_pool = pool.clone()
    for src, dst, rows in copies:
        want_pool[:, dst, :, :, :rows] = pool[:, src, :, :, :rows]
    return out_table, out_len, out_pages, ref, want_pool, err


def _fork_check(pool, table, length, parent, keep=None, grow=None, pinned=None):
    want = _fork_reference(pool, table, length, parent, keep, grow, pinned)
    err = _i([0])
    ws = torch.full((sd2.load_library().sd2_pages_fork_workspace_bytes(len(parent), pool.shape[1]),), 0x5A,
                    dtype=torch.uint8, device="cuda")
    f = sd2.pages_fork(pool, _i(table), _i(length), _i(parent), keep=None if keep is None else _i(keep),
                       grow=None if grow is None else _i(grow), pinned=None if pinned is None else _i(pinned),
                       workspace=ws, err=err)
    assert f.table.tolist() == want[0] and f.length.tolist() == want[1] and f.pages.tolist() == want[2]
    assert f.ref.tolist() == want[3] and int(err) == want[5]
    assert torch.equal(_bits(pool), _bits(want[4]))
    return f


def _fresh(lens, stride, n_blocks, seed):
    ids = random.Random(seed).sample(range(n_blocks), sum(-(-x // 16) for x in lens))
    table, at = [], 0
    for x in lens:
        m = -(-x // 16)
        table.append(ids[at:at + m] + [0] * (stride - m))
        at += m
    return table


@pytest.mark.parametrize("L,Hkv,hd", [(1, 2, 64), (3, 8, 128), (2, 1, 8), (2, 3, 24)])
def test_fork_one_prompt(L, Hkv, hd):
    """Four continuations of one prompt: whole pages shared, one keeps the tail, three get copies and room."""
    for n in (1, 15, 16, 17, 37):
        pool = _pool(L, 40, Hkv, hd, seed=n)
        f = _fork_check(pool, _fresh([n], 6, 40, n), [n], [0] * 4, grow=[5, 0, 40, 16])
        assert f.length.tolist() == [n] * 4


def test_fork_frees_rolls_back_and_starts_empty():
    pool = _pool(2, 64, 2, 64)
    lens = [50, 33, 16, 0, 31]
    table = _fresh(lens, 8, 64, 3)
    f = _fork_check(pool, table, lens, [4, -1, 0, 0, 0, 1, 2], keep=[31, 9, 50, 48, 49, 0, 12], grow=[1, 20, 0, 0, 0, 17, 4])
    assert f.length.tolist() == [31, 0, 50, 48, 49, 0, 12]
    g = _fork_check(pool, f.table.tolist(), f.length.tolist(), [-1, -1])     # all given up
    assert sum(g.ref.tolist()) == 0 and g.pages.tolist() == [0, 0]


def test_fork_out_of_pages():
    """Too few free pages: granted in order, a tail without a page is cut, the shortage reported."""
    pool = _pool(1, 5, 2, 64)
    f = _fork_check(pool, _fresh([40], 4, 5, 4), [40], [0, 0, 0, 0], grow=[0, 10, 0, 9])
    assert f.length.tolist() == [40, 40, 32, 32]
    pool = _pool(1, 3, 2, 64)
    f = _fork_check(pool, _fresh([40], 4, 3, 4), [40], [0, 0], grow=[0, 9])
    assert f.length.tolist() == [40, 32] and f.pages.tolist() == [3, 2]


def test_fork_bad_parent_counts_as_none():
    pool = _pool(1, 8, 1, 64)
    _fork_check(pool, _fresh([20], 3, 8, 5), [20], [7, 0, 2 ** 31 - 1], grow=[3, 3, 0])


def test_fork_bad_page_id_is_reported():
    pool = _pool(1, 8, 1, 64)
    before = pool.clone()
    err = _i([0])
    f = sd2.pages_fork(pool, _i([[3, 99, 2, 0], [5, -4, 0, 0]]), _i([40, 20]), _i([0, 1]), err=err)
    assert int(err) == ERR_RANGE
    assert f.table[0].tolist()[:3] == [3, 0, 2] and f.pages.tolist() == [3, 2]
    assert f.table[1].tolist()[0] == 5 and torch.equal(_bits(pool), _bits(before))


@pytest.mark.parametrize("seed", range(12))
def test_fork_chains(seed):
    """Generations of forks, rollbacks and pins: each against the rules, and every held position keeps its
    content through all of them."""
    r = random.Random(seed)
    L, Hkv, hd, stride, n_blocks = r.choice([(1, 2, 64, 9, 90), (2, 1, 128, 20, 400), (2, 2, 8, 5, 33)])
    pool = _pool(L, n_blocks, Hkv, hd, seed)
    n = r.randrange(1, 6)
    lens = [r.randrange(0, 16 * stride // 2) for _ in range(n)]
    while sum(-(-x // 16) for x in lens) > n_blocks // 2:
        lens = [x // 2 for x in lens]
    table = _fresh(lens, stride, n_blocks, seed)
    pinned = [0] * n_blocks
    for x in range(0, n_blocks, 11):
        pinned[x] = r.choice((0, 0, 1, 2))

    def rows(t, b, m):
        return [_bits(pool[:, t[b][j // 16], :, :, j % 16]).clone() for j in range(0, m, 7)]

    for _ in range(4):
        m = r.randrange(1, 9)
        parent = [r.randrange(-1, len(table)) for _ in range(m)]
        keep = [r.randrange(0, 16 * stride) if r.random() < 0.4 else lens[p] if p >= 0 else 0 for p in parent]
        grow = [r.choice((0, 1, 16, 33)) for _ in range(m)]
        old = [rows(table, p, min(k, lens[p])) if p >= 0 else [] for p, k in zip(parent, keep)]
        f = _fork_check(pool, table, lens, parent, keep, grow, pinned)
        table, lens = f.table.tolist(), f.length.tolist()
        for b in range(m):
            for x, y in zip(old[b], rows(table, b, lens[b])):
                assert torch.equal(x, y)


def test_fork_of_a_large_pool():
    """Needs that reach far beyond the first scan step over the pool, and a long table row."""
    n_blocks, stride = 60000, 3000
    pool = _pool(1, n_blocks, 1, 8)
    lens = [16 * 2000 + 5, 7]
    pinned = [1 if x < 30000 and x % 3 else 0 for x in range(n_blocks)]
    f = _fork_check(pool, _fresh(lens, stride, n_blocks, 6), lens, [0, 1, 0, 1, 1] + [-1] * 600,
                    grow=[16 * 900] * 5 + [40] * 600, pinned=pinned)
    assert f.pages.tolist()[5] == 3


# ------------------------------------------------------------------------------------------ compact
def _compact_check(pool, table, pages, ref):
    n_blocks, stride = pool.shape[1], len(table[0])
    live = [x for x in range(n_blocks) if ref[x] > 0]
    n = len(live)
    holes = [x for x in range(n) if ref[x] <= 0]
    movers = [x for x in live if x >= n]
    assert len(holes) == len(movers)
    to = {x: x for x in live if x < n}
    to.update(zip(movers, holes))
    want = pool.clone()
    for a, b in zip(movers, holes):
        want[:, b] = pool[:, a]
    err = _i([0])
    c = sd2.pages_compact(pool, _i(table), _i(pages), _i(ref), err=err)
    want_ref = [0] * n_blocks
    for x in live:
        want_ref[to[x]] = ref[x]
    bad = any(table[s][i] not in to for s in range(len(table)) for i in range(min(pages[s], stride)))
    assert int(err) == (ERR_RANGE if bad else 0)
    assert c.n_live.tolist() == [n] and c.ref.tolist() == want_ref
    assert c.map.tolist() == [to.get(x, -1) for x in range(n_blocks)]
    assert c.table.tolist() == [[to.get(table[s][i], 0) if i < pages[s] else 0 for i in range(stride)]
                                for s in range(len(table))]
    assert torch.equal(_bits(pool), _bits(want))
    return c


@pytest.mark.parametrize("L,Hkv,hd", [(1, 2, 64), (3, 8, 128), (2, 3, 24)])
@pytest.mark.parametrize("n_blocks,share", [(1, 1.0), (1, 0.0), (33, 0.5), (200, 0.05), (200, 0.97), (3000, 0.4)])
def test_compact(L, Hkv, hd, n_blocks, share):
    r = random.Random(n_blocks)
    ref = [r.randrange(1, 4) if r.random() < share else 0 for _ in range(n_blocks)]
    if n_blocks == 1:
        ref = [int(share)]
    live = [x for x in range(n_blocks) if ref[x]]
    r.shuffle(live)
    table, pages, stride = [], [], 1 + len(live) // 3
    for s in range(4):
        part = live[s * len(live) // 4:(s + 1) * len(live) // 4][:stride]
        pages.append(len(part))
        table.append(part + [r.randrange(0, n_blocks)] * (stride - len(part)))
    _compact_check(_pool(L, n_blocks, Hkv, hd, seed=n_blocks), table, pages, ref)


def test_compact_reports_dead_and_bad_entries():
    _compact_check(_pool(1, 9, 1, 64), [[8, 2, 99], [-1, 4, 8]], [3, 2], [0, 0, 0, 0, 1, 0, 0, 0, 2])


def test_compact_of_a_large_pool():
    """More pages than one pass of the rank kernel's CTAs covers."""
    r = random.Random(9)
    n = 400000
    ref = [1 if r.random() < 0.3 else 0 for _ in range(n)]
    live = [x for x in range(n) if ref[x]][-200:]
    _compact_check(_pool(1, n, 1, 8), [live], [200], ref)


def test_fork_then_compact_keeps_every_position():
    pool = _pool(2, 120, 2, 64, 8)
    lens = [100, 37, 64]
    f = _fork_check(pool, _fresh(lens, 10, 120, 8), lens, [0, 0, 2], grow=[3, 3, 3])
    before = [[_bits(pool[:, f.table[b, j // 16], :, :, j % 16]).clone() for j in range(int(f.length[b]))] for b in range(3)]
    c = _compact_check(pool, f.table.tolist(), f.pages.tolist(), f.ref.tolist())
    for b in range(3):
        for j, x in enumerate(before[b]):
            assert torch.equal(x, _bits(pool[:, c.table[b, j // 16], :, :, j % 16]))
    assert int(c.table.max()) < int(c.n_live)


@pytest.mark.parametrize("seed", range(4))
def test_fork_chains_beyond_one_block(seed):
    """The same rules where the plan runs over several blocks: a pool larger than one block counts, or a batch."""
    r = random.Random(100 + seed)
    n_blocks, stride, n = (13000, 40, 5) if seed % 2 else (900, 33, 2100)
    pool = _pool(1, n_blocks, 1, 8, seed)
    lens = [r.randrange(0, 300) for _ in range(6)]
    table = _fresh(lens, stride, n_blocks, seed)
    pinned = [1 if r.random() < 0.1 else 0 for _ in range(n_blocks)]
    for _ in range(2):
        parent = [r.randrange(-1, len(table)) for _ in range(n)]
        keep = [r.randrange(0, 16 * stride) if r.random() < 0.5 else lens[p] if p >= 0 else 0 for p in parent]
        f = _fork_check(pool, table, lens, parent, keep, [r.choice((0, 0, 0, 1, 20)) for _ in parent], pinned)
        table, lens = f.table.tolist(), f.length.tolist()


def test_page_operators_in_a_captured_graph():
    """Fork and compaction replayed on other tables give those tables' results."""
    lens = [50, 20]
    pool = _pool(1, 32, 1, 64, 5)
    a, b = _fresh(lens, 5, 32, 1), _fresh(lens, 5, 32, 2)
    live, n, parent = _i(a), _i(lens), _i([0, 1, 0])
    side = torch.cuda.Stream()

    def both():
        f = sd2.pages_fork(pool, live, n, parent, grow=None)
        return f, sd2.pages_compact(pool, f.table, f.pages, f.ref)
    with torch.cuda.stream(side):
        both()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            f, c = both()
    for table in (a, b):
        fresh = _pool(1, 32, 1, 64, 6)
        pool.copy_(fresh)
        live.copy_(_i(table))
        want = _fork_reference(fresh, table, lens, [0, 1, 0], None, None, None)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert f.table.tolist() == want[0] and f.length.tolist() == want[1] and f.ref.tolist() == want[3]
        for s in range(3):
            for j in range(want[1][s]):
                got = pool[0, c.table[s, j // 16], :, :, j % 16]
                assert torch.equal(_bits(got), _bits(want[4][0, want[0][s][j // 16], :, :, j % 16]))


def test_fork_with_more_room_asked_than_a_table_has():
    top = 2 ** 31 - 1
    f = _fork_check(_pool(2, 60, 2, 64, 9), _fresh([37, 96, 5], 6, 60, 9), [37, 96, 5], [0, 1, 2, -1, 0], keep=[top, 90, 0, 9, 20],
                    grow=[top, top, top, 1 << 30, -top])
    assert f.pages.tolist() == [6, 6, 6, 6, 2]


def test_fork_at_the_limit_of_default_shared_memory():
    """Plans whose counters come to just under and just over what a block gets without asking: each the first fork of
    its process, since a larger one raises the limit for those after it."""
    sizes = [(4, 4079), (4, 4080), (4, 4088), (4, 4089), (30, 4032), (512, 3072)]
    script = ("import sys; sys.path[:0] = ['tests', '.']\n"
              "import test_gpu_pages as t\n"
              "n, blocks = int(sys.argv[1]), int(sys.argv[2])\n"
              "t._fork_check(t._pool(1, blocks, 1, 8), t._fresh([20], 2, blocks, 1), [20], [0] * n, grow=[3] * n)\n")
    procs = [subprocess.Popen([sys.executable, "-c", script, str(n), str(m)], cwd=ROOT, stdout=subprocess.PIPE,
                              stderr=subprocess.STDOUT, text=True) for n, m in sizes]
    for size, p in zip(sizes, procs):
        out, _ = p.communicate(timeout=300)
        assert p.returncode == 0, (size, out)


@pytest.mark.parametrize("n_blocks", [8, 13000])
def test_fork_of_bad_page_ids_shares_no_page_unawares(n_blocks):
    """A whole page out of range becomes page 0, held and counted like any other: it is not granted, and its owner may
    not append to it. A partial last page out of range is dropped: its sequence is cut to its whole pages."""
    pool = _pool(2, n_blocks, 1, 8)
    before, err = pool.clone(), _i([0])
    # sequence 2 ends inside page 0; its child 2 would keep it as its own if nobody else held it
    f = sd2.pages_fork(pool, _i([[3, n_blocks, 2, 0], [5, -4, 0, 0], [7, 0, 0, 0]]), _i([40, 20, 25]), _i([0, 1, 2]),
                       grow=_i([16, 0, 0]), err=err)
    assert int(err) == ERR_RANGE
    assert f.table.tolist() == [[3, 0, 2, 1], [5, 4, 0, 0], [7, 6, 0, 0]]
    assert f.length.tolist() == [40, 16, 25] and f.pages.tolist() == [4, 2, 2]
    assert f.ref.tolist() == [1] * 8 + [0] * (n_blocks - 8)
    want = before.clone()
    want[:, 6, :, :, :9] = before[:, 0, :, :, :9]
    assert torch.equal(_bits(pool), _bits(want))
    # a row more for each: nothing of it lands in page 0
    rows, err = torch.ones(3, 1, 8, device="cuda"), _i([0])
    sd2.pages_append(rows, rows, pool, f.table, 0, _i([0, 1, 2, 3]), f.length + 1, err=err)
    for page, row in ((2, 8), (4, 0), (6, 9)):
        want[0, page, :, :, row] = 1.0
    assert int(err) == 0 and torch.equal(_bits(pool), _bits(want))
    # and in the next generation page 0 is shared, not somebody's own
    g = sd2.pages_fork(pool, f.table, f.length, _i([0, 2]), err=err)
    assert int(err) == 0 and g.table.tolist() == [[3, 0, 2, 0], [7, 6, 0, 0]] and g.ref.tolist()[:8] == [1, 0, 1, 1, 0, 0, 1, 1]
