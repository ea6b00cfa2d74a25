"""Prompts over pools much larger than what they see: the pages are widened under numbers of their own. Results are those of the
same pages in a small pool bit for bit (the same kernel on the same values), and the definition's. Bounds are those of
test_gpu_quantized.py."""
import pytest
import torch

import paged
from paper_2511_09844_gb300 import sd2
from test_gpu_quantized import ERR_RANGE, check

pytestmark = pytest.mark.gpu

ROWS = [([150, 200], [300, 1200]), ([300], [300]), ([257, 0, 300, 129], [387, 40, 303, 906]), ([600, 700, 100], [600, 3700, 100]),
        ([40] * 40, [40 + 7 * i for i in range(40)])]


def pages_of(c, n_bytes=600 << 20):
    """Pages of a pool that would take so many bytes as bf16."""
    return n_bytes // (2 * c["Hkv"] * 16 * c["hd"] * 2)


def on_device(c, n=None):
    """The case's tensors on the device, its pages at random places of a pool of n pages (of NaN); or in its own pool."""
    d = {k: v.cuda() for k, v in c.items() if isinstance(v, torch.Tensor)}
    if n is None:
        return d
    small = c["pool"].shape[1]
    ids = torch.randperm(n, generator=torch.Generator().manual_seed(1))[:small]
    pool = torch.full((2, n, *c["pool"].shape[2:]), 0x7F, dtype=torch.uint8, device="cuda")
    pool[:, ids.cuda()] = d["pool"].view(torch.uint8)
    scale = torch.full((2, n, *c["scale"].shape[2:]), 200, dtype=torch.uint8, device="cuda")
    scale[:, ids.cuda()] = d["scale"]
    inside = (c["table"] >= 0) & (c["table"] < small)
    table = torch.where(inside, ids[c["table"].long().clamp(0, small - 1)].int(), torch.where(c["table"] < 0, -1, n)).int()
    return dict(d, pool=pool.view(torch.float8_e4m3fn), scale=scale, table=table.cuda())


def need_of(c, max_kv, n_blocks):
    return sd2.load_library().sd2_attention_quantized_workspace_bytes(c["q"].shape[0], len(c["rows"]), c["H"], c["Hkv"], c["hd"], max_kv, n_blocks,
                                                                      c["window"], c["sinks"])


def run(c, n=None, max_kv=None):
    """In a pool of n pages, or the case's own."""
    d = on_device(c, n)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    max_kv = max(c["kv"]) if max_kv is None else max_kv
    ws = torch.full((need_of(c, max_kv, d["pool"].shape[1]),), 255, dtype=torch.uint8, device="cuda")   # whatever it held before
    out, lse = sd2.attention_quantized(d["q"], d["pool"], d["scale"], d["table"], c["layer"], d["cu"], d["kv_len"], max_kv=max_kv,
                                       window=c["window"], sinks=c["sinks"], return_lse=True, workspace=ws, err=err)
    torch.cuda.synchronize()
    return out.cpu(), lse.cpu(), int(err)


@pytest.mark.parametrize("H,Hkv,hd", [(8, 2, 128), (14, 2, 64), (16, 4, 64)])
@pytest.mark.parametrize("rows,kv", ROWS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 5), (1, 0), (300, 40)])
def test_the_same_as_in_a_small_pool(H, Hkv, hd, rows, kv, window, sinks):
    c = paged.case(rows, kv, H, Hkv, hd, seed=H, eight=True, window=window, sinks=sinks)
    n = pages_of(c)
    assert need_of(c, max(kv), n) < 300 << 20
    o = paged.definition(c)
    want = run(c)
    check(c, *want[:2], few=False, want=o)
    for max_kv in (max(kv), 16 * c["table"].shape[1], max(kv) + 100):   # (the table has more columns than that, or has not)
        got = run(c, n, max_kv)
        assert got[2] == 0
        assert (torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])) or max_kv != max(kv)
        check(c, *got[:2], few=False, want=o)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("rows,kv", ROWS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 40)])
def test_lengths_beyond_what_the_call_was_told(hd, rows, kv, window, sinks):
    """A larger length is still right, on one sequence or all, whatever the room."""
    c = paged.case(rows, kv, 8, 2, hd, seed=3, eight=True, window=window, sinks=sinks)
    o = paged.definition(c)
    for claim in (1, 200, 600, max(kv) - 16):
        out, lse, err = run(c, pages_of(c), max(claim, 1))
        assert err == 0
        check(c, out, lse, few=False, want=o)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (150, 20)])
def test_pages_that_sequences_share(hd, window, sinks):
    """Forked prompts: the first 288 positions' pages are the same ones, for 40 sequences of different lengths; some see them, some
    do not; two have the first page only in common; and a page may be another place's, too."""
    rows, kv = [30 + i % 3 * 20 for i in range(40)], [330 + 11 * (i % 5) + 40 * (i % 3) for i in range(40)]
    c = paged.case(rows, kv, 8, 2, hd, seed=5, eight=True, window=window, sinks=sinks)
    own = c["table"].clone()
    c["table"][:, :18] = c["table"][7, :18]
    c["table"][11:13, 1:] = own[11:13, 1:]
    c["table"][9, 2] = c["table"][9, 4]
    c["rows"][3], c["kv"][3] = 30, 31        # (sees two pages only)
    c["rows"][0], c["kv"][0] = 30, 30
    c["cu"] = torch.tensor([0] + c["rows"]).cumsum(0).int()
    c["kv_len"] = torch.tensor(c["kv"], dtype=torch.int32)
    c["q"] = c["q"][: int(c["cu"][-1])]
    want, got = run(c), run(c, pages_of(c))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    check(c, *got[:2], few=False)


@pytest.mark.parametrize("hd", [64, 128])
def test_bad_pages_are_hidden(hd):
    c = paged.case([200, 150], [700, 420], 8, 2, hd, seed=8, eight=True)
    c["table"][0, 3] = -1
    c["table"][1, 9] = c["pool"].shape[1]
    want, got = run(c), run(c, pages_of(c))
    assert want[2] == got[2] == ERR_RANGE
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.isfinite(got[0]).all()


def test_a_table_shorter_than_the_cache():
    for window in (0, 300):
        c = paged.case([200, 300], [500, 900], 8, 2, 64, seed=1, eight=True, window=window, sinks=2)
        c["table"] = c["table"][:, :30].contiguous()
        for max_kv in (900, 300, 5000):
            out, lse, err = run(c, pages_of(c), max_kv)
            assert err == 0
            check(c, out, lse, few=False)


def test_rows_of_no_sequence_are_left_as_they_were():
    """Packed rows before the first offset and behind the last one; with lengths as told, and beyond."""
    c = paged.case([150, 200], [300, 700], 8, 2, 64, seed=6, eight=True)
    d = on_device(c, pages_of(c))
    M, first, more = 350, 2, 3
    q = torch.full((first + M + more, 8, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    q[first:first + M] = d["q"]
    cu, lib, p = d["cu"] + first, sd2.load_library(), sd2._ptr
    o = paged.definition(c)
    for max_kv in (700, 400):
        out, lse = torch.full((first + M + more, 512), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((first + M + more, 8), 7.0, device="cuda")
        ws = torch.full((lib.sd2_attention_quantized_workspace_bytes(first + M + more, 2, 8, 2, 64, max_kv, d["pool"].shape[1], 0, 0),), 255,
                        dtype=torch.uint8, device="cuda")
        assert ws.nbytes < 300 << 20
        assert lib.sd2_attention_quantized(p(q), 512, first + M + more, 8, 2, 64, p(d["pool"]), p(d["scale"]), d["pool"].shape[1], p(d["table"]),
                                           d["table"].shape[1], 1, p(cu), p(d["kv_len"]), 2, max_kv, 0, 0, p(out), p(lse), p(ws), ws.nbytes, None,
                                           sd2._stream()) == sd2.SD2_OK
        torch.cuda.synchronize()
        out, lse = out.cpu(), lse.cpu()
        check(c, out[first:first + M], lse[first:first + M], few=False, want=o)
        for t in (out, lse):
            assert (t[:first] == 7.0).all() and (t[first + M:] == 7.0).all()


def test_a_captured_call_follows_the_lengths():
    """Also beyond what it was told when it was captured, and back; two graphs share the workspace."""
    c = paged.case([150, 300], [300, 900], 8, 2, 128, seed=2, eight=True)
    d = on_device(c, pages_of(c))
    ws = torch.full((need_of(c, 400, d["pool"].shape[1]),), 255, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(side):
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                out = sd2.attention_quantized(d["q"], d["pool"], d["scale"], d["table"], 1, d["cu"], d["kv_len"], max_kv=400, return_lse=True,
                                              workspace=ws)
            graphs.append((g, out))
        for k, kv in enumerate(([300, 400], [300, 900], [150, 300], [160, 777], [200, 390])):
            x = dict(c, kv=kv, kv_len=torch.tensor(kv, dtype=torch.int32))
            d["kv_len"].copy_(x["kv_len"])
            g, out = graphs[k % 2]
            out[0].fill_(7.0)
            g.replay()
            side.synchronize()
            check(x, out[0].cpu(), out[1].cpu(), few=False)


def test_a_short_prompt_in_a_pool_beyond_4_gb():
    """Still a prompt's way: 16 heads of 128, pages of 128 KB as bf16."""
    c = paged.case([300], [400], 32, 16, 128, seed=4, eight=True)
    n = pages_of(c, (4 << 30) + (64 << 20))
    assert need_of(c, 400, n) < 64 << 20
    want, got = run(c), run(c, n)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("rows,kv", [([1, 2, 1], [500, 3000, 40]), ([150, 300], [300, 1200])])
@pytest.mark.parametrize("hd", [64, 128])
def test_a_compacted_cache(hd, rows, kv):
    """Values as 16-bit words through pages_compact, the exponent bytes by its map: the same results."""
    c = paged.case(rows, kv, 8, 2, hd, seed=6, eight=True)
    d = on_device(c, 700)
    pages = torch.tensor([(x + 15) // 16 for x in kv], dtype=torch.int32)
    ref = torch.zeros(700, dtype=torch.int32)
    for s, n in enumerate(pages):
        ref[d["table"][s, :n].cpu().long()] += 1
    want = run(c)
    got = sd2.pages_compact(d["pool"].view(torch.bfloat16), d["table"], pages.cuda(), ref.cuda())
    old = torch.nonzero(got.map >= 0)[:, 0]
    scale = d["scale"].clone()
    scale[:, got.map[old].long()] = d["scale"][:, old]
    n = int(got.n_live)
    assert n == int(pages.sum()) and int(got.table.max()) < n
    out, lse = sd2.attention_quantized(d["q"], d["pool"][:, :n].contiguous(), scale[:, :n].contiguous(), got.table, c["layer"], d["cu"], d["kv_len"],
                                       max_kv=max(kv), return_lse=True)
    assert torch.equal(out.cpu(), want[0]) and torch.equal(lse.cpu(), want[1])
