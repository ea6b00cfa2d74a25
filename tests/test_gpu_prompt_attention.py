"""Prompt attention over the paged cache (sd2_attention_prompt) against its definition in 64 bits.

The bound of every output is derived from the arithmetic: probabilities are rounded to bf16 before the
second product and the result once more, each by at most a relative 2^-8 (8 significant bits: half of
the spacing 2^-7), everything else is 32-bit; so |out - o| <= 2^-8 (sum_j p_j |v_j| + |o|), with
2e-4 sum_j p_j |v_j| on top for the 32-bit terms (scores of at most a few tens carry about 1e-4 of
relative error into a probability). Log-sum-exps carry only the
scores' 32-bit error: at most hd * 2^-23 * sum_i |q_i k_i| / sqrt(hd), below 4e-4 for the inputs here.
Pages no row may see, and the rows of a last page beyond the cached length, hold NaN.
"""
import pytest
import torch

from paper_2511_09844_gb300 import sd2

pytestmark = pytest.mark.gpu

ERR_RANGE = 4
LSE_TOL = 4e-4


def _case(rows, kv, H, Hkv, hd, seed=0, layers=2, layer=1, slack=2, scale=1.5):
    """Packed queries and a pool whose visible rows are random, everything else NaN."""
    g = torch.Generator().manual_seed(seed)
    n = len(rows)
    pages = [(x + 15) // 16 for x in kv]
    stride = max(1, max(pages)) + slack
    n_blocks = sum(pages) + 5
    ids = torch.randperm(n_blocks, generator=g)[: sum(pages)].tolist()
    pool = torch.full((layers, n_blocks, 2, Hkv, 16, hd), float("nan"), dtype=torch.bfloat16)
    table = torch.zeros(n, stride, dtype=torch.int32)
    at = 0
    for s in range(n):
        for i in range(pages[s]):
            p, fill = ids[at], min(16, kv[s] - 16 * i)
            table[s, i] = p
            pool[layer, p, :, :, :fill] = torch.randn(2, Hkv, fill, hd, generator=g).to(torch.bfloat16)
            at += 1
    cu = torch.tensor([0] + rows).cumsum(0).to(torch.int32)
    q = (torch.randn(sum(rows), H, hd, generator=g) * scale).to(torch.bfloat16)
    return dict(q=q, pool=pool, table=table, cu=cu, kv_len=torch.tensor(kv, dtype=torch.int32), rows=rows, kv=kv,
                layer=layer, H=H, Hkv=Hkv, hd=hd)


def _definition(c):
    """(out, lse, sum_j p_j |v_j|) in float64."""
    H, Hkv, hd = c["H"], c["Hkv"], c["hd"]
    M = c["q"].shape[0]
    out, mag = torch.zeros(M, H, hd, dtype=torch.float64), torch.zeros(M, H, hd, dtype=torch.float64)
    lse = torch.full((M, H), float("-inf"), dtype=torch.float64)
    for s, (n, L) in enumerate(zip(c["rows"], c["kv"])):
        if n == 0 or L == 0:
            continue
        kv = c["pool"][c["layer"], c["table"][s, : (L + 15) // 16].long()].double()
        k = kv[:, 0].transpose(0, 1).reshape(Hkv, -1, hd)[:, :L].repeat_interleave(H // Hkv, 0)
        v = kv[:, 1].transpose(0, 1).reshape(Hkv, -1, hd)[:, :L].repeat_interleave(H // Hkv, 0)
        r0 = int(c["cu"][s])
        z = torch.einsum("rhd,hkd->hrk", c["q"][r0:r0 + n].double(), k) / hd ** 0.5
        p = torch.arange(L - n, L)
        z.masked_fill_(torch.arange(L)[None, :] > p[:, None], float("-inf"))
        seen = p >= 0
        zs = z[:, seen]
        lse[r0:r0 + n][seen] = torch.logsumexp(zs, -1).T
        w = torch.softmax(zs, -1)
        out[r0:r0 + n][seen] = torch.einsum("hrk,hkd->rhd", w, v)
        mag[r0:r0 + n][seen] = torch.einsum("hrk,hkd->rhd", w, v.abs())
    return out.reshape(M, -1), lse, mag.reshape(M, -1)


def _bound(o, mag):
    return 2 ** -8 * (mag + o.abs()) + 2e-4 * mag


def _run(c, max_kv=None, **kw):
    d = {k: v.cuda() for k, v in c.items() if isinstance(v, torch.Tensor)}
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = sd2.attention_prompt(d["q"], d["pool"], d["table"], c["layer"], d["cu"], d["kv_len"],
                                    max_kv=max(c["kv"]) if max_kv is None else max_kv, return_lse=True, err=err, **kw)
    torch.cuda.synchronize()
    return out.cpu(), lse.cpu(), int(err.item())


def _check(c, out, lse, want=None):
    o, l, mag = want or _definition(c)
    off = (out.double() - o).abs() - _bound(o, mag)
    assert torch.isfinite(out).all()
    assert off.max().item() <= 1e-6, off.max().item()
    empty = torch.isinf(l)
    assert torch.equal(torch.isinf(lse) & (lse < 0), empty)
    assert (lse.double() - l)[~empty].abs().max().item() <= LSE_TOL if (~empty).any() else True
    assert (out.view(l.shape[0], l.shape[1], -1)[empty] == 0).all()


HEADS = [(4, 4, 64), (2, 2, 64), (14, 2, 64), (8, 2, 64), (8, 2, 128), (10, 2, 128), (3, 1, 128)]


@pytest.mark.parametrize("H,Hkv,hd", HEADS)
@pytest.mark.parametrize("rows,prefix", [
    ([1], [0]), ([37], [0]), ([128], [0]), ([129], [0]), ([300, 1, 64, 17], [0, 0, 0, 0]),
    ([1], [15]), ([1], [16]), ([5, 40], [1000, 3]), ([257, 6], [130, 777])])
def test_against_the_definition(H, Hkv, hd, rows, prefix):
    c = _case(rows, [a + b for a, b in zip(rows, prefix)], H, Hkv, hd, seed=len(rows) + H)
    out, lse, err = _run(c)
    assert err == 0
    _check(c, out, lse)


@pytest.mark.parametrize("H,Hkv,hd", [(32, 1, 64), (65, 1, 64), (96, 1, 128), (128, 1, 64), (128, 1, 128), (24, 2, 128)])
def test_many_heads_per_kv_head(H, Hkv, hd):
    c = _case([3, 21], [3, 200], H, Hkv, hd, seed=H)
    out, lse, err = _run(c)
    assert err == 0
    _check(c, out, lse)


@pytest.mark.parametrize("hd", [64, 128])
def test_rows_that_see_nothing_and_empty_sequences(hd):
    """More new rows than cached positions leave the first rows nothing; sequences of no rows, of no cache."""
    c = _case([0, 20, 5, 0, 3, 0], [0, 7, 0, 40, 3, 0], 8, 2, hd, seed=5)
    out, lse, err = _run(c, max_kv=40)
    assert err == 0
    _check(c, out, lse)
    assert torch.isinf(lse[:13]).all() and torch.isfinite(lse[13:20]).all() and torch.isinf(lse[20:25]).all()


@pytest.mark.parametrize("rows,prefix", [([1], [5000]), ([6, 17], [20000, 9001]), ([2, 1, 9], [4095, 4096, 100]),
                                         ([33, 1], [3333, 0])])
@pytest.mark.parametrize("H,Hkv,hd", [(8, 2, 128), (14, 2, 64)])
@pytest.mark.parametrize("claim", ["exact", "short", "long"])
def test_few_rows_on_long_caches(rows, prefix, H, Hkv, hd, claim):
    """Few rows: the cache is cut into splits that are joined. max_kv only sizes the split."""
    kv = [a + b for a, b in zip(rows, prefix)]
    c = _case(rows, kv, H, Hkv, hd, seed=7)
    out, lse, err = _run(c, max_kv={"exact": max(kv), "short": 64, "long": 1 << 20}[claim])
    assert err == 0
    _check(c, out, lse)


@pytest.mark.parametrize("hd", [64, 128])
def test_large_scores_and_growing_maxima(hd):
    """Peaked softmaxes whose running maximum grows along the cache by far more than a tile's spread."""
    c = _case([200], [700], 4, 2, hd, seed=11, scale=1.0)
    ramp = torch.linspace(0.05, 6.0, 700)
    layer, table = c["layer"], c["table"]
    for j in range(700):
        c["pool"][layer, table[0, j // 16].long(), 0, :, j % 16] *= ramp[j]
    out, lse, err = _run(c)
    o, l, mag = _definition(c)
    assert err == 0
    # scores to about 60: their 32-bit error, hd * 2^-23 * sum |q k| / sqrt(hd), is up to 4 times that of the others
    off = (out.double() - o).abs() - _bound(o, mag) - 2e-3 * mag
    assert off.max().item() <= 1e-6
    assert (lse.double() - l).abs().max().item() <= 4 * LSE_TOL


def test_infinite_scores_weigh_one_position():
    """A key that wins by more than 32 bits can express: its value alone, exactly."""
    c = _case([40], [200], 4, 2, 64, seed=12)
    c["q"][:] = 1.0
    c["pool"][c["layer"], c["table"][0, 3].long(), 0, :, 5] = 1000.0     # position 53
    out, lse, err = _run(c)
    v = c["pool"][c["layer"], c["table"][0, 3].long(), 1, :, 5]
    assert err == 0 and torch.equal(out.view(40, 2, 2, 64), v[None, :, None].expand(40, 2, 2, 64))


def test_strided_queries_other_streams_and_repeats():
    """Queries cut out of a fused projection's rows, on a side stream with a caller's workspace: the bits of
    the plain call, every time."""
    c = _case([70, 129, 3], [70, 500, 2003], 8, 2, 128, seed=13)
    out, lse, _ = _run(c)
    _check(c, out, lse)
    d = {k: v.cuda() for k, v in c.items() if isinstance(v, torch.Tensor)}
    fused = torch.full((c["q"].shape[0], 12, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    fused[:, 2:10] = d["q"]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    need = sd2.load_library().sd2_attention_prompt_workspace_bytes(fused.shape[0], 3, 8, 2, 128, 2003)
    ws = torch.full((need,), 0xAB, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        o2, l2 = sd2.attention_prompt(fused[:, 2:10], d["pool"], d["table"], c["layer"], d["cu"], d["kv_len"], max_kv=2003,
                                      return_lse=True, workspace=ws, stream=side)
        side.synchronize()
        assert torch.equal(o2.cpu(), out) and torch.equal(l2.cpu(), lse)


def test_table_without_room_and_rows_of_no_sequence():
    """A length beyond the table's room is read to its end; rows after the last sequence are not written."""
    c = _case([4], [64], 4, 2, 64, seed=14, slack=0)
    out, lse, err = _run(c)
    _check(c, out, lse)
    d = {k: v.cuda() for k, v in c.items() if isinstance(v, torch.Tensor)}
    longer = d["kv_len"] + 36                       # rows at 96 .. 99, positions 64 .. 99 have no page
    o2 = sd2.attention_prompt(d["q"], d["pool"], d["table"], c["layer"], d["cu"], longer, max_kv=100)
    every = dict(c, q=c["q"])
    z = _definition(dict(every, rows=[4], kv=[64]))[0]
    k = c["pool"][c["layer"], c["table"][0].long()].double()
    kk = k[:, 0].transpose(0, 1).reshape(2, 64, 64).repeat_interleave(2, 0)
    vv = k[:, 1].transpose(0, 1).reshape(2, 64, 64).repeat_interleave(2, 0)
    w = torch.softmax(torch.einsum("rhd,hkd->hrk", c["q"].double(), kk) / 8, -1)
    o, mag = torch.einsum("hrk,hkd->rhd", w, vv), torch.einsum("hrk,hkd->rhd", w, vv.abs())
    assert z.shape == o.reshape(4, -1).shape
    assert ((o2.cpu().double().view_as(o) - o).abs() - _bound(o, mag)).max().item() <= 1e-6
    # three extra packed rows beyond cu_rows[n_seq]
    lib = sd2.load_library()
    q = torch.cat([d["q"], d["q"][:3]])
    guard = torch.full((7, 256), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(lib.sd2_attention_prompt_workspace_bytes(7, 1, 4, 2, 64, 64), dtype=torch.uint8, device="cuda")
    st = lib.sd2_attention_prompt(sd2._ptr(q), 256, 7, 4, 2, 64, sd2._ptr(d["pool"]), d["pool"].shape[1],
                                  sd2._ptr(d["table"]), d["table"].shape[1], c["layer"], sd2._ptr(d["cu"]),
                                  sd2._ptr(d["kv_len"]), 1, 64, sd2._ptr(guard), None, sd2._ptr(ws), ws.numel(), None,
                                  sd2._stream())
    torch.cuda.synchronize()
    assert st == 0 and torch.equal(guard[:4].cpu(), out) and (guard[4:] == 7.0).all()


def test_bad_page_ids_are_reported():
    c = _case([5, 6], [50, 60], 4, 2, 64, seed=15)
    want = _definition(c)
    for bad in (-1, c["pool"].shape[1], 2 ** 31 - 1, -2 ** 31):
        t = dict(c, table=c["table"].clone())
        t["table"][0, 1] = bad
        out, lse, err = _run(t)
        assert err == ERR_RANGE
        sub = lambda x: x[5:]  # noqa: E731
        off = (sub(out).double() - sub(want[0])).abs() - _bound(sub(want[0]), sub(want[2]))
        assert off.max().item() <= 1e-6


def test_a_cache_beyond_32_bit_offsets():
    """The last pages of a layer whose pool offsets pass 2^31 elements (a 4.5 GB pool, one layer of 2)."""
    Hkv, hd = 8, 128
    n_blocks = 36000                                  # 2 layers x 36000 x 32768 elements
    pool = torch.zeros(2, n_blocks, 2, Hkv, 16, hd, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator().manual_seed(16)
    small = _case([20], [100], 16, Hkv, hd, seed=16)
    ids = torch.arange(n_blocks - 7, n_blocks, dtype=torch.int32)
    pool[1, ids.long()] = small["pool"][1, small["table"][0, :7].long()].cuda()
    table = ids.view(1, 7).contiguous()
    assert g is not None
    out, lse = sd2.attention_prompt(small["q"].cuda(), pool, table.cuda(), 1, small["cu"].cuda(), small["kv_len"].cuda(),
                                    max_kv=100, return_lse=True)
    _check(small, out.cpu(), lse.cpu())


def test_tokens_one_at_a_time_agree_with_the_whole_prompt():
    """Each row alone (its own call, as in decoding) against the packed call: the same definition."""
    c = _case([30], [90], 8, 2, 128, seed=17)
    want = _definition(c)
    d = {k: v.cuda() for k, v in c.items() if isinstance(v, torch.Tensor)}
    one = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    outs, lses = [], []
    for i in range(30):
        o, l = sd2.attention_prompt(d["q"][i:i + 1], d["pool"], d["table"], c["layer"], one, d["kv_len"] - 29 + i,
                                    max_kv=90, return_lse=True)
        outs.append(o.cpu())
        lses.append(l.cpu())
    _check(c, torch.cat(outs), torch.cat(lses), want)


def test_agrees_with_decode_attention():
    """The rows of a verification block through both attention kernels of the library."""
    c = _case([6, 6], [500, 131], 32, 8, 128, seed=18)
    c["pool"].nan_to_num_(0.0)                        # decode attention wants finite pages
    out, lse, _ = _run(c)
    d = {k: v.cuda() for k, v in c.items() if isinstance(v, torch.Tensor)}
    i = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    pos = i(list(range(494, 500)) + list(range(125, 131)))
    dec = sd2.attention(d["q"].float(), d["pool"], d["table"], c["layer"], pos, i([0, 6]), i([6, 6]), i([0, 1]), 6, 4, 128)
    o, l, mag = _definition(c)
    # both round probabilities and results to bf16
    assert ((dec.cpu().double() - out.double()).abs() - 2 * _bound(o, mag)).max().item() <= 1e-6


def test_refusals_of_device_tensors():
    """What the binding refuses of tensors on the GPU: types, shapes, strides, layers."""
    c = _case([4], [20], 4, 2, 64, seed=19)
    d = {k: v.cuda() for k, v in c.items() if isinstance(v, torch.Tensor)}
    ok = dict(q=d["q"], pool=d["pool"], table=d["table"], layer=1, cu_rows=d["cu"], kv_len=d["kv_len"], max_kv=20)
    sd2.attention_prompt(**ok)
    for bad in (dict(q=d["q"].float()), dict(q=d["q"].transpose(0, 1)), dict(q=d["q"][:, :3]), dict(q=d["q"][..., :32]),
                dict(q=d["q"][:1].expand(4, 4, 64)), dict(pool=d["pool"][:, ::2]), dict(pool=d["pool"].float()),
                dict(pool=d["pool"][0]), dict(table=d["table"].long()), dict(table=d["table"].T), dict(layer=2),
                dict(layer=-1), dict(cu_rows=d["cu"][:1]), dict(kv_len=d["kv_len"].float()), dict(kv_len=d["kv_len"].cpu()),
                dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(sd2.SD2Error, match="EINVAL"):
            sd2.attention_prompt(**dict(ok, **bad))
    assert sd2.attention_prompt(**dict(ok, q=d["q"][:0], cu_rows=d["cu"] * 0)).shape == (0, 256)


@pytest.mark.parametrize("n", [33, 70])
@pytest.mark.parametrize("H,Hkv,hd", [(8, 2, 128), (14, 2, 64)])
def test_many_sequences(n, H, Hkv, hd):
    """More sequences than one warp holds at a time, empty ones and prefixes among them."""
    g = torch.Generator().manual_seed(n)
    rows = [int(x) for x in torch.randint(0, 90, (n,), generator=g)]
    rows[3] = rows[n - 1] = 0
    prefix = [int(x) if i % 3 else 0 for i, x in enumerate(torch.randint(0, 200, (n,), generator=g))]
    c = _case(rows, [a + b for a, b in zip(rows, prefix)], H, Hkv, hd, seed=n)
    out, lse, err = _run(c)
    assert err == 0
    _check(c, out, lse)


def test_many_sequences_of_one_row_each():
    """A decode batch through the prompt kernel: 40 sequences, split."""
    kv = [1 + 37 * i for i in range(40)]
    c = _case([1] * 40, kv, 2, 1, 128, seed=41)
    out, lse, err = _run(c)
    assert err == 0
    _check(c, out, lse)


def test_two_streams_at_once():
    """Calls that overlap on the GPU, each with its own workspace and error word, keep their own results."""
    cases = [_case([300, 45], [300, 700], 8, 2, 128, seed=51), _case([2, 7], [3000, 2500], 14, 2, 64, seed=52)]
    want = [_run(c)[:2] for c in cases]
    dev = [{k: v.cuda() for k, v in c.items() if isinstance(v, torch.Tensor)} for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, (c, d, st) in enumerate(zip(cases, dev, streams)):
            got[i].append(sd2.attention_prompt(d["q"], d["pool"], d["table"], c["layer"], d["cu"], d["kv_len"],
                                               max_kv=max(c["kv"]), return_lse=True, stream=st))
    torch.cuda.synchronize()
    for i, (out, lse) in enumerate(want):
        for o, l in got[i]:
            assert torch.equal(o.cpu(), out) and torch.equal(l.cpu(), lse)


def test_captured_call_follows_the_device_lengths():
    """A captured call reads offsets and lengths when it is replayed: other lengths, other results, no recapture."""
    a = _case([100, 20], [100, 420], 8, 2, 128, seed=61)
    b = _case([20, 100], [320, 100], 8, 2, 128, seed=61, slack=9)     # another division of the same 120 rows
    want = [_definition(a), _definition(b)]
    width = max(a["table"].shape[1], b["table"].shape[1])
    n_blocks = max(a["pool"].shape[1], b["pool"].shape[1])
    dev = {}
    for name, c in (("a", a), ("b", b)):
        t = torch.zeros(2, width, dtype=torch.int32)
        t[:, :c["table"].shape[1]] = c["table"]
        p = torch.zeros(2, n_blocks, *c["pool"].shape[2:], dtype=torch.bfloat16)
        p[:, :c["pool"].shape[1]] = c["pool"]
        dev[name] = [x.cuda() for x in (c["q"], p, t, c["cu"], c["kv_len"])]
    live = [x.clone() for x in dev["a"]]
    call = lambda: sd2.attention_prompt(live[0], live[1], live[2], 1, live[3], live[4], max_kv=420, return_lse=True)  # noqa: E731
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out, lse = call()
    for name, c, w in (("a", a, want[0]), ("b", b, want[1]), ("a", a, want[0])):
        for x, y in zip(live, dev[name]):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        _check(c, out.cpu(), lse.cpu(), w)


def test_rows_beside_other_sequences_nan():
    """A sequence whose queries are NaN, or whose cache is, spoils its own rows only."""
    c = _case([40, 30, 50], [40, 300, 50], 8, 2, 128, seed=71)
    want = _definition(c)
    c["q"][45:50] = float("nan")
    ids = c["table"][2, :4].long()
    c["pool"][c["layer"], ids] = float("nan")
    out, lse, err = _run(c)
    assert err == 0
    o, l, mag = want
    keep = [i for i in range(70) if not 45 <= i < 50]
    assert ((out[keep].double() - o[keep]).abs() - _bound(o[keep], mag[keep])).max().item() <= 1e-6
    assert torch.isnan(out[45:50].float()).all() and torch.isnan(out[70:].float()).all()


def test_nan_through_split_caches():
    """The same where the positions are split and joined: a NaN anywhere in what a row sees reaches that row."""
    c = _case([1, 2], [3000, 2600], 8, 2, 128, seed=72)
    want = _definition(c)
    c["pool"][c["layer"], c["table"][1, 100].long(), 0, 1, 3] = float("nan")     # position 1603, KV head 1
    out, lse, err = _run(c)
    o, l, mag = want
    assert err == 0
    clean = torch.ones(3, 8, 128, dtype=torch.bool)
    clean[1:, 4:] = False                                                        # heads 4 .. 7 of sequence 1
    off = ((out.double() - o).abs() - _bound(o, mag)).view(3, 8, 128)
    assert off[clean].max().item() <= 1e-6
    assert torch.isnan(out.float().view(3, 8, 128)[~clean]).all() and torch.isnan(lse[1:, 4:]).all()
    assert torch.isfinite(lse[0]).all() and torch.isfinite(lse[1:, :4]).all()


@pytest.mark.parametrize("H,Hkv,hd", [(128, 1, 64), (2, 2, 64)])
def test_thousands_of_sequences(H, Hkv, hd):
    """More tiles than a grid's second dimension holds, and a search over thousands of sequences (spot checks:
    all share one page table row's pages, so the definition is that of one sequence)."""
    n = 33000
    g = torch.Generator().manual_seed(81)
    pool = torch.randn(1, 2, 2, Hkv, 16, hd, generator=g).to(torch.bfloat16)
    rows = torch.randint(1, 5, (n,), generator=g)
    rows[7] = 0
    cu = torch.cat([torch.zeros(1, dtype=torch.long), rows.cumsum(0)])
    kv = rows + torch.randint(0, 20, (n,), generator=g)
    M = int(cu[-1])
    q = torch.randn(M, H, hd, generator=g).to(torch.bfloat16)
    table = torch.tensor([[1, 0]], dtype=torch.int32).expand(n, 2).contiguous()
    out, lse = sd2.attention_prompt(q.cuda(), pool.cuda(), table.cuda(), 0, cu.int().cuda(), kv.int().cuda(), max_kv=24,
                                    return_lse=True)
    out, lse = out.cpu(), lse.cpu()
    for s in [0, 1, 6, 8, 31, 32, 33, 63, 64, 1000, 16500, n - 33, n - 2, n - 1]:
        a, b, L = int(cu[s]), int(cu[s + 1]), int(kv[s])
        c = dict(q=q[a:b], pool=pool, table=table[:1], layer=0, cu=torch.tensor([0, b - a]), rows=[b - a], kv=[L], H=H,
                 Hkv=Hkv, hd=hd)
        _check(c, out[a:b], lse[a:b])
    assert torch.isfinite(lse).all()


@pytest.mark.parametrize("H,Hkv,hd", [(4, 4, 64), (8, 2, 128), (14, 2, 64)])
@pytest.mark.parametrize("claim", [1, 1 << 20])
def test_pieces_for_one_query_tile(H, Hkv, hd, claim):
    """Rows that fill no more than one query tile: both take turns over the cache and are joined, with one to many
    K/V tiles for them, rows that see only the first of them, or none."""
    rows, kv = [1, 3, 20, 9, 7, 12, 5], [128, 129, 300, 1000, 257, 5, 130]
    c = _case(rows, kv, H, Hkv, hd, seed=91)
    out, lse, err = _run(c, max_kv=claim)
    assert err == 0
    _check(c, out, lse)


@pytest.mark.parametrize("H,Hkv,hd", [(8, 2, 128), (14, 2, 64), (3, 1, 128), (4, 4, 64)])
@pytest.mark.parametrize("rows,prefix", [([300, 70], [0, 0]), ([150, 40], [333, 1000]), ([9, 12], [600, 0]),
                                         ([33], [3333]), ([129], [127])])
def test_values_that_only_later_rows_see(rows, prefix, H, Hkv, hd):
    """An infinity or NaN in V reaches its own column of the rows that see its position, and nothing else, although
    earlier rows share tiles with it."""
    kv = [a + b for a, b in zip(rows, prefix)]
    c = _case(rows, kv, H, Hkv, hd, seed=len(rows) + hd)
    want = _definition(c)                             # of the finite values
    put = []                                          # sequence, position, KV head, column, value
    for s, (n, p) in enumerate(zip(rows, prefix)):
        put += [(s, p + n // 2, 0, 5, float("nan")), (s, p + n - 1, Hkv - 1, hd - 1, float("inf")),
                (s, p + 2, Hkv - 1, hd // 2, float("-inf")), (s, p + n // 3, 0, 6, float("nan"))]
    mask = torch.zeros(sum(rows), H, hd, dtype=torch.bool)
    spoilt = {}
    for s, j, h, d, x in put:
        c["pool"][c["layer"], int(c["table"][s, j // 16]), 1, h, j % 16, d] = x
        r0, r1 = int(c["cu"][s]) + j - prefix[s], int(c["cu"][s + 1])
        heads = slice(h * (H // Hkv), (h + 1) * (H // Hkv))
        mask[r0:r1, heads, d] = True
        spoilt[(s, h, d)] = (slice(r0, r1), heads, d, x)
    out, lse, err = _run(c)
    assert err == 0
    assert (lse.double() - want[1]).abs().max().item() <= LSE_TOL
    got, o, mag = (t.view(sum(rows), H, hd) for t in (out.double(), want[0], want[2]))
    assert torch.isfinite(got[~mask]).all()
    assert ((got - o).abs() - _bound(o, mag))[~mask].max().item() <= 1e-6
    for a, b, d, x in spoilt.values():
        assert torch.isnan(got[a, b, d]).all() if x != x else not torch.isfinite(got[a, b, d]).any()


def test_values_of_no_number_everywhere():
    """All of V NaN: every row is, and the log-sum-exps are what they were."""
    c = _case([700, 30], [700, 90], 8, 2, 128, seed=4)
    want = _definition(c)
    c["pool"][c["layer"], :, 1] = float("nan")
    out, lse, err = _run(c)
    assert err == 0 and torch.isnan(out.float()).all()
    assert (lse.double() - want[1]).abs().max().item() <= LSE_TOL


@pytest.mark.parametrize("H,Hkv,hd", [(8, 2, 128), (14, 2, 64), (128, 1, 64)])
@pytest.mark.parametrize("tiles", [1, 2, 3, 4, 5])
def test_few_rows_on_each_number_of_tiles(H, Hkv, hd, tiles):
    """Rows for one slot: from some number of K/V tiles on two slots share them."""
    kv = [128 * tiles - 127, 128 * tiles - 1, 128 * tiles]
    c = _case([1, min(5, kv[1]), 1], kv, H, Hkv, hd, seed=tiles)
    out, lse, err = _run(c, max_kv=kv[2])
    assert err == 0
    _check(c, out, lse)


def test_a_block_freed_behind_pending_work_is_not_taken_on_another_stream():
    """Memory that the current stream still writes when a call on another stream needs as much: the call's own results
    stay what they are."""
    c = _case([300, 45], [300, 700], 8, 2, 128, seed=51)
    out, lse, _ = _run(c)
    d = {k: v.cuda() for k, v in c.items() if isinstance(v, torch.Tensor)}
    side = torch.cuda.Stream()
    busy = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        block, stats = torch.empty(345, 1024, dtype=torch.bfloat16, device="cuda"), torch.empty(345, 8, device="cuda")
        for _ in range(20):
            busy = busy @ busy                                   # some milliseconds of work before the blocks are written
        block.fill_(7.0)
        stats.fill_(7.0)
        del block, stats
        o, l = sd2.attention_prompt(d["q"], d["pool"], d["table"], c["layer"], d["cu"], d["kv_len"], max_kv=700,
                                    return_lse=True, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(o.cpu(), out) and torch.equal(l.cpu(), lse)


def _without(c, bad):
    """_definition with the positions of the pages `bad` (sequence, index in its table row) hidden from every row."""
    H, Hkv, hd = c["H"], c["Hkv"], c["hd"]
    M = c["q"].shape[0]
    out, mag = torch.zeros(M, H, hd, dtype=torch.float64), torch.zeros(M, H, hd, dtype=torch.float64)
    lse = torch.full((M, H), float("-inf"), dtype=torch.float64)
    for s, (n, L) in enumerate(zip(c["rows"], c["kv"])):
        kv = c["pool"][c["layer"], c["table"][s, : (L + 15) // 16].long()].double()
        k = kv[:, 0].transpose(0, 1).reshape(Hkv, -1, hd)[:, :L].repeat_interleave(H // Hkv, 0)
        v = kv[:, 1].transpose(0, 1).reshape(Hkv, -1, hd)[:, :L].repeat_interleave(H // Hkv, 0)
        r0, at = int(c["cu"][s]), torch.arange(L)
        hidden = at[None, :] > torch.arange(L - n, L)[:, None]
        for b, i in bad:
            if b == s:
                hidden |= at[None, :] // 16 == i
        seen = ~hidden.all(1)
        z = torch.einsum("rhd,hkd->hrk", c["q"][r0:r0 + n].double(), k) / hd ** 0.5
        z = z.masked_fill(hidden, float("-inf"))[:, seen]
        lse[r0:r0 + n][seen] = torch.logsumexp(z, -1).T
        w = torch.softmax(z, -1)
        out[r0:r0 + n][seen] = torch.einsum("hrk,hkd->rhd", w, v)
        mag[r0:r0 + n][seen] = torch.einsum("hrk,hkd->rhd", w, v.abs())
    return out.reshape(M, -1), lse, mag.reshape(M, -1)


@pytest.mark.parametrize("H,Hkv,hd", [(8, 2, 128), (14, 2, 64), (3, 1, 128), (4, 4, 64)])
@pytest.mark.parametrize("rows,kv,bad", [
    ([300, 5], [300, 300], [(0, 0), (1, 18)]),                                   # the first page, a partial last page
    ([40, 7], [777, 1000], [(0, i) for i in range(8, 16)] + [(0, 20), (1, 62)]),   # a whole K/V tile
    ([1, 2], [5000, 3000], [(0, 100), (0, 312)] + [(1, i) for i in range(64)]),    # split positions
    ([3, 20], [40, 200], [(0, i) for i in range(3)] + [(1, 5)]),                   # nothing left to see
    ([700, 9, 130], [700, 400, 130], [(0, 1), (0, 2), (0, 43)])])                # clean pieces after others
def test_positions_of_bad_pages_are_hidden(rows, kv, bad, H, Hkv, hd):
    """A page id outside the pool is reported, and its positions weigh nothing: not as zeros, which would count in
    every sum."""
    c = _case(rows, kv, H, Hkv, hd, seed=len(bad) + hd)
    want = _without(c, bad)
    t = dict(c, table=c["table"].clone())
    for n, (s, i) in enumerate(bad):
        t["table"][s, i] = (-1, c["pool"].shape[1], 2 ** 31 - 1, -2 ** 31)[n % 4]
    out, lse, err = _run(t)
    assert err == ERR_RANGE
    _check(c, out, lse, want)


@pytest.mark.parametrize("H,Hkv,hd", [(8, 2, 128), (14, 2, 64)])
def test_bad_pages_beside_values_that_only_later_rows_see(H, Hkv, hd):
    c = _case([60], [200], H, Hkv, hd, seed=23)
    bad = [(0, 2), (0, 9)]
    o, l, mag = _without(c, bad)
    c["pool"][c["layer"], int(c["table"][0, 11]), 1, 0, 7, 5] = float("nan")        # position 183: rows from 43 on
    t = dict(c, table=c["table"].clone())
    t["table"][0, 2], t["table"][0, 9] = -1, c["pool"].shape[1]
    out, lse, err = _run(t)
    assert err == ERR_RANGE
    spoilt = torch.zeros(60, H, hd, dtype=torch.bool)
    spoilt[43:, : H // Hkv, 5] = True
    spoilt = spoilt.view(60, -1)
    assert torch.isnan(out[spoilt].float()).all() and torch.isfinite(out[~spoilt].float()).all()
    assert ((out.double() - o).abs() - _bound(o, mag))[~spoilt].max().item() <= 1e-6
    assert (lse.double() - l).abs().max().item() <= LSE_TOL


@pytest.mark.parametrize("H,Hkv,hd", [(8, 2, 128), (14, 2, 64)])
@pytest.mark.parametrize("rows,prefix", [([1], [0]), ([130], [0]), ([20], [300]), ([1, 3], [3000, 0]), ([300], [500])])
@pytest.mark.parametrize("size", [-3e35, -2e30, -1e12, 1e6, 1e12, 2e37])
def test_scores_of_any_size(size, rows, prefix, H, Hkv, hd):
    """Scores far beyond what an exponent holds, all of a row's alike: its result is the mean of what it sees, its
    log-sum-exp that score."""
    c = _case(rows, [a + b for a, b in zip(rows, prefix)], H, Hkv, hd, seed=31)
    g = torch.Generator().manual_seed(32)
    part = abs(size) * hd ** 0.5 / hd
    base = (torch.rand(hd, generator=g) + 1) * part ** 0.5
    c["q"][:] = base.to(torch.bfloat16)
    key = (part / base * (1 if size > 0 else -1)).to(torch.bfloat16)
    nan = torch.isnan(c["pool"][:, :, 0])
    c["pool"][:, :, 0] = torch.where(nan, c["pool"][:, :, 0], key)
    out, lse, err = _run(c)
    o, l, mag = _definition(c)
    assert err == 0
    assert ((out.double() - o).abs() - _bound(o, mag)).max().item() <= 1e-6
    # hd products and sums in 32 bits, each within 2^-23, and the factor's and the result's roundings
    assert ((lse.double() - l).abs() <= (hd + 4) * 2.0 ** -23 * l.abs() + LSE_TOL).all()


@pytest.mark.parametrize("H,Hkv,hd", [(8, 2, 128), (14, 2, 64)])
@pytest.mark.parametrize("rows,kv", [([1], [300]), ([50], [400]), ([2], [4000])])
@pytest.mark.parametrize("low,high", [(-3e35, -1e30), (-1e33, 2.0), (3.0, 1e15), (1e12, 1e36)])
def test_far_scores_after_others(low, high, rows, kv, H, Hkv, hd):
    """Positions of one far score and, later, some of a higher one: from the first of these on a row is their mean."""
    c = _case(rows, kv, H, Hkv, hd, seed=33)
    layer, L, n = c["layer"], kv[0], rows[0]
    c["q"][:] = 2.0 ** 40
    key = lambda z: z * hd ** 0.5 / hd / 2.0 ** 40  # noqa: E731
    tops = [L - n, L - n - 130, L - n // 2 - 1]
    for j in range(L):
        c["pool"][layer, int(c["table"][0, j // 16]), 0, :, j % 16] = key(high if j in tops else low)
    out, lse, err = _run(c)
    o, l, mag = _definition(c)
    assert err == 0
    assert ((out.double() - o).abs() - _bound(o, mag)).max().item() <= 1e-6
    assert ((lse.double() - l).abs() <= (hd + 4) * 2.0 ** -23 * l.abs() + LSE_TOL).all()


@pytest.mark.parametrize("H,Hkv,hd", [(32, 8, 128), (32, 8, 64), (14, 2, 64)])
def test_long_prompts_of_many_pieces(H, Hkv, hd):
    """Several pieces of many K/V tiles per block, one after another through the same ring and barriers: chosen rows
    against the definition, every row finite."""
    rows, prefix = [4001, 257, 3000, 3], [0, 1500, 129, 0]
    kv = [a + b for a, b in zip(rows, prefix)]
    c = _case(rows, kv, H, Hkv, hd, seed=hd + H)
    out, lse, err = _run(c)
    assert err == 0 and torch.isfinite(out.float()).all() and torch.isfinite(lse).all()
    g = torch.Generator().manual_seed(5)
    for s, (n, p) in enumerate(zip(rows, prefix)):
        at = sorted({0, n - 1, min(127, n - 1), min(128, n - 1)} | set(torch.randint(0, n, (24,), generator=g).tolist()))
        data = c["pool"][c["layer"], c["table"][s, : (kv[s] + 15) // 16].long()].double()
        k = data[:, 0].transpose(0, 1).reshape(Hkv, -1, hd)[:, : kv[s]]
        v = data[:, 1].transpose(0, 1).reshape(Hkv, -1, hd)[:, : kv[s]]
        for i in at:
            m, seen = int(c["cu"][s]) + i, p + i + 1
            x = c["q"][m].double().view(Hkv, H // Hkv, hd)
            z = torch.einsum("hgd,hkd->hgk", x, k[:, :seen]) / hd ** 0.5
            w = torch.softmax(z, -1)
            o = torch.einsum("hgk,hkd->hgd", w, v[:, :seen]).reshape(-1)
            mag = torch.einsum("hgk,hkd->hgd", w, v[:, :seen].abs()).reshape(-1)
            assert ((out[m].double() - o).abs() - _bound(o, mag)).max().item() <= 1e-6
            assert (lse[m].double() - torch.logsumexp(z, -1).reshape(-1)).abs().max().item() <= LSE_TOL


@pytest.mark.parametrize("low,high", [(45425.5, 45426.5), (45426.5, 45425.5), (-45426.5, -45425.5), (45424.0, 45425.0)])
@pytest.mark.parametrize("kv", [300, 3000])
def test_scores_around_the_limit_of_plain_statistics(low, high, kv):
    """Positions a factor e apart, in the same tile and in splits, on either side of where statistics are kept apart
    (2^16 in log2). There a statistic's rounding is 2^-8 in log2: two of them are worth 2^-7 in a weight."""
    c = _case([1], [kv], 2, 1, 64, seed=41)
    c["q"][:] = 0.0
    c["q"][:, :, :2] = 1.0
    for j in range(kv):
        page, at = int(c["table"][0, j // 16]), j % 16
        z = 8 * (low if j < kv // 2 else high)
        big = 362496.0 if z > 0 else -362496.0
        c["pool"][c["layer"], page, 0, :, at] = 0.0
        c["pool"][c["layer"], page, 0, :, at, 0] = big
        c["pool"][c["layer"], page, 0, :, at, 1] = z - big
        c["pool"][c["layer"], page, 1, :, at] = 1.0 if j < kv // 2 else -1.0
    out, lse, err = _run(c)
    o, l, mag = _definition(c)
    assert err == 0
    assert abs(o).max() < 0.6                          # (both levels weigh)
    assert ((out.double() - o).abs() - _bound(o, mag) - 2 ** -7 * mag).max().item() <= 1e-6
    assert ((lse.double() - l).abs() <= 68 * 2.0 ** -23 * l.abs() + LSE_TOL).all()
