"""Which kernel takes a call of few query vectors per sequence and KV head, on both sides of each limit, and that its results are within
that kernel's own bounds (test_gpu_quantized.py, test_gpu_window.py). Long caches are announced: the kernels' parts, whose size
depends on the vectors of an item, then show in the workspace."""
import pytest
import torch

import paged
import test_gpu_quantized as quantized
import test_gpu_window as window_tests
from paper_2511_09844_gb300 import sd2

pytestmark = pytest.mark.gpu

CLAIM = 1 << 20


def round256(n):
    return (n + 255) // 256 * 256


def of_parts(M, n_seq, G, Hkv, hd, kq, blocks):
    """The workspace of items of kq vectors cut into shares of so many blocks."""
    items = min(M * G, M * G // kq + n_seq) * Hkv
    return 256 + round256((1 + 2 * items) * 16) + round256(2 * blocks * kq * (hd + 4) * 4)


def case_of(vectors, hd, **kw):
    """Two sequences of `vectors` query vectors per KV head, one KV head."""
    G = next(g for g in (8, 7, 6, 5, 4, 3, 2, 1) if vectors % g == 0)
    rows = [vectors // G] * 2
    return paged.case(rows, [rows[0] + 900, rows[0] + 333], G, 1, hd, seed=vectors, **kw), G


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("vectors,kq", [(1, 8), (8, 8), (9, 16), (16, 16), (17, 0), (24, 0), (32, 0)])
def test_through_a_window(vectors, kq, hd):
    c, G = case_of(vectors, hd, window=700, sinks=5)
    M, sm = c["q"].shape[0], torch.cuda.get_device_properties(0).multi_processor_count
    wide = dict(c, window=1 << 19)            # (what a call sees decides how it is cut)
    need = sd2.load_library().sd2_attention_window_workspace_bytes(M, 2, G, 1, hd, CLAIM, wide["window"], c["sinks"])
    for k in (8, 16):
        assert (need == of_parts(M, 2, G, 1, hd, k, sm)) == (k == kq)
    for x in (wide, c):
        out, lse, err = window_tests.run(x, max_kv=CLAIM)
        assert err == 0
        window_tests.check(x, out, lse)


@pytest.mark.parametrize("hd,limits", [(64, [(8, 8), (9, 16), (17, 24), (25, 32), (32, 32), (33, 128), (127, 128), (256, 128)]),
                                       (128, [(8, 8), (9, 16), (17, 24), (24, 24), (25, 128), (127, 128), (384, 128)])])
def test_over_the_8_bit_cache(hd, limits):
    sm = torch.cuda.get_device_properties(0).multi_processor_count
    for vectors, kq in limits:
        c, G = case_of(vectors, hd, eight=True)
        M = c["q"].shape[0]
        need = sd2.load_library().sd2_attention_quantized_workspace_bytes(M, 2, G, 1, hd, CLAIM, c["pool"].shape[1], 0, 0)
        assert need == of_parts(M, 2, G, 1, hd, kq, sm * (2 if kq == 8 else 1)), vectors
        out, lse, err = quantized.run(c, max_kv=CLAIM)
        assert err == 0
        quantized.check(c, out, lse)


@pytest.mark.parametrize("H,Hkv,hd", [(8, 2, 128), (2, 2, 64), (40, 2, 64)])
def test_thousands_of_sequences_over_the_8_bit_cache(H, Hkv, hd):
    """All sequences share one table row's pages, so the definition is that of one sequence; by the kernel of few vectors, within the
    bound of probabilities in f16."""
    n = 5000
    g = torch.Generator().manual_seed(81)
    one = paged.case([1], [90], H, Hkv, hd, seed=4, eight=True, layers=1, layer=0, window=37, sinks=3)
    rows = torch.randint(0, 2, (n,), generator=g)
    kv = rows + torch.randint(0, 80, (n,), generator=g)
    cu = torch.cat([torch.zeros(1, dtype=torch.long), rows.cumsum(0)])
    M = int(cu[-1])
    q = torch.randn(M, H, hd, generator=g).to(torch.bfloat16)
    d = {k: v.cuda() for k, v in one.items() if isinstance(v, torch.Tensor)}
    table = d["table"].expand(n, -1).contiguous()
    for claim in (90, 100000):
        out, lse = sd2.attention_quantized(q.cuda(), d["pool"], d["scale"], table, 0, cu.int().cuda(), kv.int().cuda(), max_kv=claim, window=37, sinks=3,
                                           return_lse=True)
        out, lse = out.cpu(), lse.cpu()
        for s in [i for i in (0, 1, 2, 30, 31, 32, 33, 63, 64, 65, 1000, 1001, 2500, 2501, n - 33, n - 32, n - 3, n - 2, n - 1) if rows[i]]:
            a, L = int(cu[s]), int(kv[s])
            x = dict(one, q=q[a:a + 1], cu=torch.tensor([0, 1]), rows=[1], kv=[L])
            quantized.check(x, out[a:a + 1], lse[a:a + 1])


@pytest.mark.parametrize("rows,kv", [([1, 2, 1], [500, 3000, 40]), ([9, 12, 7], [600, 2100, 7])])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("claim", [3000, CLAIM])
def test_captured_lengths_and_pages_beyond_32_bits(rows, kv, hd, claim):
    """Page ids whose bytes lie beyond 2^32 in the second layer, through a captured call whose lengths change."""
    c = paged.case(rows, kv, 8, 2, hd, seed=3, eight=True)
    n_blocks = (9 << 29) // (2 * 2 * 16 * hd)
    pool = torch.zeros(2, n_blocks, 2, 2, 16, hd, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    scale = torch.zeros(2, n_blocks, 2, 2, dtype=torch.uint8, device="cuda")
    small = c["pool"].shape[1]
    ids = n_blocks - 1 - torch.randperm(n_blocks // 8, generator=torch.Generator().manual_seed(1))[:small]
    pool.view(torch.uint8)[:, ids.cuda()] = c["pool"].view(torch.uint8).cuda()
    scale[:, ids.cuda()] = c["scale"].cuda()
    q, cu, length, table = c["q"].cuda(), c["cu"].cuda(), c["kv_len"].cuda(), ids[c["table"].long()].int().cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out, lse = sd2.attention_quantized(q, pool, scale, table, 1, cu, length, max_kv=claim, return_lse=True)
        for x in (kv, [max(r, k // 3) for r, k in zip(rows, kv)], kv):
            length.copy_(torch.tensor(x))
            graph.replay()
            side.synchronize()
            quantized.check(dict(c, kv=x), out.cpu(), lse.cpu())
