"""Items that are cut into parts: a NaN (or, in bf16, an infinity) of V reaches the rows that see it however far the scores of
its part lie below the others'. For the kernels of few vectors and of tiles, over the 8-bit cache, and of few vectors over the
bf16 cache through a window. Bounds are those of test_gpu_quantized.py."""
import pytest
import torch

import paged
from paper_2511_09844_gb300 import sd2
from test_gpu_quantized import check

pytestmark = pytest.mark.gpu

L, FAR = 8000, 4000


def far_case(rows, hd, eight, far_first, window=0):
    """One sequence whose scores on one half of the cache lie some 130 (heads of 64) or 180 below those on the other: queries
    4 in every element, keys -4 there, and small elsewhere."""
    c = paged.case([rows], [L], 8, 2, hd, seed=rows + hd, eight=False, window=window)
    g = torch.Generator().manual_seed(3)
    ids = c["table"][0, : L // 16].long()
    k = torch.randn(L, 2, hd, generator=g) * 0.05
    k[slice(0, FAR) if far_first else slice(FAR, L)] -= 4.0
    pool = c["pool"].float()
    pool[c["layer"], ids, 0] = k.view(-1, 16, 2, hd).transpose(1, 2)
    c["q"] = torch.full_like(c["q"], 4.0)
    if eight:
        c["pool"], c["scale"] = paged.quantized(pool)
    else:
        c["pool"] = pool.to(torch.bfloat16)
    return c


def put(c, p, head, col, value):
    """An odd value into V of position p."""
    at = (c["layer"], int(c["table"][0, p // 16]), 1, head, p % 16, col)
    if "scale" in c:
        c["pool"].view(torch.uint8)[at] = 0x7F
    else:
        c["pool"][at] = value


def run(c, claim):
    """`claim`: the length that the call is told, which only chooses the way."""
    d = {k: v.cuda() for k, v in c.items() if isinstance(v, torch.Tensor)}
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    batch = (d["table"], c["layer"], d["cu"], d["kv_len"])
    if "scale" in c:
        out, lse = sd2.attention_quantized(d["q"], d["pool"], d["scale"], *batch, max_kv=claim, return_lse=True, err=err)
    else:
        out, lse = sd2.attention_window(d["q"], d["pool"], *batch, c["window"], max_kv=claim, return_lse=True, err=err)
    assert int(err) == 0
    return out.cpu(), lse.cpu()


@pytest.mark.parametrize("far_first", [True, False])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("rows,eight,claim", [(1, True, L), (4, True, L), (12, True, 1 << 20), (30, True, 1 << 20), (1, False, L), (4, False, L)])
def test_a_nan_of_a_far_part_is_not_lost(rows, eight, claim, hd, far_first):
    """(12 and 30 rows, 48 and 120 vectors of a KV head, go by tiles where the cache is said to be long.)"""
    c = far_case(rows, hd, eight, far_first, window=0 if eight else L)
    if eight:                                # (a tile's parts of 128 vectors show in the workspace)
        need = sd2.load_library().sd2_attention_quantized_workspace_bytes(rows, 1, 8, 2, hd, claim, c["pool"].shape[1], 0, 0)
        assert (need > 2 * 148 * 128 * (hd + 4) * 4) == (rows > 4)
    out, lse = run(c, claim)
    check(c, out, lse, few=eight)
    base = 0 if far_first else FAR
    for p, head, col in ((base + 40, 0, 3), (base + 2000, 1, hd - 1), (base + 3500, 0, 17)):
        put(c, p, head, col, float("nan"))
    out, lse = run(c, claim)
    want = paged.definition(c)
    assert torch.isnan(want[0]).sum() == rows * 4 * 3
    check(c, out, lse, few=eight, want=want)


@pytest.mark.parametrize("far_first", [True, False])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_an_infinity_of_a_far_part_is_not_lost(hd, sign, far_first):
    c = far_case(2, hd, False, far_first, window=L)
    put(c, (0 if far_first else FAR) + 1900, 1, 5, sign * float("inf"))
    out, _ = run(c, L)
    odd = ~torch.isfinite(out.view(2, 8, hd))
    assert odd[:, 4:, 5].all() and int(odd.sum()) == 2 * 4
