"""Scores of the 8-bit cache's attention over all exponents: keys under any exponent byte from 10 to 246 and queries of any
magnitude, by each of the three ways (few vectors, tiles, prompts). Bounds are those of test_gpu_quantized.py.

A query times 2^p and keys times 2^-p leave the scores as they were. In the kernels of few vectors and of tiles the powers of two
are applied exactly, whatever they are. Prompts multiply bf16 numbers, which are to be normal ones (queries of 2^-110 on)."""
import pytest
import torch

import paged
from paper_2511_09844_gb300 import sd2
from test_gpu_quantized import check
from test_gpu_quantized import run as run_case

pytestmark = pytest.mark.gpu

# rows and cached lengths that go through the kernel of few vectors, of tiles, and of prompts (8/2 heads), and the length the call is
# told (40 vectors and more go by tiles where caches are long)
WAYS = {"few": ([1, 3], [300, 1200]), "tiles": ([10, 12], [300, 1200]), "prompts": ([150, 200], [300, 1200])}
CLAIM = {"few": 1200, "tiles": 1 << 20, "prompts": 1200}


def run(c, way):
    need = sd2.load_library().sd2_attention_quantized_workspace_bytes(sum(c["rows"]), 2, 8, 2, c["hd"], CLAIM[way], c["pool"].shape[1], c["window"],
                                                                      c["sinks"])
    if way != "prompts" and not c["window"]:  # (a tile's parts of 128 vectors show in the workspace; what a small window sees goes by few)
        assert (need > 2 * 148 * 128 * (c["hd"] + 4) * 4) == (way == "tiles")
    return run_case(c, max_kv=CLAIM[way])


def moved(way, hd, q_power, k_power, window=0, shrink=0):
    """Queries times 2^q_power, keys' exponents k_power higher (within the range), keys' values before scaling 2^shrink smaller."""
    c = paged.case(*WAYS[way], 8, 2, hd, seed=9, eight=True, spread=0.0, window=window)
    c["q"] = (c["q"].double() * 2.0 ** q_power).to(torch.bfloat16)
    ids = torch.cat([c["table"][s, : (n + 15) // 16] for s, n in enumerate(c["kv"])]).long()
    b = c["scale"][c["layer"], ids, 0].long() + k_power
    c["scale"][c["layer"], ids, 0] = b.clamp(paged.LOW, paged.HIGH).to(torch.uint8)
    if shrink:
        raw = c["pool"][c["layer"]].float()
        raw[:, 0] *= 2.0 ** -shrink
        raw = raw.to(torch.float8_e4m3fn).view(torch.uint8)
        c["pool"].view(torch.uint8)[c["layer"]] = raw
    return c, b


@pytest.mark.parametrize("window", [0, 100])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("way,power", [("few", -125), ("few", -118), ("few", -112), ("few", 110), ("tiles", -125), ("tiles", -118),
                                       ("tiles", -112), ("tiles", 110), ("prompts", -110), ("prompts", 110)])
def test_keys_at_the_ends_of_the_exponents(way, power, hd, window):
    c, b = moved(way, hd, power, -power, window)
    assert (b.max() > 228 if power < 0 else b.min() < 12)
    assert torch.isfinite(c["q"].float()).all() and c["q"].float().abs().max() > 0
    want = paged.definition(c)
    assert want[1].abs().max() < 100
    out, lse, err = run(c, way)
    assert err == 0
    check(c, out, lse, few=way != "prompts", want=want)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("way", ["few", "tiles"])
def test_the_largest_queries(way, hd):
    """Elements of some 2^121 to 2^125 on keys that are small under the smallest exponents."""
    c, b = moved(way, hd, 121, -110, shrink=8)
    c["q"] = (c["q"].double() * torch.exp2(-3.0 - torch.arange(c["q"].shape[1]).double() % 4)[:, None]).to(torch.bfloat16)
    c["q"][0, 0] = 0.0
    c["q"][0, 0, 5] = 2.0 ** 125
    assert b.min() >= paged.LOW and torch.isfinite(c["q"].float()).all() and c["q"].float().abs().max() > 2.0 ** 120
    want = paged.definition(c)
    assert want[1].abs().max() < 100
    out, lse, err = run(c, way)
    assert err == 0
    check(c, out, lse, want=want)


@pytest.mark.parametrize("window", [0, 100, 1000])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("way,q_power,k_power", [("few", -80, -80), ("few", -125, -110), ("tiles", -80, -80), ("tiles", -125, -110),
                                                 ("tiles", -60, -90), ("prompts", -80, -80)])
def test_scores_that_are_all_but_zero(way, q_power, k_power, hd, window):
    """Products far below fp32's smallest number: every position that is seen has the same weight."""
    c, _ = moved(way, hd, q_power, k_power, window)
    out, lse, err = run(c, way)
    assert err == 0
    check(c, out, lse, few=way != "prompts")


def leads(c):
    """For each row and head, how far the best score lies above the second, and the most that a computed score may be off: each
    of hd sums rounds (or cuts off) up to 2^-23 of at most |q| . |k| / sqrt(hd), each element of q up to 2^-25 of the largest."""
    H, Hkv, hd = c["H"], c["Hkv"], c["hd"]
    lead, off = [], []
    for s, (n, L) in enumerate(zip(c["rows"], c["kv"])):
        kv = paged.blocks(c, c["table"][s, : (L + 15) // 16].long())
        k = kv[:, 0].transpose(0, 1).reshape(Hkv, -1, hd)[:, :L].repeat_interleave(H // Hkv, 0)
        r0 = int(c["cu"][s])
        q = c["q"][r0:r0 + n].double()
        z = torch.einsum("rhd,hkd->rhk", q, k).masked_fill(~paged.seen(c, n, L)[:, None], float("-inf")) / hd ** 0.5
        two = z.topk(2, -1).values
        lead.append(two[..., 0] - two[..., 1])
        off.append((hd + 8) * 2.0 ** -23 * (q.abs().amax(-1)[..., None] * k.abs().sum(-1)[None]).amax(-1) / hd ** 0.5)
    return torch.cat(lead), torch.cat(off)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("way", ["few", "tiles"])
def test_scores_near_the_largest_number(way, hd):
    """Scores of some 2^126 whose products q . k, sqrt(hd) times as large, lie beyond fp32's range: the best position takes
    everything."""
    c, b = moved(way, hd, -1, 125)
    assert b.max() <= paged.HIGH
    o, l, mag = paged.definition(c)
    assert l.max() * hd ** 0.5 > 2.0 ** 128 and l.max() < 2.0 ** 127
    lead, off = leads(c)
    clear = lead > 2 * off + 100
    assert clear.double().mean() > 0.8
    out, lse, err = run(c, way)
    assert err == 0
    assert ((lse.double() - l).abs() <= off + 1).all()
    good = (out.double() - o).abs() <= 2 ** -8 * o.abs() + (2 ** -11 + 2e-4) * mag + 1e-6
    assert good.view(*clear.shape, hd)[clear].all()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("way", ["few", "tiles", "prompts"])
def test_scores_beyond_the_largest_number(way, hd):
    """Not zeros, as for a row that sees nothing: the best position takes everything, its score's log-sum-exp is infinite in fp32; or, of
    prompts, NaN, as a softmax in fp32 gives it."""
    c, _ = moved(way, hd, 12, 125)
    out, lse, err = run(c, way)
    assert err == 0
    if way == "prompts":
        assert torch.isnan(out).all() and torch.isnan(lse).all()
        return
    o, l, mag = paged.definition(c)
    lead, off = leads(c)
    clear = lead > 2 * off + 100
    assert clear.double().mean() > 0.8 and l.min() > 2.0 ** 130
    assert (lse == float("inf")).all()
    good = (out.double() - o).abs() <= 2 ** -8 * o.abs() + (2 ** -11 + 2e-4) * mag + 1e-6
    assert good.view(*clear.shape, hd)[clear].all()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("way", ["few", "tiles"])
def test_the_largest_queries_on_the_largest_keys(way, hd):
    """Beyond fp32 even before the query's power: NaN, or the best position's value, but no zeros."""
    c, _ = moved(way, hd, 125, 125)
    assert torch.isfinite(c["q"].float()).all()
    out, lse, err = run(c, way)
    assert err == 0
    nan = torch.isnan(lse)[..., None].expand(*lse.shape, hd).reshape(out.shape)
    assert torch.equal(torch.isnan(out), nan)
    assert nan.any() and ((lse == float("inf")) | torch.isnan(lse)).all()


@pytest.mark.parametrize("power", [-117, 119])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("way,claim", [("few", 6000), ("few", 64), ("tiles", 1 << 20)])
def test_values_at_the_ends_of_the_exponents(way, claim, hd, power):
    """V under the smallest or the largest exponent, with scores that rise after the first pages by less than moves a row's reference, so
    that its sum is far above 1; items cut into parts, and (a cache that is said to be short) a whole one."""
    c = paged.case([1] if way == "few" else [12], [6000], 8, 2, hd, seed=1, eight=True, spread=0.0)
    ids = c["table"][0, : 375].long()
    c["scale"][c["layer"], ids, 1] = paged.BIAS + power
    c["pool"].view(torch.uint8)[c["layer"], ids, 1] &= 0x7F                # (no sums that cancel)
    k = torch.full((6000, 2, hd), 8.6 / (4 * hd ** 0.5))
    k[:256] = 0.0                           # (the first two pages of each of a block's eight warps)
    pool, scale = paged.quantized(k.view(375, 16, 2, hd).transpose(1, 2))
    c["pool"].view(torch.uint8)[c["layer"], ids, 0] = pool.view(torch.uint8)
    c["scale"][c["layer"], ids, 0] = scale
    c["q"] = torch.full_like(c["q"], 4.0)
    o, l, mag = paged.definition(c)
    out, lse, err = run_case(c, max_kv=claim)
    assert err == 0
    assert (lse.double() - l).abs().max() <= 4e-4
    # (a result near 2^-117 is a normal bf16 number or off by at most half the smallest subnormal, 2^-134)
    assert ((out.double() - o).abs() <= 2 ** -8 * o.abs() + (2 ** -11 + 2e-4) * mag + 2.0 ** -134).all()
