"""The shared cache's operators together: the example of forked continuations against dense attention in 64
bits, and the engine's prompt attention switch against the oracle."""
import os
import sys

import pytest
import torch

import parity
from conftest import ROOT
from paper_2511_09844_gb300 import sd2
from paper_2511_09844_gb300 import workloads as W

sys.path.insert(0, os.path.join(ROOT, "examples"))
import shared_prompt  # noqa: E402

pytestmark = pytest.mark.gpu


def _dense(model, layer, tokens, rows):
    """(output, sum_j p_j |v_j|) of the last `rows` rows over the sequence's own tokens, in float64 on the CPU."""
    x = model.qkv[layer][torch.tensor(tokens, device="cuda")].double().cpu()
    q, k, v = x.split((model.heads, model.kv_heads, model.kv_heads), dim=1)
    rep = model.heads // model.kv_heads
    k, v = k.repeat_interleave(rep, 1), v.repeat_interleave(rep, 1)
    n = len(tokens)
    z = torch.einsum("rhd,khd->hrk", q[n - rows:], k) / model.head_dim ** 0.5
    z.masked_fill_(torch.arange(n)[None, :] > torch.arange(n - rows, n)[:, None], float("-inf"))
    w = torch.softmax(z, -1)
    return torch.einsum("hrk,khd->rhd", w, v).reshape(rows, -1), torch.einsum("hrk,khd->rhd", w, v.abs()).reshape(rows, -1)


@pytest.mark.parametrize("heads,kv_heads,head_dim", [(32, 8, 128), (14, 2, 64)])
def test_forked_continuations(heads, kv_heads, head_dim):
    """Reading, forking, decoding, rolling back, dropping and compacting: every output of every step is that of the
    sequence alone. Both kernels round probabilities and results to bf16, 2^-8 relative each."""
    model, steps = shared_prompt.run(heads=heads, kv_heads=kv_heads, head_dim=head_dim)
    assert len(steps) == 4
    for outs, seqs, rows in steps:
        for layer in range(model.layers):
            for got, tokens, n in zip(outs[layer], seqs, rows):
                o, mag = _dense(model, layer, tokens, n)
                bound = 2 ** -8 * (mag + o.abs()) + 2e-4 * mag
                assert ((got.cpu().double() - o).abs() - bound).max().item() <= 1e-6


class _PromptEngine(sd2.SD2Engine):
    """The engine with its prompts through the prompt attention kernel."""

    def prefill(self, *args, **kw):
        self.set_prompt_attention(True)
        return super().prefill(*args, **kw)


@pytest.mark.parametrize("graphs", [True, False])
def test_prompts_through_prompt_attention(monkeypatch, graphs):
    """A ragged batch with grouped heads: prefill logits, taps and every decision after it against the oracle."""
    monkeypatch.setattr(sd2, "SD2Engine", _PromptEngine)
    work = parity.tiny_work(verifier=W.shrink(W.TINY_V, n_kv_heads=2), k=3)
    vw, dw, st = parity.tiny_weights(work, seed=31)
    prompts = [W.make_prompts(work.verifier.vocab, 1, (n, n), seed=n)[0] for n in (1, 16, 17, 65, 130)]
    rep = parity.run(work, vw, dw, st, prompts, [1.0, 0.0, 0.7, 1.0, 0.0], seed=5, n_steps=3, graphs=graphs)
    assert rep.decisions > 40


def test_prompts_with_wide_heads(monkeypatch):
    """Heads of 128, four per KV head, a prompt over several K/V tiles."""
    monkeypatch.setattr(sd2, "SD2Engine", _PromptEngine)
    shape = W.shrink(W.TINY_V, n_heads=8, n_kv_heads=2, head_dim=128, n_layers=4)
    work = parity.tiny_work(verifier=shape, k=2)
    vw, dw, st = parity.tiny_weights(work, seed=32)
    parity.run(work, vw, dw, st, W.make_prompts(shape.vocab, 2, (300, 301), seed=8), [1.0, 0.0], seed=6, n_steps=2)


def test_the_switch_changes_nothing_when_off():
    """Off, on, off again: the decode kernel's prefill gives its bits back; on, the logits agree within rounding."""
    work = parity.tiny_work()
    vw, dw, st = (parity.to_device(x) for x in parity.tiny_weights(work, seed=33))
    prompts = W.make_prompts(work.verifier.vocab, 1, (90, 90), seed=9)
    eng = sd2.SD2Engine(work, vw, dw, st, max_batch=1, max_ctx=128, max_prefill_tokens=90)
    try:
        got = []
        for on in (None, True, False):
            if on is not None:
                eng.set_prompt_attention(on)
            eng.prefill(prompts, [0.0], 3)
            got.append(eng.buffer(sd2.BUF_TARGET).view(work.k + 1, -1)[0].clone())
            eng.check()
        assert torch.equal(got[0], got[2])
        assert parity.row_rel_err(got[1], got[0]) <= 2e-2
    finally:
        eng.close()
