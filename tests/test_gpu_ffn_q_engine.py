"""Models whose feed-forward network runs in 8 bits (SD_DTYPE_BF16_FFN_Q), through the engine's prefill, draft and verify
passes, against a float64 model with codes at the same places."""
import functools

import numpy as np
import pytest

import qref
import synth
from oracle import model as om
from sdcase import run_gpu_steps, say

pytestmark = pytest.mark.gpu


class FFNQ(om.Model):
    """A bf16 model (fp16 operands) whose feed-forward products read codes: the oracle's layers, one row set at a time."""

    def codes(self, x):
        return qref.row_values(*qref.quantise_rows(x.astype(np.float32).astype(np.float64)), x.shape[1])

    @functools.cached_property
    def quantised(self):
        s, w = self.s, dict(self.w)
        for l in range(s.n_layers):
            g, u = w[f"l{l}.w_gate"], w[f"l{l}.w_up"]
            gu = np.stack([g.reshape(-1, 16, s.d_model), u.reshape(-1, 16, s.d_model)], 1).reshape(2 * s.d_ffn, s.d_model)
            v = qref.weight_values(*qref.quantise_weight(gu)).reshape(-1, 2, 16, s.d_model)
            w[f"l{l}.w_gate"], w[f"l{l}.w_up"] = (v[:, i].reshape(s.d_ffn, s.d_model) for i in (0, 1))
            w[f"l{l}.w_down"] = qref.weight_values(*qref.quantise_weight(w[f"l{l}.w_down"]))
        return w

    def logits(self, toks, n):
        s, w, q = self.s, self.ops, self.quantised
        pos = np.arange(len(toks))
        x = w["embed"][np.asarray(toks)]
        for l in range(s.n_layers):
            p = f"l{l}."
            h = self.r(om.rmsnorm(x, w[p + "attn_norm"], s.rms_eps))
            heads = lambda m, k: (h @ w[p + m].T).reshape(-1, k, s.head_dim)
            qq, kk = om.rope(heads("wq", s.n_heads), pos, s.rope_theta), self.r(om.rope(heads("wk", s.n_kv_heads), pos, s.rope_theta))
            o = om.causal_attention(qq, kk, self.r(heads("wv", s.n_kv_heads)), 0).reshape(len(toks), -1)
            x = x + self.r(o) @ w[p + "wo"].T
            h = self.codes(om.rmsnorm(x, w[p + "ffn_norm"], s.rms_eps))
            x = x + self.codes(om.silu(h @ q[p + "w_gate"].T) * (h @ q[p + "w_up"].T)) @ q[p + "w_down"].T
        return self.r(om.rmsnorm(x[-n:], w["final_norm"], s.rms_eps)) @ w["lm_head"].T


def engine(shape, draft, tw, dw, B, gamma, ctx, **kw):
    from paper_2510_11331_amd import SDEngine
    return SDEngine(shape, draft, tw.__getitem__, dw.__getitem__, max_slots=B, max_batch=B, gamma_max=gamma, max_ctx=ctx, **kw)


SHAPES = {"mha": synth.ModelShape(2, 256, 4, 4, 512, 1008, "bf16"), "odd": synth.ModelShape(2, 320, 5, 1, 448, 1008, "bf16")}
LONG = synth.ModelShape(2, 256, 4, 4, 10304, 1008, "bf16")
DRAFT = synth.ModelShape(1, 192, 3, 1, 320, 1008, "bf16")


@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("lens,gamma", [((37, 5), 3), ((130, 71, 9, 66, 20, 33, 8, 90, 3, 50, 64, 17, 25, 40), 4)])
def test_verify_logits(name, lens, gamma):
    """8 and 70 verified rows (streaming and row tiles), prompts in chunks of 64 and 256 rows.  What separates the two sides:
    a value on the border of two codes (2^-3 apart) falls on either side where the 16-bit operands before it differ in
    their last place (2^-11): a share of 2^-11 / 2^-4 = 2^-7 of the codes, 2^-3 sqrt(2^-7) = 1.1 % of a feed-forward
    output, whose part of a logit is at most all of it; two layers, three sets of codes each: 3 % is under sqrt(6) times that."""
    say("ffn_q verify", name, lens)
    check_verify(SHAPES[name], lens, gamma)


@pytest.mark.parametrize("lens,gamma", [((37, 5), 3), ((130, 71, 9, 66, 20, 33, 8, 90, 3, 50, 64, 17, 25, 40), 4)])
def test_verify_logits_ranges(lens, gamma):
    """A feed-forward width whose down projection takes K in ranges (with 8 and 70 rows, and in prefill), which the next norm
    adds: as above."""
    say("ffn_q verify ranges", lens)
    check_verify(LONG, lens, gamma)


def check_verify(shape, lens, gamma):
    tw, dw = synth.model_weights(shape, 5), synth.model_weights(DRAFT, 6)
    prompts = synth.prompts(len(lens), list(lens), shape.vocab)
    model = FFNQ(shape, tw)
    for rows in (64, 256):
        eng = engine(shape, DRAFT, tw, dw, len(lens), gamma, max(lens) + 2 * gamma + 16, prefill_rows=rows, ffn_q=True)
        _, _, b, z = run_gpu_steps(eng, list(range(len(lens))), prompts, gamma, 1, 9, list(range(len(lens))), keep_logits=True)
        assert eng.check_flags() == 0
        drafts = b.draft_tok.cpu().numpy()
        eng.close()
        for k, p in enumerate(prompts):
            ref = model.logits(list(p) + [int(t) for t in drafts[k]], gamma + 1)
            err = np.linalg.norm(z[0, k] - ref) / np.linalg.norm(ref)
            assert err < 0.03, (rows, k, err)


def test_draft_distribution_and_steps():
    """A draft with an 8-bit feed-forward: its distributions are those of its model; steps by graph replay equal eager
    ones bit for bit; the plain engine beside it is not touched."""
    import torch
    from paper_2510_11331_amd import StepGraph
    from paper_2510_11331_amd.engine import uniforms_device
    say("ffn_q draft")
    shape = SHAPES["odd"]
    tw, dw = synth.model_weights(shape, 5), synth.model_weights(DRAFT, 6)
    prompts = synth.prompts(3, [20, 33, 7], shape.vocab)
    u = uniforms_device(synth.uniform_table(3, [0, 1, 2], 4, 3))
    runs = []
    for graph in (False, True):
        eng = engine(shape, DRAFT, tw, dw, 3, 3, 80, ffn_q=True, draft_ffn_q=True)
        eng.prefill([0, 1, 2], prompts, [30] * 3)
        b = eng.batch([0, 1, 2], 3)
        eng.draft_step(b, 0, u[0])
        q0 = b.q[:, 0].clone()
        step = StepGraph(eng, b).run if graph else (lambda x: eng.step(b, x))
        out = []
        for n in range(4):
            step(u[n])
            out.append((b.n_acc.clone(), b.out_tok.clone(), b.p.clone()))
        torch.cuda.synchronize()
        assert eng.check_flags() == 0
        runs.append((q0, out))
        eng.close()
    assert torch.equal(runs[0][0], runs[1][0])
    assert all(torch.equal(x, y) for a, c in zip(runs[0][1], runs[1][1]) for x, y in zip(a, c))
    model = FFNQ(DRAFT, dw)
    for k, p in enumerate(prompts):
        z = model.logits(list(p), 1)[0]
        q = np.exp(z - z.max())
        q /= q.sum()
        # logits of these models are within +- 2: an error of 3 % of their norm (as above) moves a probability by as much of it
        assert np.abs(runs[0][0][k].double().cpu().numpy() / q - 1).max() < 2 * 0.03 * np.abs(z).max() + 1e-3


def test_static_workspace():
    import torch
    from paper_2510_11331_amd.engine import uniforms_device
    say("ffn_q static workspace")
    shape = SHAPES["mha"]
    tw, dw = synth.model_weights(shape, 5), synth.model_weights(DRAFT, 6)
    prompts = synth.prompts(2, [20, 33], shape.vocab)
    u = uniforms_device(synth.uniform_table(3, [0, 1], 1, 3))
    got = []
    for static in (False, True):
        eng = engine(shape, DRAFT, tw, dw, 2, 3, 80, ffn_q=True, static_workspace=static, prefill_rows=64)
        eng.prefill([0, 1], prompts, [30] * 2)
        b = eng.batch([0, 1], 3)
        eng.step(b, u[0])
        torch.cuda.synchronize()
        got.append(b.p.clone())
        eng.close()
    assert torch.equal(*got)
