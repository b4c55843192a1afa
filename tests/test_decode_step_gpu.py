"""The decoding operators together, as a program uses them after a prefill: beam search token by token on a small model, built from
the framework's operators, against the oracle, which prefills every hypothesis from the start."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle as S
from oracle import decoder_oracle as D
from paper_2412_11272_amd import binding as wf
from paper_2412_11272_amd import synth
from tests import helpers as H

pytestmark = pytest.mark.gpu

F8, F32 = torch.float8_e4m3fn, torch.float32
SHAPE = synth.DEC_SHAPES["unit"]
ENC, PROMPTS, W, STEPS = [37, 150, 64], [5, 1, 30], 4, 5


def _i32(x):
    return torch.tensor(np.asarray(x, np.int32), device="cuda")


class Model:
    """One decoding step from operators, in fp32.  Self-attention caches: a slot of n_ctx rows for every beam, or one of a stream's beams together
    (`shared`), where a beam sees the prompt and its own tokens by its mask."""

    def __init__(self, dtype, shared):
        self.dtype, self.shared = dtype, shared
        self.w = synth.make_decoder_weights(SHAPE, 31, q_scale=4.0, affine_random=True)
        self.enc = synth.make_enc_states(sum(ENC), SHAPE.d_model, 32)
        self.prompts = synth.make_prompts(PROMPTS, SHAPE.n_vocab, 33)
        self.cu_enc = np.concatenate([[0], np.cumsum(ENC)]).astype(np.int32)
        d, B = SHAPE.d_model, len(ENC)
        g = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()  # noqa: E731
        self.layers = [{**{k: g(v) for k, v in lw.items()}, "wqkv": g(np.concatenate([lw["wq"], lw["wk"], lw["wv"]])),
                        "bqkv": g(np.concatenate([lw["bq"], 0 * lw["bq"], lw["bv"]]))} for lw in self.w["layers"]]
        self.tok, self.pos, self.fg, self.fb = g(self.w["tok_emb"]), g(self.w["pos_emb"]), g(self.w["lnf_g"]), g(self.w["lnf_b"])
        vpad = -(-SHAPE.n_vocab // 128) * 128
        self.tok_pad = torch.zeros((vpad, d), device="cuda")
        self.tok_pad[:SHAPE.n_vocab] = self.tok
        self.zero = torch.zeros(vpad, device="cuda")

        dec = wf.Decoder(SHAPE, self.w, B, sum(ENC), sum(PROMPTS), wf.WF_PRECISION_F32)
        cross = dec.cross_kv(g(self.enc))
        r = dec.prefill(self.prompts, self.cu_enc, cross, want_self_kv=True)
        torch.cuda.synchronize()
        dec.close()
        self.logits0 = r["logits"]
        slots = B if shared else B * W
        self.cross, self.own = [], []
        self.data = torch.zeros((SHAPE.n_layers, slots, SHAPE.n_ctx, 2 * d), device="cuda") if dtype == F32 else \
            torch.zeros((SHAPE.n_layers, slots, SHAPE.n_ctx, SHAPE.n_heads, 2, 64), dtype=torch.uint8, device="cuda").view(F8)
        self.exps = None if dtype == F32 else torch.zeros((SHAPE.n_layers, 2 * SHAPE.n_heads, slots * SHAPE.n_ctx), dtype=torch.uint8, device="cuda")
        first = _i32([s * SHAPE.n_ctx * (1 if shared else W) for s in range(B)])
        for l in range(SHAPE.n_layers):
            c = wf.Cache.empty(sum(ENC), SHAPE.n_heads, dtype)
            wf.op_cache_write(c, cross[l][:, :d], cross[l][:, d:], _i32([0, sum(ENC)]), _i32([0]))
            self.cross.append(c)
            o = wf.Cache(self.data[l].view(slots * SHAPE.n_ctx, *self.data.shape[3:]), None if dtype == F32 else self.exps[l])
            wf.op_cache_write(o, r["self_kv"][l][:, :d], r["self_kv"][l][:, d:], _i32(r["cu_prompt"]), first)
            self.own.append(o)
        if shared:      # bit i of a beam's words: row prompt + i of the stream's cache is one of its own tokens
            self.mask = torch.zeros((1, B * W, 1, 2), dtype=torch.int32, device="cuda")

    def logits(self, tokens, t, write=True):
        """Logits [B, W, n_vocab] behind the t-th token (t >= 0) of every beam."""
        d, B, R = SHAPE.d_model, len(ENC), len(ENC) * W
        at = np.repeat(PROMPTS, W) + t
        x = self.tok[tokens.view(-1).long()] + self.pos[_i32(at).long()]
        h = torch.empty((R, SHAPE.d_mlp), device="cuda")
        u, q, qkv = torch.empty_like(x), torch.empty_like(x), torch.empty((R, 3 * d), device="cuda")
        P = wf.WF_PRECISION_F32
        if self.shared:
            new_at, new_cu = _i32([s * SHAPE.n_ctx + PROMPTS[s] + t * W for s in range(B)]), _i32(np.arange(B + 1) * W)
            rows, cu = _i32(np.arange(B) * SHAPE.n_ctx), new_cu
            lens, since = _i32([PROMPTS[s] + (t + 1) * W for s in range(B)]), _i32(PROMPTS)
            bit = np.arange(R) % W + t * W
            if write:
                own = self.mask.view(R, 2)
                own[torch.arange(R), torch.from_numpy(bit // 32).cuda()] |= _i32(np.int32(1) << (bit % 32))
            seen = dict(mask=self.mask.view(R, 2), mask_from=since, max_q=W, max_len=SHAPE.n_ctx)
        else:
            rows, cu, lens = _i32(np.arange(R) * SHAPE.n_ctx), _i32(np.arange(R + 1)), _i32(at + 1)
            new_at, new_cu = _i32(np.arange(R) * SHAPE.n_ctx + at), cu
            seen = dict(max_q=1, max_len=SHAPE.n_ctx)
        for lw, own, cross in zip(self.layers, self.own, self.cross):
            wf.op_layernorm(x, lw["ln1_g"], lw["ln1_b"], u)
            wf.op_linear(P, u, lw["wqkv"], lw["bqkv"], qkv, 0)
            if write:
                wf.op_cache_write(own, qkv[:, d:2 * d], qkv[:, 2 * d:], new_cu, new_at)
            wf.op_cache_attention(own, qkv[:, :d], cu, rows, lens, out=u, **seen)
            wf.op_linear(P, u, lw["wo"], lw["bo"], x, 2)
            wf.op_layernorm(x, lw["lnx_g"], lw["lnx_b"], u)
            wf.op_linear(P, u, lw["xwq"], lw["xbq"], q, 0)
            wf.op_cache_attention(cross, q, _i32(np.arange(B + 1) * W), _i32(self.cu_enc[:-1]), _i32(ENC), W, max(ENC), out=u)
            wf.op_linear(P, u, lw["xwo"], lw["xbo"], x, 2)
            wf.op_layernorm(x, lw["ln2_g"], lw["ln2_b"], u)
            wf.op_linear(P, u, lw["w1"], lw["b1"], h, 1)
            wf.op_linear(P, h, lw["w2"], lw["b2"], x, 2)
        wf.op_layernorm(x, self.fg, self.fb, u)
        out = torch.empty((R, self.tok_pad.shape[0]), device="cuda")
        wf.op_linear(P, u, self.tok_pad, self.zero, out, 0)
        return out.view(B, W, -1)[:, :, :SHAPE.n_vocab]

    def move(self, parents, t):
        """The beams' states behind their new owners, after t own tokens."""
        if self.shared:
            wf.op_beam_reorder(self.mask, parents)
            return
        lens = _i32(np.asarray(PROMPTS) + t)
        wf.op_beam_reorder(self.data.view(torch.uint8) if self.dtype == F8 else self.data, parents, lens=lens)
        if self.dtype == F8:
            n = self.exps.shape[0] * self.exps.shape[1]
            wf.op_beam_reorder(self.exps.view(n, -1, SHAPE.n_ctx), parents, lens=lens)

    def search(self, keep_slots):
        B = len(ENC)
        first = self.logits0[:, None].expand(B, W, -1).contiguous()
        tok, par, sc, _ = wf.op_beam_select(first, torch.zeros((B, W), device="cuda"), n_in=_i32([1] * B), keep_slots=keep_slots)
        yield first, tok, par, sc
        self.move(par, 0)
        for t in range(STEPS):
            x = self.logits(tok, t)
            tok, par, sc, _ = wf.op_beam_select(x, sc, keep_slots=keep_slots)
            yield x, tok, par, sc
            self.move(par, t + 1)
        self.last = (tok, t + 1)


@pytest.mark.parametrize("keep_slots", [False, True], ids=["by-rank", "keep-slots"])
@pytest.mark.parametrize("shared", [False, True], ids=["slots", "shared"])
def test_beam_search_equals_the_oracles(shared, keep_slots):
    m = Model(F32, shared)
    hyps, scores = [[[]] * W for _ in ENC], np.zeros((len(ENC), W))
    for t, (x, tok, par, sc) in enumerate(m.search(keep_slots)):
        torch.cuda.synchronize()
        for s in range(len(ENC)):
            enc = m.enc[m.cu_enc[s]:m.cu_enc[s + 1]]
            ref = np.stack([D.prefill_stream(m.w, SHAPE.n_heads, list(m.prompts[s]) + hyps[s][b], enc)["logits"] for b in range(W if t else 1)])
            assert H.rel_err(x[s, :len(ref)].cpu().numpy(), ref) <= H.F32_TOL, (t, s)
            full = np.concatenate([ref, np.zeros((W - len(ref), ref.shape[1]))])
            rt, rp, rs, _ = S.beam_step(full, scores[s], W if t else 1, W, keep_slots=keep_slots)
            assert tok[s].tolist() == rt.tolist() and par[s].tolist() == rp.tolist(), (t, s)
            np.testing.assert_allclose(sc[s].cpu().numpy(), rs, atol=1e-3)
            hyps[s] = [hyps[s][p] + [int(k)] for p, k in zip(rp, rt)]
            scores[s] = rs


@pytest.mark.parametrize("shared", [False, True], ids=["slots", "shared"])
def test_a_search_over_quantised_caches(shared):
    """In 8 bits: the logits of a step equal those over 32-bit caches that hold what the quantised ones stand for."""
    m = Model(F8, shared)
    for _ in m.search(False):
        pass
    tok, t = m.last
    x = m.logits(tok, t)
    own, cross = m.own, m.cross

    def read(c):
        return wf.Cache(wf.op_cache_read(c, _i32([0, c.n_rows]), _i32([0]), c.n_rows, out_dtype=F32))

    m.own, m.cross = [read(c) for c in own], [read(c) for c in cross]
    ref = m.logits(tok, t, write=False)
    torch.cuda.synchronize()
    assert torch.isfinite(x).all() and H.rel_err(x.cpu().numpy(), ref.double().cpu().numpy()) <= H.F32_TOL
