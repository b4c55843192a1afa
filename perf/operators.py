"""Timing cases of the operators of token-by-token decoding: what a streaming-recognition program runs on the GPU after a
round's prompt prefill, once per token.

A program keeps the keys and values of its streams in caches, lets every step's queries attend to them, picks the best
continuations of each stream's beams and moves the beams' caches behind their new owners.

kinds   write     key / value rows of new tokens into a cache, in 8 bits (e4m3 with a power of two for each row and head) or as they are
        read      cache rows back into the activation type
        attend    a few queries per sequence (one token, the beams of a stream, a tree of drafted tokens) over its cache
        select    the best continuations of every stream's beams over the whole vocabulary
        reorder   the cache slots of a stream's beams take over their parents' contents

Where `own` is false the operators run in their plain form, in elementary torch operations; where it is true the
framework's entry points are called.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

HEAD = 64
BEAMS = 5
VOCAB = 51866
CONTEXT = 448
MIN_TOKENS, MAX_TOKENS = 51, 1525          # encoder tokens of 0.5 s and of 30 s of audio, hush segment included
HEADS = [(6, 6), (8, 8), (12, 12), (16, 16), (20, 20)]      # query heads, key / value heads of the models
SHARED = [(16, 4), (32, 8), (20, 4), (24, 8)]               # the same with key / value heads shared by several query heads


def listed():
    return [
        # a loaded server's round: the cross-attention keys and values of one layer, 64 ragged streams, packed
        {"name": "write-round", "kind": "write", "seqs": 64, "lo": MIN_TOKENS, "hi": MAX_TOKENS, "heads": 20, "src": "bf16", "cache": "f8"},
        # one step of the same server: each beam's new token goes behind the tokens it has
        {"name": "write-step", "kind": "write", "seqs": 64 * BEAMS, "lo": 1, "hi": 1, "heads": 20, "src": "bf16", "cache": "f8"},
        # a layer's keys and values back in the activation type, for a prompt that is prefilled again
        {"name": "read-round", "kind": "read", "seqs": 64, "lo": MIN_TOKENS, "hi": MAX_TOKENS, "heads": 20, "cache": "f8", "out": "bf16"},
        # the same for one speaker, 4 s of audio, in 32 bits
        {"name": "read-one", "kind": "read", "seqs": 1, "lo": 225, "hi": 225, "heads": 8, "cache": "f8", "out": "f32"},
        # one speaker, one new token, self-attention: the call whose latency adds up
        _attend("attend-one", 1, 1, 1, 225, 225, 8, 8, "bf16", "bf16"),
        # cross-attention of a loaded server's step: five beams share their stream's encoder tokens
        _attend("attend-round", 64, BEAMS, BEAMS, MIN_TOKENS, MAX_TOKENS, 20, 20, "bf16", "f8"),
        # verification of drafted trees over long caches, heads shared in groups of four
        _attend("attend-draft", 4, 17, 40, 20000, 65536, 32, 8, "bf16", "bf16", tree=True),
        # the 32-bit check of the middle model: every beam over a cache of its own
        _attend("attend-beams-f32", 16 * BEAMS, 1, 1, 90, CONTEXT, 16, 16, "f32", "f32"),
        # one speaker, five beams
        {"name": "select-one", "kind": "select", "streams": 1, "width": BEAMS, "vocab": VOCAB, "src": "f32", "ragged": False, "done": False},
        # a loaded server's step
        {"name": "select-round", "kind": "select", "streams": 64, "width": BEAMS, "vocab": VOCAB, "src": "f32", "ragged": False, "done": False},
        # self-attention caches of one speaker's beams on the base model, all layers
        {"name": "reorder-one", "kind": "reorder", "streams": 1, "width": BEAMS, "layers": 6, "positions": CONTEXT, "lo": 131, "hi": 131, "values": 1024, "type": "bf16"},
        # those of a loaded server, two layers of the large model
        {"name": "reorder-round", "kind": "reorder", "streams": 64, "width": BEAMS, "layers": 2, "positions": CONTEXT, "lo": 90, "hi": 320, "values": 2560, "type": "bf16"},
    ]


def _attend(name, seqs, q_lo, q_hi, lo, hi, heads, kv_heads, act, cache, tree=False):
    return {"name": name, "kind": "attend", "seqs": seqs, "q_lo": q_lo, "q_hi": q_hi, "lo": lo, "hi": hi, "heads": heads, "kv_heads": kv_heads,
            "act": act, "cache": cache, "tree": tree}


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999)))))))


def draw(rng: random.Random):
    kind = rng.choice(["write", "read", "attend", "attend", "select", "reorder"])
    if kind in ("write", "read"):
        seqs, heads = _log(rng, 1, 320), rng.choice(HEADS)[1]
        hi = _log(rng, 1, min(MAX_TOKENS, 500_000 // (heads * seqs)))
        case = {"kind": kind, "seqs": seqs, "lo": rng.randint(0, hi), "hi": hi, "heads": heads}
        if kind == "write":
            return {**case, "src": rng.choice(["f32", "bf16"]), "cache": rng.choice(["f8", "f8", "bf16", "f32"])}
        return {**case, "cache": rng.choice(["f8", "f8", "bf16", "f32"]), "out": rng.choice(["f32", "bf16"])}
    if kind == "attend":
        heads, kv = rng.choice(HEADS + SHARED)
        seqs, tree = _log(rng, 1, 320), rng.random() < 0.4
        q_hi = _log(rng, 1, 40 if seqs <= 16 else 8)
        hi = _log(rng, 1, min(65536, max(8, 1_500_000 // (seqs * kv))))
        act = rng.choice(["bf16", "bf16", "f32"])
        return _drop(_attend("", seqs, rng.randint(1, q_hi), q_hi, rng.randint(0, hi), hi, heads, kv, act, rng.choice([act, "f8"]), tree=tree))
    if kind == "select":
        width = rng.randint(1, 8)
        return {"kind": kind, "streams": _log(rng, 1, 320 // width), "width": width, "vocab": _log(rng, 40, VOCAB),
                "src": rng.choice(["f32", "f32", "bf16"]), "ragged": rng.random() < 0.5, "done": rng.random() < 0.5}
    hi, width, layers = _log(rng, 1, CONTEXT), rng.randint(2, 8), rng.randint(1, 2)
    return {"kind": kind, "streams": _log(rng, 1, 320 // width), "width": width, "layers": layers, "positions": CONTEXT, "lo": rng.randint(0, hi), "hi": hi,
            "values": 2 * HEAD * rng.choice(HEADS)[1], "type": "bf16" if layers == 2 else rng.choice(["bf16", "f32"])}


def _drop(case):
    del case["name"]
    return case


# ---- inputs ------------------------------------------------------------------------------------------------------------

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f8": torch.float8_e4m3fn}


def _lengths(case):
    """Tokens of each sequence and rows nobody uses in front of it: a matter of the case, whatever the seed of its values."""
    rng = random.Random("%d %d %d" % (case["seqs"], case["lo"], case["hi"]))
    lens = [rng.randint(case["lo"], case["hi"]) for _ in range(case["seqs"])]
    lens[0] = max(lens[0], 1)
    return lens, [rng.randint(0, 3) for _ in lens]


def _queries(case):
    rng = random.Random("%d %d %d q" % (case["seqs"], case["q_lo"], case["q_hi"]))
    return [rng.randint(case["q_lo"], case["q_hi"]) for _ in range(case["seqs"])]


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _prefix(lens):
    return _ints([0] + [int(x) for x in np.cumsum(lens)]) if lens else _ints([0])


def _randn(gen, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16 if dtype == torch.bfloat16 else torch.float32)


def _factor(e):
    """2^e for whole e in [-127, 127], exactly."""
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).to(torch.int32).view(torch.float32)


def _quantise(x):
    """[.., 64] in 32 bits -> the e4m3 values and the biased exponents [..] of their common powers of two."""
    x = torch.where(torch.isfinite(x), x, math.nan)
    m, p = torch.frexp(torch.nan_to_num(x).abs().amax(-1))
    e = (p - 9 + (m > 0.875).to(torch.int32)).clamp(-127, 127)
    e = torch.where(m == 0, -127, e)
    return (x * _factor(-e)[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _cache(gen, rows, heads, kind):
    """A filled cache: rows of keys | values in the activation type, or for each head 64 keys | 64 values in 8 bits and exponents [2 heads, rows]."""
    x = _randn(gen, rows, 2 * heads * HEAD, dtype=TYPES[kind])
    if kind != "f8":
        return x, None
    q, e = _quantise(x.view(rows, heads, 2, HEAD))
    return q, e.view(rows, 2 * heads).t().contiguous()


def prepare(case, seed):
    rng = random.Random(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"case": case, **globals()["_prepare_" + case["kind"]](case, rng, gen)}


def _places(case):
    """Ragged pieces of a cache: tokens of each sequence, their prefix sums, the first row of each and the cache's rows."""
    lens, gaps = _lengths(case)
    ends = np.cumsum([n + g for n, g in zip(lens, gaps)])
    return lens, _prefix(lens), _ints([int(e) - n for e, n in zip(ends, lens)]), int(ends[-1]) + 1


def _prepare_write(case, rng, gen):
    lens, cu, rows, n_rows = _places(case)
    w = case["heads"] * HEAD
    qkv = _randn(gen, sum(lens), 3 * w, dtype=TYPES[case["src"]])        # keys and values lie behind the queries of the same product
    qkv[:, :w] *= 3.0
    if case["cache"] == "f8":
        data = torch.zeros((n_rows, case["heads"], 2, HEAD), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        exps = torch.zeros((2 * case["heads"], n_rows), dtype=torch.uint8, device="cuda")
    else:
        data, exps = torch.zeros((n_rows, 2 * w), dtype=TYPES[case["cache"]], device="cuda"), None
    return {"k": qkv[:, w:2 * w], "v": qkv[:, 2 * w:], "cu": cu, "rows": rows, "data": data, "exps": exps}


def _prepare_read(case, rng, gen):
    lens, cu, rows, n_rows = _places(case)
    data, exps = _cache(gen, n_rows, case["heads"], case["cache"])
    return {"data": data, "exps": exps, "cu": cu, "rows": rows, "tokens": sum(lens)}


def _prepare_attend(case, rng, gen):
    lens, _, rows, n_rows = _places(case)
    n_q = _queries(case)
    data, exps = _cache(gen, n_rows, case["kv_heads"], case["cache"])
    q = _randn(gen, sum(n_q), case["heads"] * HEAD, dtype=TYPES[case["act"]]) * 2.0
    mask = since = None
    if case["tree"]:        # the last keys of a sequence are its drafted tokens; a draft sees its ancestors and itself
        words = (case["q_hi"] + 31) // 32
        bits = np.zeros((sum(n_q), words), np.uint32)
        at = 0
        for n, length in zip(n_q, lens):
            seen = []
            for t in range(n):
                seen.append((seen[rng.randrange(max(0, t - 6), t)] if t else 0) | 1 << t)
                for w in range(words):
                    bits[at + t, w] = seen[t] >> 32 * w & 0xFFFFFFFF
            at += n
        mask = torch.from_numpy(bits.view(np.int32)).cuda()
        since = _ints([max(0, length - n) for n, length in zip(n_q, lens)])
    return {"data": data, "exps": exps, "q": q, "cu": _prefix(n_q), "rows": rows, "lens": _ints(lens), "max_q": case["q_hi"], "max_len": case["hi"],
            "mask": mask, "since": since}


def _prepare_select(case, rng, gen):
    B, W, V = case["streams"], case["width"], case["vocab"]
    logits = _randn(gen, B, W, V) * 2.5
    likely = torch.randint(V, (B, W, 12), generator=gen, device="cuda")       # a few likely words
    logits.scatter_(2, likely, 6.0 + 3.0 * _randn(gen, B, W, 12))
    logits[:, :, V - V // 33:] = -math.inf                                    # marks that are suppressed at this place
    scores = -(torch.rand((B, W), generator=gen, device="cuda") * 6.0).cumsum(1) - 5.0
    st = {"logits": logits.to(TYPES[case["src"]]), "scores": scores, "n_in": None, "n_out": None, "done": None, "eos": V // 2}
    if case["ragged"]:      # pruned streams run with one beam, others widen again
        st["n_in"] = _ints([rng.choice([1, 1, W]) for _ in range(B)])
        st["n_out"] = _ints([rng.choice([1, W, W]) for _ in range(B)])
    if case["done"]:
        st["done"] = torch.rand((B, W), generator=gen, device="cuda") < 0.25
    return st


def _prepare_reorder(case, rng, gen):
    B, W = case["streams"], case["width"]
    state = _randn(gen, case["layers"], B * W, case["positions"], case["values"], dtype=TYPES[case["type"]])
    parents = []
    for _ in range(B):      # surviving beams stay where they are, the others' slots take over a survivor's
        alive = sorted(rng.sample(range(W), rng.randint(1, W)))
        parents.append([j if j in alive else rng.choice(alive) for j in range(W)])
    return {"state": state, "parents": _ints(parents), "lens": _ints([rng.randint(case["lo"], case["hi"]) for _ in range(B)])}


# ---- one pass ----------------------------------------------------------------------------------------------------------

def run(state):
    return globals()[("_own_" if own else "_plain_") + state["case"]["kind"]](state)


def _sequence_of(cu, n):
    """The sequence of each of n packed tokens and the token's place in it."""
    t = torch.arange(n, device="cuda", dtype=torch.int32)
    s = torch.searchsorted(cu, t, right=True) - 1
    return s, t - cu[s]


def _rows_of(st, n):
    s, at = _sequence_of(st["cu"], n)
    return (st["rows"][s] + at).long()


def _values(data, exps):
    """The cache in 32 bits: [rows, heads, 2, 64]."""
    if exps is None:
        return data.float().view(data.shape[0], 2, -1, HEAD).transpose(1, 2)
    return data.float() * _factor(exps.t().to(torch.int32) - 127).view(*data.shape[:3], 1)


def _plain_write(st):
    T = st["k"].shape[0]
    rows = _rows_of(st, T)
    kv = torch.stack([st["k"].reshape(T, -1, HEAD), st["v"].reshape(T, -1, HEAD)], 2).float()      # [T, heads, 2, 64]
    if st["exps"] is None:
        st["data"][rows] = kv.transpose(1, 2).reshape(T, -1).to(st["data"].dtype)
        return [st["data"]]
    q, e = _quantise(kv)
    st["data"].view(torch.uint8)[rows] = q.view(torch.uint8)
    st["exps"][:, rows] = e.reshape(T, -1).t()
    return [st["data"], st["exps"]]


def _plain_read(st):
    rows = _rows_of(st, st["tokens"])
    x = _values(st["data"][rows] if st["exps"] is None else st["data"].view(torch.uint8)[rows].view(torch.float8_e4m3fn),
                None if st["exps"] is None else st["exps"][:, rows])
    return x.transpose(1, 2).reshape(st["tokens"], -1).to(TYPES[st["case"]["out"]])


def _plain_attend(st):
    heads, kv = st["case"]["heads"], st["case"]["kv_heads"]
    B, L, Q, R = st["lens"].shape[0], st["max_len"], st["max_q"], st["q"].shape[0]
    key = torch.arange(L, device="cuda", dtype=torch.int32)
    here = key < st["lens"][:, None]                                                               # [B, L]
    rows = torch.where(here, st["rows"][:, None] + key, 0).long()
    x = _values(st["data"][rows.view(-1)] if st["exps"] is None else st["data"].view(torch.uint8)[rows.view(-1)].view(torch.float8_e4m3fn),
                None if st["exps"] is None else st["exps"][:, rows.view(-1)]).view(B, L, kv, 2, HEAD)
    K, V = x[:, :, :, 0].permute(0, 2, 3, 1).contiguous(), x[:, :, :, 1].transpose(1, 2).contiguous()    # [B, kv, 64, L], [B, kv, L, 64]
    row = (st["cu"][:-1, None] + torch.arange(Q, device="cuda", dtype=torch.int32)).clamp(max=R - 1).long()      # [B, Q]
    q = st["q"][row].float().view(B, Q, kv, heads // kv, HEAD).permute(0, 2, 1, 3, 4).reshape(B, kv, -1, HEAD)
    seen = here[:, None]                                                                           # [B, 1 or Q, L]
    if st["mask"] is not None:
        at = key - st["since"][:, None]                                                            # [B, L]
        word = st["mask"][row].gather(2, (at >> 5).clamp(0, st["mask"].shape[1] - 1).long()[:, None].expand(B, Q, L))
        bit = ((word >> (at & 31)[:, None]) & 1).bool() & (at < 32 * st["mask"].shape[1])[:, None]
        seen = seen & (bit | (at < 0)[:, None])
    s = torch.matmul(q, K).view(B, kv, Q, heads // kv, L) * HEAD ** -0.5
    s = torch.where(seen[:, None, :, None], s, -math.inf)
    w = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-3e38))
    total = w.sum(-1, keepdim=True)
    o = torch.matmul(w.view(B, kv, -1, L), V).view(B, kv, Q, heads // kv, HEAD)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 2, 1, 3, 4).reshape(B, Q, heads * HEAD)
    seq, at = _sequence_of(st["cu"], R)
    return o[seq, at.long()].to(TYPES[st["case"]["act"]])


def _plain_select(st):
    B, W, V = st["logits"].shape
    beam = torch.arange(W, device="cuda")
    x = st["logits"].float()
    x = torch.where(torch.isfinite(x), x, -math.inf)
    top = x.amax(-1, keepdim=True)
    lse = top.double() + torch.exp(x - top.clamp(min=-3e38)).sum(-1, keepdim=True, dtype=torch.float64).log()
    if st["done"] is not None:          # a finished beam goes on as it is
        x = torch.where(st["done"][:, :, None], torch.where(torch.arange(V, device="cuda") == st["eos"], 0.0, -math.inf), x)
        lse = torch.where(st["done"][:, :, None], 0.0, lse)
    # a row's best: by value, then the lowest token (unique keys of 64 bits, so that their order is one)
    bits = (x + 0.0).view(torch.int32).long()
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
    keys = order * 2 ** 32 + (2 ** 32 - 1 - torch.arange(V, device="cuda"))
    token = 2 ** 32 - 1 - (keys.topk(min(W, V), dim=-1).values & 0xFFFFFFFF)
    best = x.gather(2, token)
    total = torch.where(best > -math.inf, st["scores"].double()[:, :, None] + (best.double() - lse), -math.inf)
    if st["n_in"] is not None:
        total = torch.where((beam < st["n_in"][:, None])[:, :, None], total, -math.inf)
    # a stream's best: by total, then the lowest beam
    score, at = total.view(B, -1).sort(dim=1, descending=True, stable=True)
    score, at = score[:, :W], at[:, :W]
    if at.shape[1] < W:
        score = torch.nn.functional.pad(score, (0, W - at.shape[1]), value=-math.inf)
        at = torch.nn.functional.pad(at, (0, W - at.shape[1]))
    good = score > -math.inf
    if st["n_out"] is not None:
        good = good & (beam < st["n_out"][:, None])
    parent, token = at // token.shape[2], token.reshape(B, -1).gather(1, at)
    out = [torch.where(good, token, -1).int(), torch.where(good, parent, -1).int(), torch.where(good, score, -math.inf).float()]
    if st["done"] is not None:
        out.append(good & (st["done"].gather(1, parent) | (token == st["eos"])))
    return out


def _plain_reorder(st):
    state, (B, W) = st["state"], st["parents"].shape
    parent = (torch.arange(B, device="cuda", dtype=torch.int32)[:, None] * W + st["parents"]).view(-1)
    used = torch.arange(state.shape[2], device="cuda") < st["lens"].repeat_interleave(W, output_size=B * W)[:, None]
    state.copy_(torch.where(used[None, :, :, None], state[:, parent.long()], state))
    return state


_binding = None


def _wf():
    global _binding
    if _binding is None:
        from paper_2412_11272_amd import binding
        _binding = binding
    return _binding


def _own_write(st):
    wf = _wf()
    wf.op_cache_write(wf.Cache(st["data"], st["exps"]), st["k"], st["v"], st["cu"], st["rows"])
    return [st["data"]] if st["exps"] is None else [st["data"], st["exps"]]


def _own_read(st):
    wf = _wf()
    return wf.op_cache_read(wf.Cache(st["data"], st["exps"]), st["cu"], st["rows"], st["tokens"], out_dtype=TYPES[st["case"]["out"]])


def _own_attend(st):
    wf = _wf()
    return wf.op_cache_attention(wf.Cache(st["data"], st["exps"]), st["q"], st["cu"], st["rows"], st["lens"], st["max_q"], st["max_len"],
                                 mask=st["mask"], mask_from=st["since"])


def _own_select(st):
    out = _wf().op_beam_select(st["logits"], st["scores"], n_in=st["n_in"], n_out=st["n_out"], done=st["done"], eos=st["eos"])
    return list(out if st["done"] is not None else out[:3])


def _own_reorder(st):
    return _wf().op_beam_reorder(st["state"], st["parents"], lens=st["lens"])


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------

BYTES = {"f32": 4, "bf16": 2}


def _row_bytes(heads, kind):
    return heads * (2 * HEAD + 2) if kind == "f8" else heads * 2 * HEAD * BYTES[kind]


def work(case):
    kind = case["kind"]
    if kind in ("write", "read"):
        plain = case["heads"] * 2 * HEAD * BYTES[case["src" if kind == "write" else "out"]]
        return {"bytes": sum(_lengths(case)[0]) * (plain + _row_bytes(case["heads"], case["cache"])), "flops": 0}
    if kind == "attend":
        lens, n_q = _lengths(case)[0], _queries(case)
        return {"bytes": sum(lens) * _row_bytes(case["kv_heads"], case["cache"]) + sum(n_q) * 2 * case["heads"] * HEAD * BYTES[case["act"]],
                "flops": 4.0 * HEAD * case["heads"] * sum(n * q for n, q in zip(lens, n_q))}
    if kind == "select":        # on average: ragged streams have one beam two times in three, a quarter of the beams is done
        rows = case["streams"] * ((case["width"] + 2) / 3 if case["ragged"] else case["width"]) * (0.75 if case["done"] else 1.0)
        return {"bytes": rows * case["vocab"] * BYTES[case["src"]], "flops": 3.0 * rows * case["vocab"]}
    W, mean = case["width"], (case["lo"] + case["hi"]) / 2      # on average (W - 1) / 2 slots of a stream take over another's
    return {"bytes": case["layers"] * case["streams"] * (W - 1) * mean * case["values"] * BYTES[case["type"]], "flops": 0}


# ---- the operators' definitions in 64 bits -----------------------------------------------------------------------------------

def _two(e):
    """2^e in 64 bits for whole e, exactly (the power function need not be)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "reorder":                      # values are moved, none is computed
        return None
    if kind == "select":
        return _exact_select(st)
    cu, rows = st["cu"].tolist(), st["rows"].tolist()
    pieces = [(s, cu[s], cu[s + 1], rows[s]) for s in range(len(rows))]
    if kind == "write":
        k, v = (t.double().view(t.shape[0], case["heads"], HEAD) for t in (st["k"].contiguous(), st["v"].contiguous()))
        if case["cache"] != "f8":
            data = st["data"].double()
            for _, a, b, row in pieces:
                data[row:row + b - a] = torch.cat([k[a:b].flatten(1), v[a:b].flatten(1)], 1)
            return [data]
        data = torch.zeros(st["data"].shape, dtype=torch.float64, device="cuda")
        for _, a, b, row in pieces:
            for i, x in enumerate((k[a:b], v[a:b])):
                largest = x.abs().amax(-1, keepdim=True)
                e = torch.ceil(torch.log2(largest / 448))
                e = torch.where(largest > 448 * _two(e), e + 1, torch.where(largest <= 224 * _two(e), e - 1, e))
                y = x / _two(e)
                step = _two(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
                data[row:row + b - a, :, i] = torch.round(y / step) * step
        return [data, None]
    if kind == "read":
        return torch.cat([_exact_rows(st, row, b - a, case["heads"], case["cache"]).transpose(1, 2).flatten(1) for _, a, b, row in pieces])
    out = torch.zeros((st["q"].shape[0], case["heads"], HEAD), dtype=torch.float64, device="cuda")
    since = st["since"].tolist() if st["since"] is not None else None
    lens, group = st["lens"].tolist(), case["heads"] // case["kv_heads"]
    for s, a, b, row in pieces:
        kv = _exact_rows(st, row, lens[s], case["kv_heads"], case["cache"])
        q = st["q"][a:b].double().view(b - a, case["heads"], HEAD)
        hidden = None
        if since is not None:
            place = torch.arange(lens[s], device="cuda") - since[s]
            word = torch.cat([st["mask"][a:b].long() & 0xFFFFFFFF, torch.zeros((b - a, 1), dtype=torch.int64, device="cuda")], 1)
            hidden = ((word[:, (place.clamp(min=0) // 32).clamp(max=word.shape[1] - 1)] >> (place.clamp(min=0) % 32)) & 1 == 0) & (place >= 0)
        for h in range(case["heads"]):
            logit = q[:, h] @ kv[:, h // group, 0].t().contiguous() / math.sqrt(HEAD)
            if hidden is not None:
                logit = logit.masked_fill(hidden, -math.inf)
            weight = torch.softmax(logit, -1).nan_to_num(0.0)
            out[a:b, h] = weight @ kv[:, h // group, 1].contiguous()
    return out.flatten(1)


def _exact_rows(st, row, n, heads, kind):
    """[n, heads, 2, 64]"""
    if kind != "f8":
        return st["data"][row:row + n].double().view(n, 2, heads, HEAD).transpose(1, 2)
    e = st["exps"][:, row:row + n].t().double().view(n, heads, 2, 1) - 127
    return st["data"].view(torch.uint8)[row:row + n].view(torch.float8_e4m3fn).double() * _two(e)


def _exact_select(st):
    B, W, V = st["logits"].shape
    scores = torch.full((B, W), -math.inf, dtype=torch.float64)
    count = lambda name, s: W if st[name] is None else int(st[name][s])  # noqa: E731
    for s in range(B):
        found = []
        for b in range(count("n_in", s)):
            if st["done"] is not None and bool(st["done"][s, b]):
                found.append(st["scores"][s, b:b + 1].double())
                continue
            x = st["logits"][s, b].double()
            found.append(st["scores"][s, b].double() + torch.log_softmax(x[torch.isfinite(x)], 0))
        best = torch.cat(found).sort(descending=True).values[:count("n_out", s)]
        scores[s, :best.shape[0]] = best.cpu()
    return [None, None, scores] + ([None] if st["done"] is not None else [])
