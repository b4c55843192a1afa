"""Key / value caches on the GPU: writing (as they come and in 8 bits), reading back, and attention of a few queries per sequence, against the
64-bit definitions of oracle/decode_oracle.py."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle as D
from paper_2412_11272_amd import binding as wf

pytestmark = pytest.mark.gpu

F8, BF, F32 = torch.float8_e4m3fn, torch.bfloat16, torch.float32
U = 2.0 ** -24          # half a step of fp32


def _i32(x):
    return torch.tensor(np.asarray(x, np.int32), device="cuda")


def _np(t):
    return t.detach().double().cpu().numpy()


def _poison(cache):
    """Every byte of a cache as no call leaves it: NaN values, exponents of 2^127."""
    if cache.exps is None:
        cache.data.fill_(float("nan"))
    else:
        cache.data.view(torch.uint8).fill_(0x7f)
        cache.exps.fill_(254)
    return cache


def _sources(T, H, dtype, seed, ld_extra=0):
    """k and v as views behind the queries of one product, row stride 3 * 64 H + ld_extra."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, 3 * 64 * H + ld_extra), generator=g) * torch.exp2(torch.randint(-20, 20, (T, 1), generator=g).float())
    x = x.to(dtype).cuda()
    return x[:, 64 * H:128 * H], x[:, 128 * H:192 * H]


LAYOUTS = {
    # lens, first rows, cache rows, tokens of the buffers (those behind the last sequence belong to none)
    "one-token": ([1], [0], 1, 1),
    "ragged": ([5, 0, 1, 130, 64, 0], [7, 0, 3, 400, 20, 9], 600, 200),
    "padded": ([3, 2], [10, 0], 20, 9),
    "outside": ([4, 4, 4], [-2, 18, 30], 20, 12),           # rows before, across and behind the cache's end are left out
    "many": ([1 + i % 3 for i in range(1500)], [3 * i for i in range(1500)], 4500, 2999),
    "long": ([3001, 7], [11, 4000], 4100, 3010),
}


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("src", [BF, F32], ids=str)
@pytest.mark.parametrize("dtype", [F8, BF, F32], ids=str)
def test_write_then_read(dtype, src, layout):
    lens, first, n_rows, T = LAYOUTS[layout]
    H = 1 if layout in ("many", "long") else 3 if layout == "ragged" else 20
    cu = np.concatenate([[0], np.cumsum(lens)])
    k, v = _sources(T, H, src, 3, ld_extra=8)
    cache = _poison(wf.Cache.empty(n_rows, H, dtype))
    wf.op_cache_write(cache, k, v, _i32(cu), _i32(first))
    place = D.cache_rows(cu, first, n_rows, T)
    x = np.stack([_np(k).reshape(T, H, 64), _np(v).reshape(T, H, 64)], 2)         # [T, H, 2, 64]
    want = _poison(wf.Cache.empty(n_rows, H, dtype))
    for t in np.flatnonzero(place >= 0):
        if dtype == F8:
            q, e = D.quantise(x[t])
            want.data[int(place[t])] = torch.from_numpy(q).cuda().to(F32).to(F8)
            want.exps[:, int(place[t])] = torch.from_numpy(e.reshape(-1).astype(np.uint8)).cuda()
        else:
            want.data[int(place[t])] = torch.from_numpy(x[t].transpose(1, 0, 2).reshape(-1)).cuda().to(dtype)
        if T > 500 and t > 300 and t < T - 300:
            break                                                                   # the rest by the read below
    upto = place[:t + 1] if T > 500 else place
    done = torch.from_numpy(np.unique(upto[upto >= 0])).cuda()
    assert torch.equal(cache.data.view(torch.uint8).view(n_rows, -1)[done], want.data.view(torch.uint8).view(n_rows, -1)[done])
    untouched = torch.from_numpy(np.setdiff1d(np.arange(n_rows), place)).cuda()
    assert torch.equal(cache.data.view(torch.uint8).view(n_rows, -1)[untouched], want.data.view(torch.uint8).view(n_rows, -1)[untouched])
    if dtype == F8:
        assert torch.equal(cache.exps[:, done], want.exps[:, done]) and torch.equal(cache.exps[:, untouched], want.exps[:, untouched])
    for out_dtype in (F32, BF):
        out = torch.full((T, 128 * H), 7.0, device="cuda", dtype=out_dtype)
        wf.op_cache_read(cache, _i32(cu), _i32(first), T, out=out)
        got = _np(out).reshape(T, 2, H, 64).transpose(0, 2, 1, 3)
        assert (got[place == -2] == 7.0).all() and (got[place == -1] == 0.0).all()
        live = place >= 0
        if dtype == F8:       # every value within half a step of the quantisation, and exact in both output types
            scale = np.abs(x[live]).max(-1, keepdims=True)
            step = np.maximum(np.abs(x[live]) * 2.0 ** -4, scale * 2.0 ** -17)     # largest in (224, 448]: the subnormals' half step is 2^-10 of 2^8
            assert (np.abs(got[live] - x[live]) <= step).all()
        else:
            half = 2.0 ** -8 if BF in (dtype, out_dtype) else 0.0                   # twice bf16 rounds once
            assert (np.abs(got[live] - x[live]) <= half * np.abs(x[live])).all()


def test_quantisation_of_special_values():
    H = 2
    x = torch.zeros((6, 128))
    x[0, :64] = torch.linspace(-3.4e38, 3.4e38, 64)                # the largest exponents
    x[1, :64] = 2.0 ** -149 * torch.arange(64)                     # fp32 subnormals: below the smallest factor
    x[2, :3] = torch.tensor([float("nan"), float("inf"), -float("inf")]); x[2, 3:64] = torch.linspace(-5, 5, 61)
    x[3, :64] = float("inf")
    x[4, :64] = torch.linspace(447.9, 448.1, 64)                   # the border between two exponents
    x[5, :64] = 448 * 2.0 ** -20 * torch.linspace(-1, 1, 64)
    x[:, 64:] = -0.0
    cache = wf.Cache.empty(6, H, F8)
    xd = x.cuda()
    wf.op_cache_write(cache, xd, xd, _i32([0, 6]), _i32([0]))
    q, e = D.quantise(x.numpy().reshape(6, 2, 64))
    got = _np(cache.data.float()).reshape(6, 2, 2, 64)
    for kv in range(2):
        np.testing.assert_array_equal(got[:, :, kv], q)
        assert (cache.exps.cpu().numpy().reshape(H, 2, 6)[:, kv].T == e).all()
    back = wf.op_cache_read(cache, _i32([0, 6]), _i32([0]), 6, out_dtype=F32)
    want = (q * 2.0 ** (e[..., None] - 127.0)).reshape(6, 128)
    with np.errstate(over="ignore"):
        np.testing.assert_array_equal(_np(back)[:, :128], want.astype(np.float32).astype(np.float64))


# ---- attention ------------------------------------------------------------------------------------------------------------

def _filled(n_rows, H, cdtype, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n_rows, 128 * H), generator=g) * spread
    cache = wf.Cache.empty(n_rows, H, cdtype)
    xd = x.cuda().to(BF if cdtype == BF else F32)
    wf.op_cache_write(cache, xd[:, :64 * H], xd[:, 64 * H:], _i32([0, n_rows]), _i32([0]))
    return cache


def _contents(cache):
    """[n_rows, heads, 2, 64] in 64 bits."""
    if cache.exps is None:
        return _np(cache.data).reshape(cache.n_rows, 2, cache.n_heads, 64).transpose(0, 2, 1, 3)
    e = cache.exps.cpu().numpy().astype(np.float64).T.reshape(cache.n_rows, cache.n_heads, 2, 1)
    return _np(cache.data.float()) * 2.0 ** (e - 127)


def _tolerance(act, n, ref, size, dots):
    # A logit is off by 72 half steps of its 64 products' sum (its additions, the scale and the difference), a weight by twice that, by its
    # exponential's 2^-21 and, next to a bf16 operand, by the 2^-16 that two bf16 parts leave; sums of n terms by n half steps, numerator and
    # denominator; the result by its last rounding.
    tol = (2 * 72 * U * dots + 2.0 ** -21 + (2.0 ** -16 if act == BF else 0.0) + (2 * n + 64) * U) * size
    return tol * (1 + 2.0 ** -7) + (2.0 ** -8 if act == BF else U) * np.abs(ref) + 1e-37


def _check_attention(cache, q, cu, rows, lens, max_q, max_len, mask=None, since=None, scale=0.125, call=None, heads=None, some_rows=None):
    """The call's output against the definition; untouched rows must keep the marker.  Returns the output."""
    T, Hq = q.shape[0], q.shape[1] // 64
    out = torch.full((T, q.shape[1]), 77.0, device="cuda", dtype=q.dtype)
    (call or wf.op_cache_attention)(cache, q, _i32(cu), _i32(rows), _i32(lens), max_q, max_len, scale=scale, mask=mask,
                                    mask_from=None if since is None else _i32(since), out=out)
    torch.cuda.synchronize()
    got, qn, kv = _np(out).reshape(T, Hq, 64), _np(q).reshape(T, Hq, 64), _contents(cache)
    words = None if mask is None else mask.cpu().numpy().view(np.uint32)
    touched = np.zeros(T, bool)
    worst = 0.0
    for s in range(len(rows)):
        n = min(lens[s], max_len, cache.n_rows - rows[s]) if rows[s] >= 0 else 0
        n = max(n, 0)
        for r in range(cu[s], min(cu[s + 1], cu[s] + max_q, T)):
            touched[r] = True
            if some_rows is not None and r not in some_rows:
                continue
            seen = D.visible(n, None if words is None else words[r], 0 if since is None else since[s])
            for h in (range(Hq) if heads is None else heads):
                hk = h // (Hq // cache.n_heads)
                block = kv[rows[s]:rows[s] + n, hk] if n else np.zeros((0, 2, 64))
                ref, size, dots = D.attention(qn[r, h], block[:, 0], block[:, 1], scale, seen)
                tol = _tolerance(q.dtype, n, ref, size, dots)
                err = np.abs(got[r, h] - ref)
                worst = max(worst, float((err / tol).max()))
                assert (err <= tol).all(), (s, r, h, float((err / tol).max()))
    assert (got[~touched] == 77.0).all()
    print(f"worst error / tolerance {worst:.3f}", flush=True)
    return out


KINDS = [pytest.param(BF, BF, id="bf16"), pytest.param(BF, F8, id="bf16-f8"), pytest.param(F32, F32, id="f32"), pytest.param(F32, F8, id="f32-f8")]


def _q(T, Hq, dtype, seed, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((T, 64 * Hq), generator=g) * spread).to(dtype).cuda()


@pytest.mark.parametrize("heads", [(1, 1), (6, 6), (8, 2)], ids=str)
@pytest.mark.parametrize("act,cdtype", KINDS)
def test_attention_of_ragged_sequences(act, cdtype, heads):
    Hq, H = heads
    lens = [1, 0, 31, 32, 33, 64, 65, 127, 200, 15, 16, 17, 257]
    n_q = [1, 2, 1, 3, 0, 1, 5, 1, 2, 17, 1, 1, 4]
    rows, at = [], 2
    for n in lens:
        rows.append(at)
        at += n + 1
    cu = np.concatenate([[0], np.cumsum(n_q)])
    cache = _filled(at + 3, H, cdtype, 5)
    _check_attention(cache, _q(int(cu[-1]) + 3, Hq, act, 6), cu, rows, lens, max(n_q), max(lens))


@pytest.mark.parametrize("n_keys", [1500, 1501, 5003])
@pytest.mark.parametrize("act,cdtype", KINDS)
def test_attention_over_long_sequences(act, cdtype, n_keys):
    cache = _filled(n_keys + 9, 2, cdtype, 7)
    _check_attention(cache, _q(3, 4, act, 8), [0, 1, 3], [4, 0], [n_keys, n_keys - 700], 2, n_keys)


@pytest.mark.parametrize("n_q", [16, 17, 33, 64, 65, 130])
@pytest.mark.parametrize("act,cdtype", KINDS)
def test_attention_of_many_queries(act, cdtype, n_q):
    cache = _filled(150, 1, cdtype, 9)
    _check_attention(cache, _q(n_q + 2, 2, act, 10), [0, 2, n_q + 2], [0, 10], [99, 140], n_q, 140)


@pytest.mark.parametrize("act,cdtype", KINDS)
def test_attention_with_sharp_weights(act, cdtype):
    # logits of several hundred: the running maximum moves often and one key takes nearly all of the weight
    cache = _filled(700, 2, cdtype, 11, spread=6.0)
    _check_attention(cache, _q(5, 2, act, 12, spread=30.0), [0, 5], [0], [700], 5, 700)


@pytest.mark.parametrize("act,cdtype", KINDS)
def test_attention_under_a_mask(act, cdtype):
    rng = np.random.default_rng(13)
    lens, n_q = [300, 40, 33, 5, 64], [9, 40, 2, 3, 1]
    since = [259, 0, 0, 9, 31]                # bits behind a common prefix, from the first key on, past the last key
    cu = np.concatenate([[0], np.cumsum(n_q)])
    words = rng.integers(0, 1 << 32, (cu[-1], 2), dtype=np.uint32) & rng.integers(0, 1 << 32, (cu[-1], 2), dtype=np.uint32)
    words[cu[1]:cu[1] + 3] = 0                # rows that see nothing
    words[cu[2]] = [0, 1]                     # the one key behind a word's border
    words[cu[4]] = [1 << 31, 0]
    rows = np.concatenate([[0], np.cumsum(lens)[:-1]])
    cache = _filled(sum(lens), 2, cdtype, 14)
    mask = torch.from_numpy(words.view(np.int32)).cuda()
    out = _check_attention(cache, _q(int(cu[-1]), 4, act, 15), cu, rows, lens, 40, 300, mask=mask, since=since)
    assert (out[cu[1]:cu[1] + 3] == 0).all()
    _check_attention(cache, _q(int(cu[-1]), 4, act, 15), cu, rows, lens, 40, 300, mask=mask)          # no mask_from: bits from key 0, none behind 64


@pytest.mark.parametrize("act,cdtype", KINDS)
def test_what_a_row_does_not_see_does_not_reach_it(act, cdtype):
    # NaN and infinities in rows between the sequences, behind their ends and under the mask; a key that is seen and not finite shows
    lens, n_q = [70, 35], [4, 18]
    rows, cu = [3, 90], [0, 4, 22]
    cache = _filled(140, 2, cdtype, 16)
    mask = np.zeros((22, 3), np.uint32)
    mask[:, 0] = 0x55555555
    mask[:, 1] = 0x55555555
    mask[3, 0] |= 1 << 7                       # the last row of the first sequence sees key 7, the others do not
    if cdtype == F8:
        bad = torch.full((1, 2, 2, 64), 0x7f, dtype=torch.uint8, device="cuda").view(F8)
        put = lambda r: cache.data.view(torch.uint8).__setitem__(slice(r, r + 1), bad.view(torch.uint8))  # noqa: E731
    else:
        row = torch.full((1, cache.data.shape[1]), float("nan"), device="cuda", dtype=cdtype)
        row[:, ::3] = float("inf")
        row[:, 1::3] = -float("inf")
        put = lambda r: cache.data.__setitem__(slice(r, r + 1), row)  # noqa: E731
    clean = _contents(cache)
    for r in [0, 2, 73, 74, 89, 125, 139]:
        put(r)
    put(rows[0] + 7)
    put(rows[1] + 9)
    q = _q(22, 4, act, 17)
    m = torch.from_numpy(mask.view(np.int32)).cuda()
    out = torch.empty_like(q)
    wf.op_cache_attention(cache, q, _i32(cu), _i32(rows), _i32(lens), 18, 70, mask=m, out=out)
    got = _np(out).reshape(22, 4, 64)
    assert not np.isfinite(got[3]).any()
    qn = _np(q).reshape(22, 4, 64)
    for r in [0, 1, 2, 4, 5, 21]:
        s = 0 if r < 4 else 1
        seen = D.visible(lens[s], mask[r], 0)
        for h in range(4):
            ref, size, dots = D.attention(qn[r, h], clean[rows[s]:rows[s] + lens[s], h // 2, 0], clean[rows[s]:rows[s] + lens[s], h // 2, 1], 0.125, seen)
            assert (np.abs(got[r, h] - ref) <= _tolerance(act, lens[s], ref, size, dots)).all(), (r, h)


@pytest.mark.parametrize("n_q", [1, 5, 20, 40])
@pytest.mark.parametrize("act,cdtype", KINDS)
def test_long_masked_sequences_split_over_workgroups(act, cdtype, n_q):
    # the tail is masked, a hidden key of it is NaN, and one row sees nothing behind the common prefix; the prefix of the second sequence is empty
    lens, since = [4001, 2500], [3910, 0]
    rows, cu = [5, 4100], [0, n_q, 2 * n_q]
    cache = _filled(6700, 1, cdtype, 48)
    clean = _contents(cache)
    rng = np.random.default_rng(49)
    words = rng.integers(0, 1 << 32, (2 * n_q, 80), dtype=np.uint32)
    words[:, 0] &= ~np.uint32(1 << 9)
    words[0, :3] = 0
    words[n_q] = 0                            # sees nothing at all
    hidden = [rows[0] + since[0] + 9, rows[1] + 9]
    for r in hidden:
        if cdtype == F8:
            cache.data.view(torch.uint8)[r] = 0x7f
        else:
            cache.data[r] = float("nan")
    q, mask = _q(2 * n_q, 2, act, 50), torch.from_numpy(words.view(np.int32)).cuda()
    got = _np(wf.op_cache_attention(cache, q, _i32(cu), _i32(rows), _i32(lens), n_q, 4100, mask=mask, mask_from=_i32(since))).reshape(2 * n_q, 2, 64)
    assert np.isfinite(got).all() and not got[n_q].any()
    qn = _np(q).reshape(2 * n_q, 2, 64)
    for r in sorted({0, n_q - 1, n_q, 2 * n_q - 1}):
        s = int(r >= n_q)
        seen = D.visible(lens[s], words[r], since[s])
        for h in range(2):
            kv = clean[rows[s]:rows[s] + lens[s], 0]
            ref, size, dots = D.attention(qn[r, h], kv[:, 0], kv[:, 1], 0.125, seen)
            assert (np.abs(got[r, h] - ref) <= _tolerance(act, lens[s], ref, size, dots)).all(), (r, h)


def test_values_that_are_not_finite_reach_only_their_place():
    # a value of infinity in one place of a key that all rows see: that place alone is infinite
    cache = _filled(50, 1, BF, 18)
    cache.data[20, 64 + 5] = float("inf")
    q = _q(3, 1, BF, 19)
    for mask in (None, torch.full((3, 2), -1, dtype=torch.int32, device="cuda")):
        out = wf.op_cache_attention(cache, q, _i32([0, 3]), _i32([0]), _i32([50]), 3, 50, mask=mask)
        assert (out[:, 5] == float("inf")).all() and torch.isfinite(out).sum() == 3 * 63


@pytest.mark.parametrize("act,cdtype", KINDS)
def test_lengths_and_rows_outside_their_bounds(act, cdtype):
    cache = _filled(64, 1, cdtype, 20)
    # longer than max_len, across the cache's end, before its start, behind it, a negative length
    rows, lens = [0, 60, -1, 64, 10], [50, 30, 10, 5, -3]
    out = _check_attention(cache, _q(8, 1, act, 21), [0, 1, 2, 3, 4, 5], rows, lens, 1, 40)
    assert (out[2:5] == 0).all() and (out[5:] == 77).all()
    # more queries than max_q, and prefix sums that leave the buffer
    _check_attention(cache, _q(8, 1, act, 21), [0, 6, 20], [0, 3], [20, 30], 3, 40)


@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
@pytest.mark.parametrize("act,cdtype", KINDS)
def test_attention_scales_of_any_sign(act, cdtype, scale):
    cache = _filled(90, 1, cdtype, 40)
    q = _q(20, 2, act, 41, spread=1.0)
    mask = torch.from_numpy(np.random.default_rng(42).integers(0, 1 << 32, (20, 3), dtype=np.uint32).view(np.int32)).cuda()
    _check_attention(cache, q, [0, 3, 20], [0, 7], [45, 77], 17, 80, scale=scale)
    _check_attention(cache, q, [0, 3, 20], [0, 7], [45, 77], 17, 80, scale=scale, mask=mask)


@pytest.mark.parametrize("n_seqs", [1, 300])
def test_attention_over_nothing(n_seqs):
    cache = _filled(64, 8, BF, 43)
    q = _q(n_seqs, 8, BF, 44)
    out = wf.op_cache_attention(cache, q, _i32(range(n_seqs + 1)), _i32([0] * n_seqs), _i32([9] * n_seqs), 1, 0)
    assert not out.any()
    assert wf.op_cache_attention(cache, q[:0], _i32([0, 0]), _i32([0]), _i32([5]), 1, 5).shape == (0, 512)


@pytest.mark.parametrize("length", [5, 64, 65, 256, 257])
@pytest.mark.parametrize("act,cdtype", KINDS)
def test_attention_of_many_short_sequences(act, cdtype, length):
    # enough sequences that a workgroup has one, two or four waves by the longest one
    B, H = 160, 8
    lens = [(length * (i % 7)) // 6 for i in range(B)]
    rows = [(i * 37) % 900 for i in range(B)]
    cache = _filled(1200, H, cdtype, 45)
    cu = list(range(B + 1))
    some = {0, 1, 6, 40, 101, 159}
    _check_attention(cache, _q(B, H, act, 46), cu, rows, lens, 1, length, heads=[0, 7], some_rows=some)
    words = np.random.default_rng(47).integers(0, 1 << 32, (B, 3), dtype=np.uint32)
    _check_attention(cache, _q(B, H, act, 46), cu, rows, lens, 1, length, heads=[0, 7], some_rows=some, mask=torch.from_numpy(words.view(np.int32)).cuda(),
                     since=[max(0, n - 70) for n in lens])


def test_attention_strides_and_shapes():
    cache = _filled(100, 2, BF, 22)
    wide = _q(6, 6, BF, 23)
    q = wide[:, 128:384].contiguous()
    ref = wf.op_cache_attention(cache, q, _i32([0, 6]), _i32([0]), _i32([100]), 6, 100)
    out = torch.zeros((6, 512), device="cuda", dtype=BF)
    wf.op_cache_attention(cache, wide[:, 128:384], _i32([0, 6]), _i32([0]), _i32([100]), 6, 100, out=out[:, 64:320])
    assert torch.equal(out[:, 64:320], ref) and not out[:, :64].any() and not out[:, 320:].any()
    q3 = q.view(6, 4, 64)
    assert torch.equal(wf.op_cache_attention(cache, q3, _i32([0, 6]), _i32([0]), _i32([100]), 6, 100), ref.view(6, 4, 64))
    with pytest.raises(ValueError):
        wf.op_cache_attention(cache, q.t(), _i32([0, 6]), _i32([0]), _i32([100]), 6, 100)
    with pytest.raises(ValueError):
        wf.op_cache_attention(cache, q, _i32([0, 6, 7]), _i32([0]), _i32([100]), 6, 100)
    with pytest.raises(TypeError):
        wf.op_cache_attention(cache, q, _i32([0, 6]).long(), _i32([0]), _i32([100]), 6, 100)
    with pytest.raises(wf.WfError) as e:
        wf.op_cache_attention(cache, q.float(), _i32([0, 6]), _i32([0]), _i32([100]), 6, 100)
    assert e.value.code == wf.WF_E_INVALID_ARG


@pytest.mark.parametrize("act,cdtype", [(BF, F8), (BF, BF), (F32, F32)], ids=str)
def test_one_sequence_of_a_cache_beyond_32_bit_offsets(act, cdtype):
    # 6 GiB of rows; the sequence starts before the 4 GiB mark and ends behind it
    H = 20
    row_bytes = 128 * H * (1 if cdtype == F8 else 2 if cdtype == BF else 4)
    n_rows = (6 << 30) // row_bytes
    if cdtype == F8:
        data = torch.zeros((n_rows, H, 2, 64), dtype=torch.uint8, device="cuda").view(F8)
        cache = wf.Cache(data, torch.zeros((2 * H, n_rows), dtype=torch.uint8, device="cuda"))
    else:
        cache = wf.Cache(torch.zeros((n_rows, 128 * H), dtype=cdtype, device="cuda"))
    first = (4 << 30) // row_bytes - 150
    T = 300
    k, v = _sources(T, H, act, 24)
    k = (k.float() / k.float().abs().amax(1, keepdim=True) * 3).to(act)
    v = (v.float() / v.float().abs().amax(1, keepdim=True) * 3).to(act)
    small = wf.Cache.empty(T, H, cdtype)
    for c, row in ((cache, first), (small, 0)):
        wf.op_cache_write(c, k, v, _i32([0, T]), _i32([row]))
    assert torch.equal(wf.op_cache_read(cache, _i32([0, T]), _i32([first]), T), wf.op_cache_read(small, _i32([0, T]), _i32([0]), T))
    q = _q(5, H, act, 25)
    a = wf.op_cache_attention(cache, q, _i32([0, 5]), _i32([first]), _i32([T]), 5, T)
    assert torch.equal(a, wf.op_cache_attention(small, q, _i32([0, 5]), _i32([0]), _i32([T]), 5, T)) and a.any()
    # and one sequence longer than 4 GiB: zeros in front of the tokens weigh as much as their logit of 0 says
    if cdtype != F8:
        b = wf.op_cache_attention(cache, q, _i32([0, 5]), _i32([0]), _i32([first + T]), 5, n_rows)
        kv = _contents(small)
        for r, h in ((0, 0), (4, 19)):
            s = kv[:, h, 0] @ _np(q)[r, 64 * h:64 * h + 64] * 0.125
            w = np.exp(s)
            ref = w @ kv[:, h, 1] / (w.sum() + first)
            size = w @ np.abs(kv[:, h, 1]) / (w.sum() + first)
            # 2^20 keys: sums in parts, off by less than 2^12 half steps each
            assert (np.abs(_np(b)[r, 64 * h:64 * h + 64] - ref) <= (2.0 ** -8 if act == BF else 0) * np.abs(ref) + (2.0 ** -12 + 2.0 ** -16) * size).all()


@pytest.mark.parametrize("heads", [(40, 1), (96, 2)], ids=str)
@pytest.mark.parametrize("act,cdtype", KINDS)
def test_attention_of_large_head_groups(act, cdtype, heads):
    Hq, H = heads
    cache = _filled(180, H, cdtype, 51)
    _check_attention(cache, _q(6, Hq, act, 52), [0, 1, 5], [3, 60], [57, 120], 4, 120, heads=[0, 1, Hq // H - 1, Hq - 1])


def test_a_workspace_of_the_callers_own():
    import ctypes as C
    cache, q = _filled(6000, 2, F8, 53), _q(4, 4, BF, 54)
    args = (_i32([0, 1, 4]), _i32([0, 1000]), _i32([6000, 5000]), 3, 6000)
    want = wf.op_cache_attention(cache, q, *args)
    a = wf.WfCacheQuery(dtype=wf.WF_DTYPE_BF16, n_heads=4, n_seqs=2, n_q_rows=4, max_q=3, max_len=6000, scale=0.125)
    need = wf.lib().wf_cache_attention_workspace(C.byref(cache._c), C.byref(a))
    assert need > 0
    room = torch.full((need + 64,), 0xff, dtype=torch.uint8, device="cuda")        # of any content, and not written past its end
    for _ in range(3):
        assert torch.equal(wf.op_cache_attention(cache, q, *args, workspace=room[:need]), want)
    assert (room[need:] == 0xff).all()
    with pytest.raises(wf.WfError) as e:
        wf.op_cache_attention(cache, q, *args, workspace=room[:need - 16])
    assert e.value.code == wf.WF_E_CAPACITY


def test_a_captured_step_follows_the_lengths_on_the_device():
    # one graph: the new token's row is written, then attended to; replayed while lengths, rows and inputs change
    H, cap, B = 4, 120, 3
    for cdtype in (F8, BF):
        cache = wf.Cache.empty(B * cap, H, cdtype)
        fill = _filled(B * cap, H, BF, 26)
        start = [i * cap for i in range(B)]
        wf.op_cache_write(cache, fill.data[:, :64 * H], fill.data[:, 64 * H:], _i32([0, B * cap]), _i32([0]))
        eager = wf.Cache(cache.data.clone(), None if cache.exps is None else cache.exps.clone())
        qkv, cu = torch.zeros((B, 3 * 64 * H), device="cuda", dtype=BF), _i32(range(B + 1))
        rows, at, lens = _i32(start), _i32(start), _i32([0] * B)
        out = torch.zeros((B, 64 * H), device="cuda", dtype=BF)

        def step(c, o):
            wf.op_cache_write(c, qkv[:, 64 * H:128 * H], qkv[:, 128 * H:], cu, at)
            wf.op_cache_attention(c, qkv[:, :64 * H], cu, rows, lens, 1, cap, out=o)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(wf.Cache(cache.data.clone(), None if cache.exps is None else cache.exps.clone()), torch.empty_like(out))
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(cache, out)
        for i in range(6):
            gen = torch.Generator().manual_seed(100 + i)
            n = [1 + 17 * i, 30 + i, cap - 6 + i]
            qkv.copy_(torch.randn(qkv.shape, generator=gen).to(BF).cuda())
            lens.copy_(_i32(n))
            at.copy_(_i32([s + m - 1 for s, m in zip(start, n)]))
            g.replay()
            torch.cuda.synchronize()
            want = torch.empty_like(out)
            step(eager, want)
            torch.cuda.synchronize()
            assert torch.equal(out, want) and torch.equal(cache.data.view(torch.uint8), eager.data.view(torch.uint8)), (cdtype, i)


def test_calls_on_two_streams_at_once():
    caches = [_filled(3000, 4, F8, 27 + i) for i in range(2)]
    qs = [_q(4, 8, BF, 30 + i) for i in range(2)]
    want = [wf.op_cache_attention(c, q, _i32([0, 4]), _i32([0]), _i32([3000]), 4, 3000) for c, q in zip(caches, qs)]
    args = [_i32([0, 4]), _i32([0]), _i32([3000])]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            got[i].append(wf.op_cache_attention(caches[i], qs[i], *args, 4, 3000, stream=s.cuda_stream))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            assert torch.equal(g, want[i])


@pytest.mark.parametrize("heads", [(4, 128), (16, 32)], ids=str)
def test_heads_of_another_size_are_refused(heads):
    cache = _filled(20, 8, BF, 60)
    args = (_i32([0, 3]), _i32([0]))
    x, other = _q(3, 8, BF, 61), _q(3, 8, BF, 62).view(3, *heads)
    for k, v in ((other, other), (x, other), (other, x)):
        with pytest.raises(ValueError):
            wf.op_cache_write(cache, k, v, *args)
    with pytest.raises(ValueError):
        wf.op_cache_attention(cache, other, *args, _i32([20]), 3, 20)
    with pytest.raises(ValueError):
        wf.op_cache_attention(cache, x, *args, _i32([20]), 3, 20, out=torch.empty_like(other))


@pytest.mark.parametrize("src", [BF, F32], ids=str)
def test_finite_values_come_back_finite(src):
    # next to the largest finite value the nearest code would stand for 2^128
    top = torch.finfo(src).max
    x = torch.zeros((3, 64))
    x[0, :3] = torch.tensor([top, -top, 1.5 * 2.0 ** 127])
    x[1, :4] = torch.tensor([1.9375 * 2.0 ** 127, 1.875 * 2.0 ** 127, 1.75 * 2.0 ** 127, -1.0])
    x[2] = -top
    x = x.to(src)
    cache = wf.Cache.empty(3, 1, F8)
    wf.op_cache_write(cache, x.cuda(), x.cuda(), _i32([0, 3]), _i32([0]))
    q, e = D.quantise(x.double().numpy())
    want = q * 2.0 ** (e[:, None] - 127.0)
    assert np.isfinite(want.astype(np.float32)).all()
    for out_dtype in (F32, BF):
        back = wf.op_cache_read(cache, _i32([0, 3]), _i32([0]), 3, out_dtype=out_dtype)
        np.testing.assert_array_equal(_np(back).reshape(3, 2, 64), np.stack([want, want], 1))       # e4m3's 4 bits fit both types
    # one key has all the weight: its value comes out as it is
    for act in (BF, F32):
        out = wf.op_cache_attention(cache, torch.zeros((3, 64), dtype=act, device="cuda"), _i32([0, 1, 2, 3]), _i32([0, 1, 2]), _i32([1, 1, 1]), 1, 1)
        np.testing.assert_array_equal(_np(out), want)


def test_a_split_sequence_next_to_the_largest_length():
    # Bounds of 2^31 - 1 keys split in two: a sequence just longer than a part, whose last keys alone hold something.  Keys of zero weigh the same.
    n, B = (1 << 30) + 70, 512
    if torch.cuda.mem_get_info()[0] < 160 << 30:
        pytest.skip("needs 140 GB for one cache")
    data = torch.zeros((n, 1, 2, 64), dtype=torch.uint8, device="cuda")
    exps = torch.full((2, n), 127, dtype=torch.uint8, device="cuda")
    data[1 << 30:, 0, 1] = 0x38                        # 1
    exps[1, 1 << 30:] = 127 + 30
    cache = wf.Cache(data.view(F8), exps)
    lens = [5] * B
    lens[77] = n
    out = wf.op_cache_attention(cache, _q(B, 1, BF, 63), _i32(range(B + 1)), _i32([0] * B), _i32(lens), 1, 2 ** 31 - 1)
    got, want = _np(out), 70 * 2.0 ** 30 / n
    assert (np.abs(got[77] - want) <= 2.0 ** -8 * want).all()         # sums of whole numbers below 2^24 of them and their multiples: exact
    assert not got[:77].any() and not got[78:].any()
    del cache, data, exps
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n_keys", [40, 1600])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("act,cdtype", KINDS)
def test_logits_beyond_fp32_do_not_look_like_no_keys(act, cdtype, masked, n_keys):
    # q . k = 64 * 2^63 is finite, 2^60 times it is not: NaN and no zeros; rows of ordinary logits beside them stay as they are
    cache = wf.Cache.empty(n_keys, 1, cdtype)
    x = torch.zeros((n_keys, 64), dtype=act if cdtype == F8 else cdtype, device="cuda")
    x[:, :] = 2.0 ** 63
    wf.op_cache_write(cache, x, torch.ones_like(x), _i32([0, n_keys]), _i32([0]))
    q = torch.zeros((18, 64), dtype=act, device="cuda")
    q[1], q[17] = 1.0, 1.0
    q[2] = -1.0                                        # every logit -infinity in fp32: each weighs nothing
    mask = torch.full((18, 2), -1, dtype=torch.int32, device="cuda") if masked else None
    for n_q in (3, 18):
        out = _np(wf.op_cache_attention(cache, q[:n_q], _i32([0, n_q]), _i32([0]), _i32([n_keys]), n_q, n_keys, scale=2.0 ** 60,
                                        mask=mask if mask is None else mask[:n_q]))
        assert np.isnan(out[1]).all() and (out[0] == 1.0).all() and not out[2].any() and (out[3:17] == 1.0).all()
        assert n_q == 3 or np.isnan(out[17]).all()


def test_calls_do_not_follow_a_cache_whose_memory_moved():
    for dtype in (BF, F8):
        cache = _filled(40, 2, dtype, 64)
        q, args = _q(2, 2, BF, 65), (_i32([0, 2]), _i32([0]))
        with pytest.raises(AttributeError):
            cache.data = torch.zeros_like(cache.data)
        t = cache.data if dtype == BF else cache.exps
        t.resize_(400 * t.shape[0], *t.shape[1:])
        for call in (lambda: wf.op_cache_write(cache, q, q, *args), lambda: wf.op_cache_read(cache, *args, 2),
                     lambda: wf.op_cache_attention(cache, q, *args, _i32([9]), 2, 9)):
            with pytest.raises(ValueError):
                call()


@pytest.mark.parametrize("act,cdtype", KINDS)
def test_bounds_beyond_32_bits_bound_nothing(act, cdtype):
    cache = _filled(90, 2, cdtype, 66)
    _check_attention(cache, _q(7, 4, act, 67), [0, 3, 7], [0, 30], [71, 60], 2 ** 33 + 1, 2 ** 32 + 5)


@pytest.mark.parametrize("n_keys", [40, 1700])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("act,cdtype", KINDS)
def test_large_logits_still_share_out_the_weight(act, cdtype, masked, n_keys):
    # q . k is one product of a few bits, the logit in powers of two is not: its rounded value is off by up to 2^-25 of it.  Equal logits share the
    # weight, whatever their size; keys far below others have none.
    for p in (20, 29, 31, 33, 34, 35, 40, 63, 100):
        for sign in (1, -1):
            cache = _filled(n_keys, 1, cdtype, 70)
            k = torch.zeros((n_keys, 64))
            k[:, 0] = sign * 1.625 * 2.0 ** p
            if sign < 0:
                k[n_keys - 3:, 0] = 0.0                # for the second sequence: three keys have all the weight
            kd = k.to(act).cuda()
            v = _np(wf.op_cache_read(cache, _i32([0, n_keys]), _i32([0]), n_keys, out_dtype=F32))[:, 64:]
            wf.op_cache_write(cache, kd, torch.from_numpy(v).to(act).cuda(), _i32([0, n_keys]), _i32([0]))
            v = _contents(cache)[:, 0, 1]
            q = torch.zeros((20, 64), dtype=act, device="cuda")
            q[:, 0] = 1.3984375
            mask = torch.full((20, -(-n_keys // 32)), -1, dtype=torch.int32, device="cuda") if masked else None
            for scale in (0.1, 0.125, 0.3):
                lens = [n_keys - 3, n_keys]
                out = _np(wf.op_cache_attention(cache, q, _i32([0, 1, 20]), _i32([0, 0]), _i32(lens), 19, n_keys, scale=scale, mask=mask))
                for rows, w in ((out[:1], v[:lens[0]]), (out[1:], v[n_keys - 3:] if sign < 0 and p > 20 else v if sign > 0 else None)):
                    if w is not None:
                        tol = _tolerance(act, len(w), w.mean(0), np.abs(w).mean(0), 0.0)
                        assert (np.abs(rows - w.mean(0)) <= tol).all(), (p, sign, scale, len(w))


@pytest.mark.parametrize("length", [60, 200])
@pytest.mark.parametrize("n_q", [9, 20])
@pytest.mark.parametrize("act,cdtype", KINDS)
def test_many_short_sequences_of_several_row_chunks(act, cdtype, n_q, length):
    # 18 and 40 rows a key head; where a workgroup has 16 of them it may have one or two waves as well
    B, H = 70, 8
    lens = [(length * (i % 6)) // 5 for i in range(B)]
    rows = [(i * 53) % 700 for i in range(B)]
    cache = _filled(900, H, cdtype, 68)
    q = _q(B * n_q, 2 * H, act, 69)
    cu = [i * n_q for i in range(B + 1)]
    some = {0, n_q - 1, n_q, 5 * n_q + 8, B * n_q - 1}
    _check_attention(cache, q, cu, rows, lens, n_q, length, heads=[0, 15], some_rows=some)
    words = torch.from_numpy(np.random.default_rng(70).integers(0, 1 << 32, (B * n_q, 2), dtype=np.uint32).view(np.int32)).cuda()
    _check_attention(cache, q, cu, rows, lens, n_q, length, heads=[0, 15], some_rows=some, mask=words, since=[max(0, n - 40) for n in lens])
