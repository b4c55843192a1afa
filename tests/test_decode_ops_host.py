"""CPU-only checks of the decoding operators' entry points: what the host refuses before it launches anything, what it
accepts without work to do, and the oracle's own pins."""
import ctypes as C
import types

import numpy as np
import pytest
import torch

from oracle import decode_oracle as D
from paper_2412_11272_amd import binding as wf

P = 1 << 20            # an aligned address nobody follows: every call below ends on the host


def _cache(**kw):
    return wf.WfCache(**{**dict(data_dev=P, exps_dev=P, n_rows=100, n_heads=4, dtype=wf.WF_DTYPE_F8), **kw})


def _write(cache, **kw):
    a = {**dict(k=P, v=P, dtype=wf.WF_DTYPE_BF16, ld=256, cu=P, row=P, B=2, n=0), **kw}
    return wf.lib().wf_op_cache_write(C.byref(cache) if cache else None, a["k"], a["v"], a["dtype"], a["ld"], a["cu"], a["row"], a["B"], a["n"], None)


def _read(cache, **kw):
    a = {**dict(cu=P, row=P, B=2, out=P, dtype=wf.WF_DTYPE_F32, n=0), **kw}
    return wf.lib().wf_op_cache_read(C.byref(cache) if cache else None, a["cu"], a["row"], a["B"], a["out"], a["dtype"], a["n"], None)


BAD_CACHE = [dict(dtype=7), dict(n_heads=0), dict(n_heads=1025), dict(n_rows=0), dict(n_rows=1 << 31)]
BAD_MEMORY = [dict(data_dev=None), dict(data_dev=P + 8), dict(exps_dev=None), dict(dtype=wf.WF_DTYPE_BF16)]


def test_struct_sizes_match_the_header():
    assert C.sizeof(wf.WfCache) == 32 and C.sizeof(wf.WfCacheQuery) == 120 and C.sizeof(wf.WfBeamStep) == 120


@pytest.mark.parametrize("bad", BAD_CACHE, ids=str)
def test_every_cache_call_refuses_a_bad_cache(bad):
    c = _cache(**bad)
    assert _write(c) == _read(c) == wf.WF_E_INVALID_ARG and "cache" in wf.last_error()
    assert wf.lib().wf_cache_attention_workspace(C.byref(c), C.byref(_query())) == wf.WF_E_INVALID_ARG
    assert wf.lib().wf_op_cache_attention(C.byref(c), C.byref(_query()), None) == wf.WF_E_INVALID_ARG


@pytest.mark.parametrize("bad", BAD_MEMORY, ids=str)
def test_every_cache_call_refuses_bad_cache_memory(bad):
    c = _cache(**bad)
    assert _write(c, n=5) == _read(c, n=5) == wf.WF_E_INVALID_ARG
    assert wf.lib().wf_op_cache_attention(C.byref(c), C.byref(_query(n_q_rows=3)), None) == wf.WF_E_INVALID_ARG


def test_write_and_read_arguments():
    c = _cache()
    assert _write(None) == _read(None) == wf.WF_E_INVALID_ARG
    assert _write(c) == _read(c) == wf.WF_OK                        # no token: nothing to do
    for bad in (dict(dtype=wf.WF_DTYPE_F8), dict(B=0), dict(n=-1), dict(n=5, cu=None), dict(n=5, row=None)):
        assert _write(c, **bad) == _read(c, **bad) == wf.WF_E_INVALID_ARG, bad
    for bad in (dict(ld=255), dict(n=5, k=None), dict(n=5, v=None), dict(n=5, k=P + 8), dict(n=5, v=P + 2), dict(n=5, ld=260)):
        assert _write(c, **bad) == wf.WF_E_INVALID_ARG, bad
    assert _write(c, n=1 << 25) == _read(c, n=1 << 25) == wf.WF_E_CAPACITY
    assert _read(c, n=5, out=None) == _read(c, n=5, out=P + 4) == wf.WF_E_INVALID_ARG


def _query(**kw):
    return wf.WfCacheQuery(**{**dict(q_dev=P, out_dev=P, ldq=512, ldo=512, cu_q_dev=P, row_dev=P, len_dev=P, dtype=wf.WF_DTYPE_BF16, n_heads=8, n_seqs=2,
                                     n_q_rows=0, max_q=4, max_len=50, scale=0.125), **kw})


def test_attention_arguments():
    c = _cache()
    L = wf.lib()

    def call(cache=c, **kw):
        return L.wf_op_cache_attention(C.byref(cache), C.byref(_query(**kw)), None)

    assert call() == wf.WF_OK                                       # no row: nothing to do
    assert L.wf_op_cache_attention(None, C.byref(_query()), None) == L.wf_op_cache_attention(C.byref(c), None, None) == wf.WF_E_INVALID_ARG
    for bad in (dict(dtype=wf.WF_DTYPE_F8), dict(n_heads=0), dict(n_heads=6), dict(n_seqs=0), dict(n_q_rows=-1), dict(max_q=0), dict(max_len=-1),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(ldq=511), dict(ldo=511), dict(mask_dev=P, mask_words=0), dict(mask_from_dev=P),
                dict(n_q_rows=1, q_dev=None), dict(n_q_rows=1, out_dev=None), dict(n_q_rows=1, cu_q_dev=None), dict(n_q_rows=1, row_dev=None),
                dict(n_q_rows=1, len_dev=None), dict(n_q_rows=1, q_dev=P + 8), dict(n_q_rows=1, out_dev=P + 8), dict(n_q_rows=1, ldq=516),
                dict(n_q_rows=1, ldo=516)):
        assert call(**bad) == wf.WF_E_INVALID_ARG, bad
    assert call(_cache(dtype=wf.WF_DTYPE_F32, exps_dev=None)) == wf.WF_E_INVALID_ARG       # bf16 queries over a fp32 cache
    assert call(n_seqs=1 << 20, n_q_rows=1 << 20, max_q=1 << 20) == wf.WF_E_CAPACITY
    assert L.wf_cache_attention_workspace(C.byref(c), C.byref(_query())) >= 0
    long = _query(n_q_rows=2, max_len=1 << 20)                      # split over workgroups: the parts need room
    need = L.wf_cache_attention_workspace(C.byref(c), C.byref(long))
    assert need > 0 and call(n_q_rows=2, max_len=1 << 20) == wf.WF_E_INVALID_ARG
    assert call(n_q_rows=2, max_len=1 << 20, workspace_dev=P, workspace_bytes=need - 1) == wf.WF_E_CAPACITY
    assert call(n_q_rows=2, max_len=1 << 20, workspace_dev=P + 8, workspace_bytes=need) == wf.WF_E_INVALID_ARG


def test_a_scale_whose_binary_logits_overflow():
    c = _cache()
    for scale in (2.4e38, -2.4e38, 3.4e38):
        assert wf.lib().wf_op_cache_attention(C.byref(c), C.byref(_query(scale=scale)), None) == wf.WF_E_INVALID_ARG
    assert wf.lib().wf_op_cache_attention(C.byref(c), C.byref(_query(scale=-2.3e38)), None) == wf.WF_OK


def _step(**kw):
    return wf.WfBeamStep(**{**dict(logits_dev=P, ld=100, score_in_dev=P, token_out_dev=P, parent_out_dev=P, score_out_dev=P, workspace_dev=P,
                                   workspace_bytes=0, dtype=wf.WF_DTYPE_F32, B=2, width=5, n_vocab=100, eos=-1), **kw})


def test_beam_select_arguments():
    L = wf.lib()

    def call(**kw):
        return L.wf_op_beam_select(C.byref(_step(**kw)), None)

    assert L.wf_op_beam_select(None, None) == L.wf_beam_select_workspace(None) == wf.WF_E_INVALID_ARG
    need = L.wf_beam_select_workspace(C.byref(_step()))
    assert need > 0
    assert call(workspace_bytes=need - 1) == wf.WF_E_CAPACITY       # all else is in order: the workspace is looked at last
    for bad in (dict(dtype=wf.WF_DTYPE_F8), dict(B=0), dict(width=0), dict(width=33), dict(n_vocab=0), dict(logits_dev=None), dict(score_in_dev=None),
                dict(token_out_dev=None), dict(parent_out_dev=None), dict(score_out_dev=None), dict(ld=99), dict(done_in_dev=P), dict(done_out_dev=P),
                dict(done_in_dev=P, done_out_dev=P, eos=100), dict(done_in_dev=P, done_out_dev=P, eos=-1), dict(workspace_dev=None),
                dict(workspace_dev=P + 8), dict(logits_dev=P + 2), dict(logits_dev=P + 1, dtype=wf.WF_DTYPE_BF16)):
        assert call(**{**dict(workspace_bytes=0), **bad}) == wf.WF_E_INVALID_ARG, bad
    assert call(B=1 << 20) == wf.WF_E_CAPACITY


def _step_over(**kw):
    return wf.lib().wf_beam_select_workspace(C.byref(_step(**kw)))


def test_beam_reorder_arguments():
    def call(dst=P, src=P, parent=P, length=None, B=2, width=3, layers=0, n_pos=10, pos_bytes=16):
        return wf.lib().wf_op_beam_reorder(dst, src, parent, length, B, width, layers, n_pos, pos_bytes, None)

    assert call() == call(layers=2, n_pos=0) == wf.WF_OK            # nothing to move
    for bad in (dict(B=0), dict(width=0), dict(width=33), dict(layers=-1), dict(n_pos=-1), dict(pos_bytes=0), dict(layers=1, dst=None),
                dict(layers=1, src=None), dict(layers=1, parent=None), dict(layers=1, src=P + 2 * 3 * 160 - 1), dict(layers=1, src=P - 16),
                dict(layers=2, n_pos=1 << 40, pos_bytes=1 << 40)):
        assert call(**bad) == wf.WF_E_INVALID_ARG, bad
    assert call(layers=2, n_pos=1 << 40) == call(layers=1, n_pos=1 << 34, pos_bytes=1) == wf.WF_E_CAPACITY
    assert _step_over(n_vocab=(1 << 28) + 1) == wf.WF_E_CAPACITY


@pytest.mark.parametrize("n_pos,pos_bytes", [((1 << 63) - 1, 1), ((1 << 63) - 4096, 1), (1, (1 << 63) - 16), ((1 << 62) - 1, 2)], ids=str)
def test_slots_next_to_the_largest_number_of_bytes(n_pos, pos_bytes):
    """Rounding such a slot up to whole workgroups leaves 64 bits."""
    assert wf.lib().wf_op_beam_reorder(P, P, P, None, 1, 1, 1, n_pos, pos_bytes, None) == wf.WF_E_CAPACITY


def test_binding_refuses_host_tensors():
    with pytest.raises(ValueError):
        wf.Cache(torch.zeros((4, 128)))
    with pytest.raises(ValueError):
        wf.op_beam_select(torch.zeros((1, 2, 10)), torch.zeros((1, 2)))
    with pytest.raises(ValueError):
        wf.op_beam_reorder(torch.zeros((1, 2, 3)), torch.zeros((1, 2), dtype=torch.int32))


def test_device_and_stream_of_a_call_without_torchs_private_functions(monkeypatch):
    """torch's private handles are used where this torch has them and not relied on."""
    t = types.SimpleNamespace(get_device=lambda: 3, device="cuda:3")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=55))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 100 + device, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 3, raising=False)
    assert wf._here(t, "q") == 3 and wf._stream_on(None, 3) == 103 and wf._stream_on(0, 3) == 0 and wf._stream_on(77, 3) == 77
    for private in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
        monkeypatch.delattr(torch._C, private)
    assert wf._here(t, "q") == 3 and wf._stream_on(None, 3) == 55
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 2)
    with pytest.raises(ValueError, match="q is on cuda:3"):
        wf._here(t, "q")


@pytest.mark.parametrize("shape", [(5, 4, 32), (5, 4, 128), (5, 1, 128), (0, 2, 32), (5, 2, 64, 1)], ids=str)
def test_a_third_dimension_is_a_heads_64_values(shape):
    """[n, 4, 128] is no 8 heads of 64: folding it would cut its heads in two."""
    with pytest.raises(ValueError, match="q"):
        wf._rows_2d(torch.zeros(shape), -1, "q")


def test_rows_of_heads_and_their_strides():
    wide = torch.zeros((7, 6, 64))
    assert wf._rows_2d(wide, -1, "q") == wf._rows_2d(wide.view(7, 384), -1, "q") == (7, 384, 384)
    assert wf._rows_2d(wide[:, 2:4], -1, "q") == (7, 128, 384)
    assert wf._rows_2d(wide[:, 3:4], -1, "q") == (7, 64, 384) and wf._rows_2d(wide[:1, 2:4], -1, "q") == (1, 128, 128)
    for bad in (wide[:, ::2], wide[:, :, ::2], wide.transpose(1, 2), wide.view(7, 384).t()):
        with pytest.raises(ValueError):
            wf._rows_2d(bad, -1, "q")


def _fake(shape, dtype, at, device=0):
    """What Cache asks of a tensor on a device."""
    t = torch.empty(shape, dtype=dtype, device="meta")
    return types.SimpleNamespace(shape=t.shape, dtype=dtype, device=f"cuda:{device}", get_device=lambda: device, is_contiguous=lambda: True, stride=t.stride,
                                 data_ptr=lambda: at)


def test_a_cache_keeps_to_the_memory_it_was_made_of(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    data, exps = _fake((9, 2, 2, 64), torch.float8_e4m3fn, 4096), _fake((4, 9), torch.uint8, 1 << 20)
    c = wf.Cache(data, exps)
    assert (c.data, c.exps, c.n_rows, c.n_heads, c.device) == (data, exps, 9, 2, 0) and c._here() == 0
    assert (c._c.data_dev, c._c.exps_dev) == (4096, 1 << 20)
    for name in ("data", "exps", "n_rows", "n_heads", "device"):
        with pytest.raises(AttributeError):
            setattr(c, name, getattr(c, name))
    for t in (data, exps):                                          # grown in place, its memory is elsewhere
        was, t.data_ptr = t.data_ptr, lambda: 1 << 30
        with pytest.raises(ValueError, match="moved"):
            c._here()
        t.data_ptr = was
    assert c._here() == 0
    c = wf.Cache(_fake((9, 256), torch.bfloat16, 4096, device=1))
    with pytest.raises(ValueError, match="cuda:1"):
        c._here()


@pytest.mark.parametrize("value", [1 << 31, (1 << 32) + 5, -(1 << 31) - 1], ids=str)
def test_numbers_that_32_bits_do_not_hold(value, monkeypatch):
    """The library's int32 would take such a number's low bits; an upper bound beyond every length is the largest one."""
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    logits = _fake((1, 1, max(value, 1)), torch.float32, P)
    logits.stride = lambda: (logits.shape[2], logits.shape[2], 1)
    scores, done = _fake((1, 1), torch.float32, P), _fake((1, 1), torch.uint8, P)
    if value > 0:
        with pytest.raises(ValueError, match="n_vocab"):
            wf.op_beam_select(logits, scores)
    logits = _fake((1, 1, 100), torch.float32, P)
    logits.stride = lambda: (100, 100, 1)
    with pytest.raises(ValueError, match="eos"):
        wf.op_beam_select(logits, scores, done=done, eos=value)
    assert wf._bound(value) == (0x7fffffff if value > 0 else -1) and wf._bound(77) == 77 and wf._bound(0x7fffffff) == 0x7fffffff


# ---- the oracle's own pins ------------------------------------------------------------------------------------------------
def test_oracle_format_is_torchs_e4m3():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(codes, D.e4m3_values())
    x = np.concatenate([np.linspace(-448, 448, 7001), np.linspace(-0.02, 0.02, 3001)]).astype(np.float32)
    x = x[:len(x) // 64 * 64].reshape(-1, 64)
    q, b = D.quantise(x)
    e = b - 127
    assert (np.abs(x).max(1) <= 448 * 2.0 ** e).all() and (np.abs(x).max(1) > 224 * 2.0 ** e).all()
    ref = torch.from_numpy((x * 2.0 ** -e[:, None]).astype(np.float32)).to(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(q, ref)
    q, b = D.quantise(np.array([[0.0] * 64, [np.nan, np.inf, -np.inf, 1.0] + [0.0] * 60, [2.0 ** -149] * 64]))
    assert b.tolist() == [0, 119, 0] and not q[0].any() and np.isnan(q[1, :3]).all() and q[1, 3] == 256.0 and not q[2].any()


def test_oracle_keeps_finite_values_finite():
    top = float(np.finfo(np.float32).max)
    x = np.zeros((4, 64))
    x[0, :3] = top, -top, 1.5 * 2.0 ** 127
    x[1, :2] = 1.9375 * 2.0 ** 127, 1.9374 * 2.0 ** 127            # where rounding would go up to 2^128, and just below
    x[2, :2] = 1.75 * 2.0 ** 127, 1.0                              # one exponent lower: 448 itself is a finite value there
    x[3] = top
    q, b = D.quantise(x)
    assert b.tolist() == [247, 247, 246, 247]
    assert q[0, :3].tolist() == [240.0, -240.0, 192.0] and q[1, :2].tolist() == [240.0, 240.0] and q[2, 0] == 448.0 and (q[3] == 240.0).all()
    assert (np.abs(q) * 2.0 ** (b[:, None] - 127.0) <= top).all()


def test_oracle_attention_is_a_softmax_over_the_visible_keys():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal(64), rng.standard_normal((40, 64)), rng.standard_normal((40, 64))
    seen = D.visible(40, [0b1011, 1 << 31], 5)
    assert np.flatnonzero(seen).tolist() == [0, 1, 2, 3, 4, 5, 6, 8]
    ref = torch.nn.functional.scaled_dot_product_attention(*(torch.from_numpy(x)[None, None] for x in (q[None], k[seen], v[seen])))
    np.testing.assert_allclose(D.attention(q, k, v, 0.125, seen)[0], ref[0, 0, 0].numpy(), rtol=1e-12, atol=1e-14)
    assert not D.attention(q, k, v, 0.125, np.zeros(40, bool))[0].any()


def test_oracle_beam_step_by_hand():
    x = np.array([[0.0, 1.0, 1.0, -np.inf], [3.0, np.nan, 3.0, np.inf]])
    tok, par, sc, dn = D.beam_step(x, np.array([-1.0, -1.0]), 2, 2)
    assert tok.tolist() == [0, 2] and par.tolist() == [1, 1]        # beam 1: two equal tokens of probability 1/2 each, the lowest first
    np.testing.assert_allclose(sc, -1.0 + np.log(0.5))
    tok, par, _, _ = D.beam_step(x, np.array([-1.0, -1.0]), 1, 2)
    assert tok.tolist() == [1, 2] and par.tolist() == [0, 0]
    tok, par, sc, dn = D.beam_step(x, np.array([-1.0, -0.5]), 2, 2, done=[0, 1], eos=3, keep_slots=True)
    assert tok.tolist() == [1, 3] and par.tolist() == [0, 1] and dn.tolist() == [False, True] and sc[1] == -0.5
