"""Beam selection and reordering on the GPU against the 64-bit definitions of oracle/decode_oracle.py."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle as D
from paper_2412_11272_amd import binding as wf

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _i32(x):
    return torch.tensor(np.asarray(x, np.int32), device="cuda")


def _check_select(logits, scores, n_in=None, n_out=None, done=None, eos=-1, keep_slots=False):
    B, W, V = logits.shape
    sc = torch.tensor(np.asarray(scores, np.float32), device="cuda")
    dn = None if done is None else torch.tensor(np.asarray(done, bool), device="cuda")
    tok, par, out, dout = wf.op_beam_select(logits, sc, n_in=None if n_in is None else _i32(n_in), n_out=None if n_out is None else _i32(n_out),
                                            done=dn, eos=eos, keep_slots=keep_slots)
    torch.cuda.synchronize()
    x, s32 = logits.double().cpu().numpy(), sc.double().cpu().numpy()
    for s in range(B):
        cut = lambda n: W if n is None else min(max(int(n[s]), 0), W)  # noqa: E731
        rt, rp, rs, rd = D.beam_step(x[s], s32[s], cut(n_in), cut(n_out), None if done is None else done[s], eos, keep_slots)
        assert tok[s].tolist() == rt.tolist() and par[s].tolist() == rp.tolist(), s
        got = out[s].double().cpu().numpy()
        some = np.isfinite(rs)
        assert (np.isneginf(got) == ~some).all()
        # half a step of fp32 at the end, and the log of a sum whose exponentials and additions are off by less than 2^-21
        assert (np.abs(got[some] - rs[some]) <= 2.0 ** -24 * np.abs(rs[some]) + 2.0 ** -21).all()
        if done is not None:
            assert dout[s].tolist() == rd.tolist()
    return tok, par


def _logits(B, W, V, seed, dtype=F32, spread=2.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((B, W, V), generator=g) * spread).to(dtype).cuda()


def _scores(B, W, seed):
    return -np.cumsum(np.random.default_rng(seed).uniform(0.1, 5.0, (B, W)), 1)


@pytest.mark.parametrize("V", [1, 2, 5, 63, 64, 65, 511, 2047, 2048, 2049, 4097, 8191, 10007, 51866])
@pytest.mark.parametrize("dtype", [F32, BF], ids=str)
def test_select_over_vocabularies(dtype, V):
    _check_select(_logits(2, 5, V, V, dtype), _scores(2, 5, V))


@pytest.mark.parametrize("W", [1, 2, 3, 4, 8, 13, 16, 31, 32])
@pytest.mark.parametrize("keep", [False, True])
def test_select_over_widths(W, keep):
    _check_select(_logits(3, W, 1003, W), _scores(3, W, W), keep_slots=keep)
    _check_select(_logits(2, W, 7, W), _scores(2, W, W), keep_slots=keep)         # fewer tokens than beams in some


def test_select_takes_the_lowest_of_equal_candidates():
    x = torch.zeros((2, 4, 3001))
    x[0, 1, [5, 2900, 17]] = 3.0
    x[1] = torch.randint(0, 3, (4, 3001), generator=torch.Generator().manual_seed(1)).float()
    x[1, 2, :100] = -0.0                                       # equal to +0
    _check_select(x.cuda(), np.zeros((2, 4)) - 1.0)
    same = _logits(1, 1, 5000, 2).expand(1, 6, 5000).contiguous()       # every beam offers the same
    tok, par = _check_select(same, np.full((1, 6), -2.5))
    assert par[0].tolist() == [0, 1, 2, 3, 4, 5] and len(set(tok[0].tolist())) == 1


@pytest.mark.parametrize("keep", [False, True])
def test_select_with_ragged_and_finished_beams(keep):
    B, W, V = 7, 5, 4001
    n_in, n_out = [5, 1, 0, 3, 5, -2, 9], [5, 5, 5, 1, 0, 3, 9]
    done = np.random.default_rng(3).random((B, W)) < 0.4
    done[0] = True                                             # every beam of the stream is done
    for d in (None, done):
        _check_select(_logits(B, W, V, 4), _scores(B, W, 5), n_in, n_out, d, eos=V - 1, keep_slots=keep)
    x = _logits(B, W, V, 4)
    x[:, :, 17] = 30.0                                         # the best token ends the beams
    _check_select(x, _scores(B, W, 5), None, None, done, eos=17, keep_slots=keep)


def test_logits_and_scores_that_are_not_finite_take_no_part():
    x = _logits(5, 4, 2500, 6)
    x[0, :, 100:] = -float("inf")                              # suppressed
    x[1, 1] = -float("inf")                                    # a beam with nothing left
    x[2] = float("nan")                                        # a stream with nothing left
    x[3, 0, ::7] = float("nan"); x[3, 1, 5] = float("inf"); x[3, 2] = -3.4e38; x[3, 3] = 3.4e38
    x[4, :, 2:] = -float("inf")                                # fewer candidates than slots
    sc = _scores(5, 4, 7)
    sc[0, 0], sc[1, 0], sc[4, 1:] = np.nan, np.inf, -np.inf
    tok, _ = _check_select(x, sc)
    assert (tok[2] == -1).all() and tok[4].tolist()[2:] == [-1, -1]


def test_select_reads_rows_of_any_stride_and_alignment():
    wide = _logits(2, 3, 1037, 8)
    for V, off in ((1001, 1), (1003, 2), (1002, 3), (1037, 0)):
        _check_select(wide[:, :, off:off + V], _scores(2, 3, 9))
    wide = _logits(2, 3, 1037, 8, BF)
    for V, off in ((1001, 1), (1003, 2), (1002, 3), (1000, 8), (1029, 5)):
        _check_select(wide[:, :, off:off + V], _scores(2, 3, 9))
    with pytest.raises(ValueError):
        wf.op_beam_select(wide[:, :, ::2], torch.zeros((2, 3), device="cuda"))


@pytest.mark.parametrize("order", ["up", "down", "late", "peaks"])
def test_select_where_the_best_come_late_or_together(order):
    V = 30011
    x = torch.linspace(-9, 9, V).expand(1, 5, V).clone()
    if order == "down":
        x = x.flip(2)
    if order == "late":
        x[:, :, :] = -5.0
        x[:, :, -3:] = torch.tensor([1.0, 2.0, 1.0])
    if order == "peaks":                                       # the best all in neighbouring places
        x[:] = torch.randn((1, 5, V), generator=torch.Generator().manual_seed(3))
        x[:, :, 20000:20040] += 20.0
    x = x.contiguous().cuda()
    _check_select(x, _scores(1, 5, 10))
    _check_select(x[:, :, 1:], _scores(1, 5, 10))


def test_select_may_overwrite_its_own_scores():
    import ctypes as C
    x, sc = _logits(3, 5, 900, 11), torch.tensor(_scores(3, 5, 11).astype(np.float32), device="cuda")
    done = torch.zeros((3, 5), dtype=torch.uint8, device="cuda")
    done[1, 2] = 1
    tok, par, score, dout = wf.op_beam_select(x, sc, done=done, eos=3)
    t2, p2 = torch.empty_like(tok), torch.empty_like(par)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    a = wf.WfBeamStep(x.data_ptr(), 900, None, None, sc.data_ptr(), done.data_ptr(), t2.data_ptr(), p2.data_ptr(), sc.data_ptr(), done.data_ptr(),
                      ws.data_ptr(), ws.numel(), wf.WF_DTYPE_F32, 3, 5, 900, 3, 0)
    assert wf.lib().wf_op_beam_select(C.byref(a), torch.cuda.current_stream().cuda_stream) == wf.WF_OK
    assert torch.equal(t2, tok) and torch.equal(p2, par) and torch.equal(sc, score) and torch.equal(done, dout)


def test_a_workspace_of_the_callers_own():
    import ctypes as C
    x, sc = _logits(3, 5, 9001, 12), torch.tensor(_scores(3, 5, 12).astype(np.float32), device="cuda")
    want = wf.op_beam_select(x, sc)
    need = wf.lib().wf_beam_select_workspace(C.byref(wf.WfBeamStep(dtype=wf.WF_DTYPE_F32, B=3, width=5, n_vocab=9001)))
    room = torch.full((need + 64,), 0xff, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        got = wf.op_beam_select(x, sc, workspace=room[:need])
        assert all(torch.equal(a, b) for a, b in zip(got[:3], want[:3]))
    assert (room[need:] == 0xff).all()
    with pytest.raises(wf.WfError) as e:
        wf.op_beam_select(x, sc, workspace=room[:need - 16])
    assert e.value.code == wf.WF_E_CAPACITY


def test_select_on_another_stream_than_the_current_one():
    x, sc = _logits(8, 5, 20000, 13), torch.tensor(_scores(8, 5, 13).astype(np.float32), device="cuda")
    want = wf.op_beam_select(x, sc)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [wf.op_beam_select(x, sc, stream=s.cuda_stream) for _ in range(5) for s in streams]
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g[:3], want[:3]))


# ---- reordering -------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("inside", [(96, "bf16"), (5, "u8"), (3, "f32"), (64, "u8")], ids=str)
@pytest.mark.parametrize("W", [1, 2, 5, 8, 9, 17, 32])
def test_reorder(W, inside):
    width, kind = inside
    B, layers, n_pos = 3, 2, 37
    g = torch.Generator().manual_seed(W)
    dt = {"bf16": torch.int16, "u8": torch.uint8, "f32": torch.int32}[kind]
    state = torch.randint(0, 255, (layers, B * W, n_pos, width), generator=g).to(dt)
    other = torch.randint(0, 255, state.shape, generator=g).to(dt)
    rng = np.random.default_rng(W)
    for lens in (None, [37, 0, 12], [50, -4, 1]):
        parents = rng.integers(-1, W + 1, (B, W))              # some say: leave the slot
        parents[0] = np.roll(np.arange(W), 1)                  # a ring: every slot is read before it is overwritten
        length = None if lens is None else _i32(lens)
        a = state.cuda()
        assert wf.op_beam_reorder(a, _i32(parents), lens=length) is a
        np.testing.assert_array_equal(a.cpu().numpy(), D.reorder(state.numpy(), parents, lens, state.numpy()))
        b = other.cuda()
        wf.op_beam_reorder(state.cuda(), _i32(parents), lens=length, out=b)
        np.testing.assert_array_equal(b.cpu().numpy(), D.reorder(state.numpy(), parents, lens, other.numpy()))


def test_reorder_of_unaligned_states_and_refusals():
    buf = torch.arange(1 + 4 * 6 * 10, dtype=torch.uint8, device="cuda")
    state = buf[1:].view(1, 4, 6, 10)
    want = D.reorder(state.cpu().numpy(), np.array([[1, 0], [1, 1]]), None, state.cpu().numpy())
    wf.op_beam_reorder(state, _i32([[1, 0], [1, 1]]))
    np.testing.assert_array_equal(state.cpu().numpy(), want)
    with pytest.raises(wf.WfError):
        wf.op_beam_reorder(buf[:200].view(1, 4, 5, 10), _i32([[1, 0], [1, 1]]), out=buf[10:210].view(1, 4, 5, 10))
    with pytest.raises(ValueError):
        wf.op_beam_reorder(state, _i32([[1, 0]]))
    with pytest.raises(TypeError):
        wf.op_beam_reorder(state, _i32([[1, 0], [1, 1]]).long())


def test_reorder_of_a_state_beyond_32_bit_offsets():
    state = torch.zeros((1, 4, 3, 1 << 29), dtype=torch.uint8, device="cuda")          # 6 GiB
    state[0, 3, :, -5:] = 9
    state[0, 2, 1, :7] = 5
    wf.op_beam_reorder(state, _i32([[3, 1, 3, 2]]))
    for j, src in ((0, 3), (2, 3), (3, 2)):
        assert (state[0, j, :, -5:] == (9 if src == 3 else 0)).all() and (state[0, j, 1, :7] == (0 if src == 3 else 5)).all()


def test_selection_and_reordering_in_a_graph():
    B, W, V, cap = 4, 5, 3001, 20
    x, sc = torch.zeros((B, W, V), device="cuda"), torch.zeros((B, W), device="cuda")
    n_in, n_out, lens = _i32([W] * B), _i32([W] * B), _i32([0] * B)
    state = torch.zeros((2, B * W, cap, 64), dtype=BF, device="cuda")
    wf.op_beam_select(x, sc, n_in=n_in, n_out=n_out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tok, par, score, _ = wf.op_beam_select(x, sc, n_in=n_in, n_out=n_out, keep_slots=True)
        wf.op_beam_reorder(state, par, lens=lens)
    for i in range(5):
        x.copy_(_logits(B, W, V, 50 + i))
        sc.copy_(torch.tensor(_scores(B, W, i).astype(np.float32)))
        n_in.copy_(_i32([1, W, 3, 1 + i % W]))
        n_out.copy_(_i32([W, W, 1 + i % W, 2]))
        lens.copy_(_i32([i, 7, cap, 1]))
        start = torch.randn(state.shape, generator=torch.Generator().manual_seed(i)).to(BF).cuda()
        state.copy_(start)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        t, p, s, _ = wf.op_beam_select(x, sc, n_in=n_in, n_out=n_out, keep_slots=True)
        want = start.clone()
        wf.op_beam_reorder(want, p, lens=lens)
        assert torch.equal(tok, t) and torch.equal(par, p) and torch.equal(score, s) and torch.equal(state, want), i


@pytest.mark.parametrize("low", [-7e4, -1e9, -1e10, -3e15, -1e30, -3e38])
@pytest.mark.parametrize("dtype", [F32, BF], ids=str)
def test_logits_suppressed_by_a_large_finite_number(dtype, low):
    # whole parts of a row, and whole rows, at a mask's value: the other tokens' totals do not feel it
    x = _logits(1, 4, 9000, 21, dtype)
    x[0, 0, 2048:] = low
    x[0, 1, :8000] = low
    x[0, 2, 5:] = low
    x[0, 3, 4096:6144] = low * torch.linspace(1.0, 1.1, 2048).to(dtype).cuda()
    tok, _ = _check_select(x, _scores(1, 4, 21))
    assert (tok >= 0).all()


@pytest.mark.parametrize("size", [6.5e4, 7e4, 1e7, 1e9, 1e10, 3.3e15, 1e25, 1.2e30, 1.3e30])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("dtype", [F32, BF], ids=str)
def test_rows_of_large_equal_logits(dtype, sign, size):
    # each of V tokens at the same value x: log sum = x + log V, of which 64 bits keep |x| 2^-53, at the oracle's end and at the kernel's
    B, W, V = 1, 3, 4500
    x = torch.full((B, W, V), sign * size, device="cuda").to(dtype)
    x[0, 1, 77:] = x[0, 1, 0] * (1 - sign * 2.0 ** -5)              # 77 tokens, all others far below
    x[0, 2, 1:] = x[0, 2, 0] * (1 - sign * 2.0 ** -5)
    sc = torch.full((B, W), -2.0, device="cuda")
    tok, par, out, _ = wf.op_beam_select(x, sc)
    xd = x.double().cpu().numpy()
    rt, rp, rs, _ = D.beam_step(xd[0], np.full(W, -2.0), W, W)
    assert np.isfinite(rs).all()
    got = out[0].double().cpu().numpy()
    # 2^-19 as stated, half a step of fp32, and 3 roundings of 64 bits of something of the logits' size on either side
    assert (np.abs(got - rs) <= 2.0 ** -19 + 2.0 ** -24 * np.abs(rs) + 6 * 2.0 ** -53 * np.abs(xd).max()).all()
    if size < 1e9:                                                  # there, log 77 and log 4500 are told apart
        assert tok[0].tolist() == rt.tolist() and par[0].tolist() == rp.tolist() == [2, 1, 1]


@pytest.mark.parametrize("V", [300, 5001, 51866])
@pytest.mark.parametrize("dtype", [F32, BF], ids=str)
def test_beams_whose_rows_are_permutations_of_each_other(dtype, V):
    # their log sums are equal, the kernel's within 2^-18 of each other: nearer totals come in any order, others in their own
    W = 6
    g = torch.Generator().manual_seed(V)
    row = torch.randn(V, generator=g) * 2.5
    row[7] = row.max() + 2.0                                    # each beam's first candidate is ahead of every second one
    x = torch.stack([row[torch.randperm(V, generator=g)] for _ in range(W)])[None].to(dtype).cuda()
    best = x[0].float().argmax(1).tolist()
    xd = x[0].double().cpu().numpy()
    lse = np.log(np.exp(xd[0] - xd[0].max()).sum()) + xd[0].max()
    gap = np.sort(xd[0])[-1] - np.sort(xd[0])[-2]
    assert gap > 1.0

    def select(scores):
        tok, par, out, _ = wf.op_beam_select(x, torch.tensor([scores], dtype=torch.float32, device="cuda"))
        return tok[0].tolist(), par[0].tolist(), out[0].double().cpu().numpy()

    tok, par, out = select([-1.0] * W)
    assert sorted(par) == list(range(W)) and tok == [best[p] for p in par]
    total = -1.0 + xd[0].max() - lse
    assert (np.abs(out - total) <= 2.0 ** -19 + 2.0 ** -24 * abs(total)).all()
    order = [4, 0, 5, 2, 1, 3]
    scores = [0.0] * W
    for i, b in enumerate(order):
        scores[b] = -1.0 - i * 2.0 ** -17
    tok, par, _ = select(scores)
    assert par == order and tok == [best[b] for b in order]
