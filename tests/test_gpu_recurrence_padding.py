"""The recurrence's bias gradient is the column sums of dgates, which are zero behind a sequence's real tokens, whatever its carried states hold."""
import numpy as np
import pytest
import torch

from oracle import mixers as om
from paper_2006_09503_amd import binding as B
from paper_2006_09503_amd.synth import round_to_bf16

from gpu_util import to_dev, to_host

pytestmark = pytest.mark.gpu

F32, BF16 = 0, 1


def backward(dtype, b, s, h, lens, gates, d_o, state, dstate):
    """(dgates, bias gradient, gradient of the first state) of one pass there and back."""
    L, p = B.lib(), lambda t: t.data_ptr()   # noqa: E731
    tdt = torch.bfloat16 if dtype == BF16 else torch.float32
    nan = lambda *shape, d=torch.float32: torch.full(shape, float("nan"), device="cuda", dtype=d)   # noqa: E731
    G, D, S, dS = to_dev(gates, dtype), to_dev(d_o, dtype), torch.from_numpy(state).cuda(), torch.from_numpy(dstate).cuda()
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    saved, ws = nan(L.k2bw_recurrence_saved(b, s, h)), nan(L.k2bw_recurrence_workspace(b, s, h))
    o, out, dg, db, dsi = nan(b, s, h, d=tdt), nan(b, h), nan(b, s, 3, h, d=tdt), nan(3 * h), nan(b, h)
    B.check(L.k2bw_recurrence_fwd(dtype, b, s, h, p(n), p(G), p(S), p(out), p(o), p(saved), p(ws), None), "fwd")
    B.check(L.k2bw_recurrence_bwd(dtype, b, s, h, p(n), p(G), p(saved), p(D), p(dS), p(dsi), p(dg), p(db), 0, p(ws), None), "bwd")
    torch.cuda.synchronize()
    return to_host(dg), to_host(db), to_host(dsi)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 3e38])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("s", [1, 50, 300])
def test_states_of_a_sequence_without_tokens_stay_out_of_the_bias_gradient(s, dtype, bad):
    """The same bits as with states of zero there, and the real sequence's own sums.  Its tolerance: the oracle's bound and, for each of at most
    48 + s / 64 additions in a row, a rounding of the running sum."""
    b, h = 2, 72
    rng = np.random.default_rng(s)
    gates, d_o = rng.standard_normal((b, s, 3, h)).astype(np.float32), rng.standard_normal((b, s, h)).astype(np.float32)
    if dtype == BF16:
        gates, d_o = round_to_bf16(gates), round_to_bf16(d_o)
    state, dstate = rng.standard_normal((2, b, h)).astype(np.float32)
    state[0] = dstate[0] = 0.0
    clean = backward(dtype, b, s, h, [0, s], gates, d_o, state, dstate)
    state[0], dstate[0] = bad, bad
    dg, db, dsi = backward(dtype, b, s, h, [0, s], gates, d_o, state, dstate)
    assert np.all(dg[0] == 0) and np.array_equal(dg, clean[0]) and np.array_equal(dsi[1], clean[2][1])
    assert np.array_equal(dsi[0], np.full(h, bad, dtype=np.float32), equal_nan=True)
    assert np.array_equal(db, clean[1])
    want, _, bound, _ = om.recurrence_bwd(gates[1:], d_o[1:], 1, s, h, None, state[1:], dstate[1:], 1e-6 if dtype == F32 else 2e-6)
    size = np.abs(want).sum((0, 1)).reshape(-1)
    tol = bound.sum((0, 1)).reshape(-1) + (48 + s / 64) * 2.0 ** -24 * size + 1e-30
    assert np.all(np.abs(db - want.sum((0, 1)).reshape(-1)) <= tol)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_behind_an_infinite_state_stay_out_of_the_bias_gradient(dtype):
    """A sequence that ends inside a tile with an infinite state: the sums are its real rows' (infinities of one sign, and what is finite), where rows
    behind would add infinity times zero."""
    b, s, h = 1, 100, 8
    gates, d_o = np.zeros((b, s, 3, h), dtype=np.float32), np.ones((b, s, h), dtype=np.float32)
    gates[:, 59, 1] = np.inf         # the last real token's new value
    gates[:, :, 2] = 1.0
    state, dstate = np.zeros((b, h), dtype=np.float32), np.ones((b, h), dtype=np.float32)
    dg, db, _ = backward(dtype, b, s, h, [60], gates, d_o, state, dstate)
    assert np.all(dg[0, 60:] == 0)
    assert np.all(dg[0, 59, 0] == -np.inf) and np.all(dg[0, 59, 2] == np.inf)   # g (h_58 - C) and dO h
    assert np.all(db[:h] == -np.inf) and np.all(db[2 * h:] == np.inf)
    # g_t = r + g_(t+1) / 2 from 1 + r at the last token, r = sigmoid(1); dC_t = g_t / 2.  60 terms in fp32
    r, g, want = 1 / (1 + np.exp(-1.0)), 2.0, 0.0
    for _ in range(60):
        g = r + g / 2
        want += g / 2
    assert np.all(np.abs(db[h:2 * h] - want) <= 64 * 2.0 ** -23 * want)
