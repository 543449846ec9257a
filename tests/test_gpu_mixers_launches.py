"""Rotary positions of tokens that several workgroups share, and the recurrence in both orders of its workgroups, element by element against the fp64
statements; tolerances as in test_gpu_mixers.py."""
import numpy as np
import pytest
import torch

from oracle import mixers as om
from paper_2006_09503_amd import binding as B
from paper_2006_09503_amd.synth import round_to_bf16

from gpu_util import to_dev, to_host

pytestmark = pytest.mark.gpu

F32, BF16 = 0, 1
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


def near(got, want, bound, dtype, what):
    over = np.abs(got.astype(np.float64).reshape(want.shape) - want) - (bound + HALF[dtype] * np.abs(want) * 1.01 + 1e-30)
    assert np.isfinite(got).all() and over.max() <= 0, (what, np.unravel_index(over.argmax(), over.shape), over.max())


# tokens, heads, head size, sections, pairing.  A workgroup has 768 vectors, 256 where both halves are 16 bytes wide in bf16; a token's are 2 heads times
# pairs over the pairs of a vector (4 | 8 elements of either half, half of that for neighbours, less where the pairs' places ask for it)
ROTARY = [(33, 64, 128, (16, 24, 24), 0), (5, 33, 128, (64,), 0), (7, 48, 128, (64,), 0), (9, 96, 64, (8, 12, 12), 0), (3, 65, 120, (30, 15, 14), 0),
          (3, 64, 128, (22, 21, 20), 0), (4, 48, 128, (64,), 1), (2, 200, 128, (16, 24, 24), 1), (2, 100, 40, (7, 6, 6), 0), (2, 500, 8, (2, 1), 0)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("case", ROTARY, ids=str)
def test_rotary_of_many_heads(case, dtype):
    tokens, heads, dh, sections, pairing = case
    n, rng = sum(sections), np.random.default_rng(heads + dh)
    axis, freq = np.repeat(np.arange(len(sections), dtype=np.uint8), sections), 1e4 ** (-np.arange(n) / n)
    x = rng.standard_normal((tokens, 3 * heads * dh)).astype(np.float32)
    x = round_to_bf16(x) if dtype == BF16 else x
    pos = rng.integers(-100000, 100000, (len(sections), tokens)).astype(np.int32)
    P = torch.from_numpy(pos).cuda()
    i = np.arange(n) if pairing == 0 else 2 * np.arange(n)
    j = i + (n if pairing == 0 else 1)
    size = np.zeros((tokens, 3 * heads * dh))
    for head in range(2 * heads):
        size[:, head * dh + i] = size[:, head * dh + j] = np.abs(x[:, head * dh + i]) + np.abs(x[:, head * dh + j])
    for inverse in (0, 1):
        X = to_dev(x, dtype)
        B.check(B.lib().k2bw_rotary(dtype, 1, tokens, heads, dh, n, pairing, axis.ctypes.data, freq.ctypes.data, len(sections), P.data_ptr(), inverse,
                                    X.data_ptr(), None), "rotary")
        got = to_host(X)
        near(got, om.rotary(x, heads, dh, axis, freq, pos, pairing, bool(inverse)), 4e-7 * size, dtype, (case, inverse))
        assert np.array_equal(got[size == 0], x[size == 0])


# b, s, h, lengths: more than 16 chains of whole lines (one group of channels after the other), lines that groups share, few chains
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("case", [(3, 700, 1024, [700, 129, 0]), (2, 1300, 2048, None), (17, 200, 64, [200, 64, 65] * 5 + [1, 199]), (3, 700, 1032, [1, 650, 700]),
                                  (1, 1100, 512, None)], ids=str)
def test_recurrence_in_both_orders_of_workgroups(case, dtype):
    b, s, h, lens = case
    rng, L, eps = np.random.default_rng(s + h), B.lib(), 1e-6 if dtype == F32 else 2e-6
    gates = rng.standard_normal((b, s, 3, h))
    gates[:, :, 0] = np.clip(gates[:, :, 0] * 2 + rng.uniform(-2, 6, h), -12, 12)
    gates, d_o = gates.astype(np.float32), rng.standard_normal((b, s, h)).astype(np.float32)
    if dtype == BF16:
        gates, d_o = round_to_bf16(gates), round_to_bf16(d_o)
    state, dstate = rng.standard_normal((2, b, h)).astype(np.float32)
    tdt, p = torch.bfloat16 if dtype == BF16 else torch.float32, lambda t: None if t is None else t.data_ptr()
    nan = lambda *shape, d=torch.float32: torch.full(shape, float("nan"), device="cuda", dtype=d)   # noqa: E731
    G, D, S, dS = to_dev(gates, dtype), to_dev(d_o, dtype), torch.from_numpy(state).cuda(), torch.from_numpy(dstate).cuda()
    n = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    if lens is not None:
        for i, k in enumerate(lens):
            G[i, k:], D[i, k:] = float("nan"), float("inf")
    saved, ws = nan(L.k2bw_recurrence_saved(b, s, h)), nan(L.k2bw_recurrence_workspace(b, s, h))
    o, out, dg, db, dsi = nan(b, s, h, d=tdt), nan(b, h), nan(b, s, 3, h, d=tdt), nan(3 * h), nan(b, h)
    B.check(L.k2bw_recurrence_fwd(dtype, b, s, h, p(n), p(G), p(S), p(out), p(o), p(saved), p(ws), None), "fwd")
    B.check(L.k2bw_recurrence_bwd(dtype, b, s, h, p(n), p(G), p(saved), p(D), p(dS), p(dsi), p(dg), p(db), 0, p(ws), None), "bwd")
    want_o, H, tol_o, tol_h = om.recurrence_fwd(gates, b, s, h, lens, state, eps)
    want_g, want_s, tol_g, tol_s = om.recurrence_bwd(gates, d_o, b, s, h, lens, state, dstate, eps)
    near(to_host(o), want_o, tol_o, dtype, "o")
    near(to_host(out), H[:, -1], tol_h[:, -1], F32, "state_out")
    near(to_host(dg), want_g, tol_g, dtype, "dgates")
    near(to_host(dsi), want_s, tol_s, F32, "dstate_in")
    tol = tol_g.sum((0, 1)).reshape(-1) + (48 + b * s / 64) * 2.0 ** -24 * np.abs(want_g).sum((0, 1)).reshape(-1)
    near(to_host(db), want_g.sum((0, 1)).reshape(-1), tol, F32, "dbias")
