"""The optimizer step and the orthogonalisation where every product is a launch: last products in every tile shape, wide and tall, in rows of gaps, in place
and apart; other layouts out than in; zeros, infinities, NaN and extreme sizes beside good matrices.

Tolerances as in test_gpu_muon.py: 16-bit operands 1.25 times what the model of their roundings is off by, plus a bf16 result's rounding; fp32 1.2e-5.
Weights: the roundings of their product and sum, and the update's own error on its part; the momentum: three roundings."""
import numpy as np
import pytest
import torch

from oracle import muon as om
from paper_2006_09503_amd import binding as B

from test_gpu_orth_accuracy import model_of_16_bits, steps_of

pytestmark = pytest.mark.gpu

F32, BF16 = 0, 1
COEF = [float(np.float32(v)) for v in om.QUINTIC] * 5
f = lambda v: float(np.float32(v))   # noqa: E731  what the C floats hold


def gradient(g, rows, cols):
    r = max(1, min(rows, cols) // 16)
    a, b = (torch.randn(s, generator=g, device="cuda") for s in ((rows, r), (r, cols)))
    return (torch.mm(a, b) / r ** 0.5 + torch.randn((rows, cols), generator=g, device="cuda")) * 1e-3


def workspace(dtype, count, rows, cols):
    return torch.full((B.lib().k2bw_orthogonalize_workspace(dtype, count, rows, cols),), float("nan"), device="cuda")


def tolerance(dtype, u, want):
    return 1.2e-5 if dtype == F32 else 1.25 * float((model_of_16_bits(u, 5, COEF) - want).norm() / want.norm())


# count, rows, cols: the last product's tiles are, at 256 CUs, 64x64 (twice; the first of rows that one launch nearly holds), 128x128, 128x256, 192x256,
# 256x256; sizes whose first two steps share a pass over X among them, each wide and tall and with ragged edges
STEPS = [(2, 199, 264), (1, 130, 72), (6, 463, 464), (6, 470, 464), (2, 351, 1376), (1, 1376, 744), (12, 405, 648), (6, 1285, 408), (6, 407, 1288), (12, 1287, 408),
         (10, 407, 1608), (10, 959, 800), (10, 967, 1160), (10, 1157, 968), (5, 2117, 968)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("case", STEPS, ids=str)
def test_muon_in_every_tile_shape(case, dtype):
    count, rows, cols = case
    g = torch.Generator(device="cuda").manual_seed(sum(case))
    ld, nesterov = count * cols + 24, count % 2
    rnd = lambda scale: torch.randn((rows, ld), generator=g, device="cuda") * scale   # noqa: E731
    w, m, G = rnd(0.02), rnd(1e-3), rnd(8e-3)
    for i in (0, count - 1):
        G[:, i * cols:(i + 1) * cols] += 8 * gradient(g, rows, cols)
    lr, beta, decay, scale, micro = 0.01, 0.95, 0.1, 0.2 * max(rows, cols) ** 0.5, 8
    out, lp = torch.full((rows, ld), 7.0, device="cuda"), torch.full((rows, ld), 7.0, device="cuda", dtype=torch.bfloat16)
    M, ws, L = m.clone(), workspace(dtype, count, rows, cols), B.lib()

    def step(w_cur, w_next, copy, m):
        B.check(L.k2bw_muon(dtype, count, rows, cols, ld, cols, w_cur.data_ptr(), w_next.data_ptr(), None if copy is None else copy.data_ptr(), m.data_ptr(),
                            G.data_ptr(), lr, beta, decay, scale, nesterov, micro, 5, None, ws.data_ptr(), None), "muon")
    step(w, out, lp, M)
    for i in sorted({0, count // 2, count - 1}):
        c = slice(i * cols, (i + 1) * cols)
        grad = G[:, c].double() / micro
        m2 = f(beta) * m[:, c].double() + (1 - f(beta)) * grad
        u = f(beta) * m2 + (1 - f(beta)) * grad if nesterov else m2
        o = steps_of(u, 5, COEF, torch.float64)
        w2 = w[:, c].double() * (1 - f(lr) * f(decay)) - f(lr) * f(scale) * o
        assert float((M[:, c].double() - m2).norm() / m2.norm()) < 3 * 2.0 ** -24
        off = float((out[:, c].double() - w2).norm())
        tol = 3 * 2.0 ** -24 * float(w2.norm()) + f(lr) * f(scale) * tolerance(dtype, u, o) * float(o.norm())
        print(f"matrix {i}: off by {off:.3e}, tolerance {tol:.3e}")
        assert off < tol, (i, off, tol)
    used = count * cols
    assert torch.equal(lp[:, :used], out[:, :used].bfloat16())
    assert (out[:, used:] == 7).all() and (lp[:, used:] == 7).all() and torch.equal(M[:, used:], m[:, used:])
    # in place, and without the copy
    W2, M2 = w.clone(), m.clone()
    step(W2, W2, None, M2)
    assert torch.equal(W2[:, :used], out[:, :used]) and torch.equal(M2, M) and torch.equal(W2[:, used:], w[:, used:])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("case", [(3, 24, 40), (3, 199, 264), (2, 264, 200), (6, 463, 464), (6, 1285, 408), (12, 407, 648)], ids=str)
def test_orthogonalize_from_one_layout_to_another(case, dtype):
    """Side by side in wider rows, to stacked with gaps, and back: the same bits as from and to matrices of their own, and gaps that stay."""
    count, rows, cols = case
    g = torch.Generator(device="cuda").manual_seed(sum(case))
    tdt, L = torch.bfloat16 if dtype == BF16 else torch.float32, B.lib()
    x = torch.stack([gradient(g, rows, cols) for _ in range(count)]).to(tdt)
    ws = workspace(dtype, count, rows, cols)

    def call(a, ld, stride, to, ld_to, stride_to):
        B.check(L.k2bw_orthogonalize(dtype, count, rows, cols, a.data_ptr(), ld, stride, to.data_ptr(), ld_to, stride_to, 5, None, ws.data_ptr(), None), "orthogonalize")
    want = torch.empty_like(x)
    call(x, cols, rows * cols, want, cols, rows * cols)
    full = x.double()
    for i in (0, count - 1):
        o = steps_of(full[i], 5, COEF, torch.float64)
        r = float((want[i].double() - o).norm() / o.norm())
        assert r < tolerance(dtype, full[i], o) + (2.0 ** -24 if dtype == F32 else 2.0 ** -8 / (3 ** 0.5 if rows * cols >= 4096 else 1.0)), (i, r)
    beside = torch.full((rows, count * cols + 40), 5.0, device="cuda", dtype=tdt)
    beside[:, :count * cols] = x.permute(1, 0, 2).reshape(rows, count * cols)
    stacked = torch.full((count, rows + 3, cols + 16), 7.0, device="cuda", dtype=tdt)
    call(beside, beside.shape[1], cols, stacked, cols + 16, (rows + 3) * (cols + 16))
    assert torch.equal(stacked[:, :rows, :cols], want)
    assert (stacked[:, rows:] == 7).all() and (stacked[:, :, cols:] == 7).all()
    stacked[:, :rows, :cols] = x
    call(stacked, cols + 16, (rows + 3) * (cols + 16), beside, beside.shape[1], cols)
    assert torch.equal(beside[:, :count * cols], want.permute(1, 0, 2).reshape(rows, count * cols)) and (beside[:, count * cols:] == 5).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [(199, 264), (408, 200), (463, 464), (1285, 408), (407, 1288), (744, 2760)], ids=str)
def test_bad_matrices_and_extreme_sizes_beside_good_ones(size, dtype):
    """2^-90 and 2^100 times a matrix (whose squares fp32 does not hold), zeros, a NaN, an infinity; products of 64x64 and of larger tiles, single steps and
    the first two together."""
    g = torch.Generator(device="cuda").manual_seed(sum(size))
    tdt, L = torch.bfloat16 if dtype == BF16 else torch.float32, B.lib()
    u = gradient(g, *size).to(tdt)
    x = torch.stack([u, u * 2.0 ** -90, u * 2.0 ** 100, u * 0, u, u, u])
    x[4, 3, 5], x[5, size[0] - 1, size[1] - 1] = float("nan"), float("inf")
    out = torch.full_like(x, 7.0)
    B.check(L.k2bw_orthogonalize(dtype, 7, *size, x.data_ptr(), size[1], u.numel(), out.data_ptr(), size[1], u.numel(), 5, None,
                                 workspace(dtype, 7, *size).data_ptr(), None), "orthogonalize")
    want = steps_of(u.double(), 5, COEF, torch.float64)
    tol = tolerance(dtype, u.double(), want) + (2.0 ** -24 if dtype == F32 else 2.0 ** -8 / 3 ** 0.5)
    for i in (0, 1, 2, 6):
        r = float((out[i].double() - want).norm() / want.norm())
        assert r < tol, (i, r, tol)
    assert (out[3] == 0).all() and torch.isnan(out[4]).all() and torch.isnan(out[5]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_same_bits_every_time_in_larger_tiles(dtype):
    g = torch.Generator(device="cuda").manual_seed(1)
    x = gradient(g, 1536, 4608).to(torch.bfloat16 if dtype == BF16 else torch.float32)[None]
    outs = []
    for i in range(4):
        out, ws = torch.empty_like(x), workspace(dtype, 1, 1536, 4608)
        ws.fill_(float(i))
        B.check(B.lib().k2bw_orthogonalize(dtype, 1, 1536, 4608, x.data_ptr(), 4608, 0, out.data_ptr(), 4608, 0, 5, None, ws.data_ptr(), None), "orthogonalize")
        outs.append(out)
    assert all(torch.equal(o, outs[0]) for o in outs)
