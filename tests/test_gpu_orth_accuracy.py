"""Steps that the orthogonalisation takes together, on matrices of a small rank and little else (few tokens against a wide layer), of unequal rows and of
coefficients that grow small singular values further than the default's, against 64 bits.

Tolerances.  16-bit operands: what the model of their roundings, one step after the other, is off by on the same input, times 1.25 for the fp32 sums and
what they turn over, plus the result's rounding to bf16 (half a step of 2^-8 spread evenly: 2^-8 / sqrt 3).  fp32: what the same iteration in 32-bit
arithmetic is off by, times 1.75: the first two steps taken together round A_0 once and pass that on through P_1, 1.4 times the iteration's error in
emulation (matrices of 256 to 1024 rows, ranks from 4 to m/2, power laws), and a quarter for another order of the sums."""
import numpy as np
import pytest
import torch

from oracle import muon as om
from paper_2006_09503_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16 = 0, 1


def rel(a, b):
    return float((a.double() - b).norm() / b.norm())


def steps_of(u, steps, coef, dtype, product=torch.mm):
    x = u.to(dtype)
    tall = x.shape[0] > x.shape[1]
    x = x.T.contiguous() if tall else x
    x = x / u.double().norm().to(dtype)
    for i in range(steps):
        a, b, c = coef[3 * i:3 * i + 3]
        s = product(x, x.T.contiguous())
        x = a * x + product(b * s + c * product(s, s), x)
    return x.T.contiguous() if tall else x


def fp16(x, scale):
    return (x * scale).half().double() / scale


def model_of_16_bits(u, steps, coef):
    """oracle/muon.py's model on the device."""
    x = u.double()
    tall = x.shape[0] > x.shape[1]
    x = x.T.contiguous() if tall else x
    x = x / x.norm()
    m = x.shape[0]
    eye = torch.eye(m, device="cuda", dtype=torch.float64)
    for i in range(steps):
        a, b, c = coef[3 * i:3 * i + 3]
        hi = fp16(x, 4096.0)
        x = hi + fp16(x - hi, 4096.0)
        alpha = (x * x).sum() / m
        A = torch.mm(hi, hi.T.contiguous()) - alpha * eye
        t = (A * A).sum() / m
        A = fp16(A, 4096.0)
        P = fp16((b + 2 * c * alpha) * A + c * (torch.mm(A, A) - t * eye), 1024.0)
        x = (a + b * alpha + c * alpha * alpha + c * t) * x + torch.mm(P, hi)
    return x.T.contiguous() if tall else x


def run(dtype, x, steps, coef=None):
    L, (count, rows, cols) = B.lib(), x.shape
    out = torch.full_like(x, float("nan"))
    ws = torch.full((L.k2bw_orthogonalize_workspace(dtype, count, rows, cols),), float("nan"), device="cuda")
    B.check(L.k2bw_orthogonalize(dtype, count, rows, cols, x.data_ptr(), cols, rows * cols, out.data_ptr(), cols, rows * cols, steps,
                                 None if coef is None else coef.ctypes.data, ws.data_ptr(), None), "orthogonalize")
    torch.cuda.synchronize()
    return out


def low_rank(g, rows, cols, rank, noise):
    a, b = (torch.randn(s, generator=g, device="cuda") for s in ((rows, rank), (rank, cols)))
    return torch.mm(a, b) / rank ** 0.5 + noise * torch.randn((rows, cols), generator=g, device="cuda")


def check(dtype, u, steps=5, coef=None):
    full = np.array(om.QUINTIC * steps if coef is None else coef, dtype=np.float32)
    c = [float(v) for v in full]
    got = run(dtype, u[None].contiguous(), steps, None if coef is None else full)[0]
    want = steps_of(u, steps, c, torch.float64)
    off = rel(got, want)
    if dtype == BF16:
        tol = 1.25 * rel(model_of_16_bits(u, steps, c), want) + 2.0 ** -8 / 3 ** 0.5
    else:
        tol = 1.75 * rel(steps_of(u, steps, c, torch.float32), want) + 2.0 ** -24
    print(f"off by {off:.3e}, tolerance {tol:.3e}")
    assert off < tol, (off, tol)


SIZES = [(1024, 4096), (1536, 4608), (4608, 1536), (700, 4200)]


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("part, noise", [(4, 0.01), (16, 0.01), (6, 0.0), (2, 0.0), (16, 1.0)], ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_small_ranks(dtype, part, noise, size):
    g = torch.Generator(device="cuda").manual_seed(sum(size) + part)
    u = low_rank(g, *size, min(size) // part, noise) * 1e-3
    check(dtype, u.bfloat16() if dtype == BF16 else u)


@pytest.mark.parametrize("steps", [2, 3, 4, 6, 7])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_small_ranks_by_numbers_of_steps(dtype, steps):
    g = torch.Generator(device="cuda").manual_seed(steps)
    u = low_rank(g, 700, 4200, 175, 0.01) * 1e-3
    check(dtype, u.bfloat16() if dtype == BF16 else u, steps)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_unequal_size(dtype):
    g = torch.Generator(device="cuda").manual_seed(1)
    u = torch.randn((1024, 4096), generator=g, device="cuda") * torch.logspace(-6, -3, 1024, device="cuda")[:, None]
    check(dtype, u.bfloat16() if dtype == BF16 else u)


# 2.9 T5(s), 2.9 T5(s / 2.9), T5 the Chebyshev polynomial 16 s^5 - 20 s^3 + 5 s: within 2.9 on [0, 1] and on what that gives, and 72.5 times what is
# small; then halves.
STEEP = (14.5, -58.0, 46.4, 5.0, -20.0 / 2.9 ** 2, 16.0 / 2.9 ** 4, 0.5, 0.0, 0.0, 0.5, 0.0, 0.0, 1.5, -0.5, 0.0)


@pytest.mark.parametrize("rows, cols", [(704, 4200), (4200, 704)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_coefficients_whose_product_leaves_fp16(dtype, rows, cols):
    """Few rows are not zero, so what a product of two steps' polynomials has on the diagonal reaches from its mean, 69, to under 0."""
    g = torch.Generator(device="cuda").manual_seed(2)
    u = torch.zeros((704, 4200), device="cuda")
    u[::16] = torch.randn((44, 4200), generator=g, device="cuda")
    u = (u if rows < cols else u.T).contiguous()
    check(dtype, u.bfloat16() if dtype == BF16 else u, 5, STEEP)
