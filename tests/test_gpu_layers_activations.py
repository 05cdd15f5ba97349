"""Activations of the hidden layers on the GPU: infinite arguments, and how exact GELU is in float32."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2609_35099_b200 as e3j

pytestmark = pytest.mark.gpu
SILU, TANH, GELU = e3j.E3J_ACT_SILU, e3j.E3J_ACT_TANH, e3j.E3J_ACT_GELU
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("act,low,high", [(0, -INF, INF), (SILU, NAN, INF), (TANH, -1.0, 1.0), (GELU, 0.0, INF)])
def test_infinite_arguments(act, low, high, dtype):
    """z = infinity by way of the bias: what the header says (silu of -infinity is -infinity / infinity)."""
    want = torch.tensor([high, low, NAN], device="cuda")
    for n in (3, 64, 200):
        b = torch.zeros(n, dtype=dtype, device="cuda")
        b[:3] = torch.tensor([INF, -INF, NAN], device="cuda")
        x, W = torch.randn(300, 16, device="cuda").to(dtype), torch.randn(16, n, device="cuda").to(dtype)
        for y in (e3j.e3j_linear_fwd(x, W, b, act=act), e3j.e3j_layer_norm_fwd(torch.randn(300, n, device="cuda").to(dtype), None, b, act=act)):
            assert torch.equal(y[:, :3].float().nan_to_num(nan=7.0), want.expand(300, 3).nan_to_num(nan=7.0)), (n, y[0, :3])
            assert torch.isfinite(y[:, 3:].float()).all()


U = 2.0 ** -24


def arguments():
    """float32 from everyday sizes to the ends of where GELU is neither 0 nor z, both signs; a multiple of 64 of them."""
    rng = np.random.default_rng(1)
    z = np.concatenate([rng.standard_normal(20000), 0.1 * rng.standard_normal(20000), 1e-3 * rng.standard_normal(4000), np.linspace(-12.5, 12.5, 50000),
                        1.5 + 1e-4 * rng.standard_normal(500), -1.5 + 1e-4 * rng.standard_normal(500), [0.0, -0.0, 1e-30, -1e-30, 1e-20]])
    return np.resize(z, (-(-z.size // 64) * 64,)).astype(np.float32)


def parts(z):
    """|Phi(z) - 1/2|, Phi(-|z|) and the density, in float64."""
    from scipy.special import ndtr
    return np.abs(0.5 - ndtr(-np.abs(z))), ndtr(-np.abs(z)), np.exp(-z * z / 2) / np.sqrt(2 * np.pi)


def through(t, kind):
    """GELU, or its slope, of each element: layers that hand their input on unchanged (a product with one is exact)."""
    x, one = t.view(-1, 64), torch.eye(64, device="cuda")
    if kind == "forward":
        return e3j.e3j_linear_fwd(x, one, act=GELU)
    if kind == "slope, up to 64 columns":
        return e3j.e3j_linear_bwd(x, one, None, torch.ones_like(x), GELU, grad_W=False, grad_b=False)[0]
    x, one = t.view(-1, 128), torch.eye(128, device="cuda")
    return e3j.e3j_linear_bwd(x, one, None, torch.ones_like(x), GELU, grad_W=False, grad_b=False)[0]


@pytest.mark.parametrize("kind", ["forward", "slope, up to 64 columns", "slope"])
def test_gelu_in_float32(kind):
    """Element by element.  u = 2^-24 is half a step of float32.  Within 1.5 of 0, Phi - 1/2 is z times a polynomial in z^2: z^2, the product and
    the polynomial (whose terms are up to 2.1 times its sum, two roundings each of the first few) lose below 8 u of it.
    Elsewhere Phi(-|z|) = e t P(t): the argument z^2 / 2 of e loses 3 u of itself (square, product, constant), so e loses 1.5 z^2 u and
    two steps (4 u), t an addition and a step (3 u), the polynomial 6 u, the two products 2 u, the fit 1 u: (1.5 z^2 + 16) u.  The density
    loses (1.5 z^2 + 4 + 2) u.  Each sum of parts and the result are rounded: u of their magnitudes.  A small absolute part stands for what is
    below the normal range."""
    z = arguments()
    z = np.resize(z, (z.size // 128 * 128,))
    got = through(torch.from_numpy(z).cuda(), kind).double().cpu().numpy().reshape(-1)
    z = z.astype(np.float64)
    middle, tail, density = parts(z)
    inner = np.abs(z) < 1.5
    near = np.abs(np.abs(z) - 1.5) < 1e-6
    e_Phi = np.where(inner & ~near, 8 * U * middle, (1.5 * z * z + 16) * U * tail + 8 * U * middle * near)
    Phi = np.where(z > 0, 0.5 + middle, tail)
    if kind == "forward":
        want = z * Phi
        bound = np.abs(z) * e_Phi + U * np.abs(want) * 1.01
    else:
        want = Phi + z * density
        bound = e_Phi + (1.5 * z * z + 6) * U * np.abs(z) * density + 2 * U * (Phi + np.abs(z) * density)
    over = np.abs(got - want) - (bound + 1e-37)
    i = int(np.argmax(over))
    assert over[i] <= 0, (z[i], got[i], want[i], abs(got[i] - want[i]) / U, bound[i] / U)


def test_gelu_is_as_exact_as_the_elementary_form():
    """2-norm over normal values of three sizes.  Rounding the result alone is a uniform error of up to half a step: between u / 2 and u of
    the value at most, 0.4 u = 2.4e-8 in the mean square; the factor Phi takes two or three such roundings beside it: sqrt(4) * 0.4 u < u."""
    for scale in (1.0, 0.1, 3.0):
        x = torch.randn(60000, 64, device="cuda") * scale
        x64 = x.double()
        want = x64 * 0.5 * torch.erfc(-x64 / 2 ** 0.5)
        y = e3j.e3j_linear_fwd(x, torch.eye(64, device="cuda"), act=GELU)
        assert (y.double() - want).norm() <= U * want.norm(), scale


@pytest.mark.parametrize("n_in,n_out", [(64, 64), (33, 130), (512, 200)])
def test_an_infinity_in_x(n_in, n_out):
    """bfloat16: infinities with the signs of W's row; float32, whose values are cut into terms: NaN.  The other rows as without it."""
    for dtype in (torch.float32, torch.bfloat16):
        x, W = torch.randn(300, n_in, device="cuda").to(dtype), (torch.rand(n_in, n_out, device="cuda") - 0.5).to(dtype)
        W[5] = torch.where(W[5] == 0, torch.ones_like(W[5]), W[5])
        want = e3j.e3j_linear_fwd(x, W)
        x[7, 5], x[200, 5] = INF, -INF
        y = e3j.e3j_linear_fwd(x, W)
        rest = torch.ones(300, dtype=torch.bool, device="cuda")
        rest[[7, 200]] = False
        assert torch.equal(y[rest], want[rest])
        if dtype == torch.bfloat16:
            assert torch.equal(y[7].float(), torch.sign(W[5].float()) * INF) and torch.equal(y[200], -y[7])
        else:
            assert torch.isnan(y[[7, 200]]).all()
