"""The radial network's hidden layers on the GPU (linear layer, layer norm) against float64, at the sizes and with the options
where they can go wrong.  The bounds are those of layer_util.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import layer_util as ref
import paper_2609_35099_b200 as e3j

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def half(dtype):
    return torch.finfo(dtype).eps / 2


def draw(seed, dtype, *shapes, scale=None):
    """Tensors of that type on the GPU and their values in float64."""
    rng = np.random.default_rng(seed)
    out = []
    for k, shape in enumerate(shapes):
        if shape is None:
            out.append((None, None))
            continue
        a = rng.standard_normal(shape) * (1.0 if scale is None else scale[k])
        t = torch.from_numpy(a).to(dtype)
        out.append((t.cuda(), t.double().numpy()))
    return out


# rows, n_in, n_out: one row, one column, tiles' borders and their neighbours, several tiles and chunks, odd widths
LINEAR = [(1, 1, 1), (1, 64, 64), (2, 8, 64), (127, 16, 24), (128, 64, 64), (129, 65, 63), (300, 97, 161), (1000, 3, 130),
          (77, 200, 7), (513, 128, 128), (260, 64, 129), (2500, 33, 66), (40, 512, 300), (700, 321, 64), (650, 68, 36)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,n_in,n_out", LINEAR)
def test_linear_forward(rows, n_in, n_out, dtype):
    options = [("none", False, False), ("silu", True, False), ("tanh", True, True), ("gelu", False, True)]
    (x, x_), (W, W_), (b, b_), (r, r_) = draw(rows + n_in, dtype, (rows, n_in), (n_in, n_out), (n_out,), (rows, n_out),
                                               scale=(1, n_in ** -0.5, 0.5, 1))
    for act, bias, residual in options:
        y = torch.full((rows, n_out), float("nan"), dtype=dtype, device="cuda")
        e3j.e3j_linear_fwd(x, W, b if bias else None, r if residual else None, ref.ACTS[act], out=y)
        want, bound = ref.linear_fwd(x_, W_, b_ if bias else None, r_ if residual else None, act, half(dtype))
        ref.assert_within(y, want, bound, act)
        assert torch.equal(y, e3j.e3j_linear_fwd(x, W, b if bias else None, r if residual else None, ref.ACTS[act]))
    assert e3j.e3j_linear_status() == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,n_in,n_out", LINEAR + [(20000, 64, 64), (9000, 40, 96)])
def test_linear_backward(rows, n_in, n_out, dtype):
    (x, x_), (W, W_), (b, b_), (g, g_) = draw(rows + n_in, dtype, (rows, n_in), (n_in, n_out), (n_out,), (rows, n_out),
                                               scale=(1, n_in ** -0.5, 0.5, 1))
    for act, bias in [("none", True), ("silu", True), ("tanh", False), ("gelu", True)]:
        got = e3j.e3j_linear_bwd(x, W, b if bias else None, g, ref.ACTS[act])
        want, bounds = ref.linear_bwd(x_, W_, b_ if bias else None, g_, act, half(dtype))
        for t, v, e, what in zip(got, want, bounds, ("grad_x", "grad_W", "grad_b")):
            ref.assert_within(t, v, e, f"{act} {what}")
        again = e3j.e3j_linear_bwd(x, W, b if bias else None, g, ref.ACTS[act])
        assert all(torch.equal(p, q) for p, q in zip(got, again))
    assert e3j.e3j_linear_status() == 0


NORM = [(1, 1), (1, 64), (3, 2), (33, 8), (129, 64), (500, 96), (70, 97), (41, 385), (300, 512), (25, 1000), (17, 1024), (9, 1025),
        (5, 4096), (6, 4095), (2000, 16), (1000, 130), (12, 2050)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,n", NORM)
def test_norm_forward(rows, n, dtype):
    (x, x_), (w, w_), (c, c_) = draw(rows + n, dtype, (rows, n), (n,), (n,), scale=(1.5, 1, 0.5))
    for act, weight, bias, eps in [("none", True, True, 1e-5), ("silu", True, False, 1e-5), ("tanh", False, True, 1e-2), ("gelu", False, False, 1e-5)]:
        y = torch.full((rows, n), float("nan"), dtype=dtype, device="cuda")
        e3j.e3j_layer_norm_fwd(x, w if weight else None, c if bias else None, eps, ref.ACTS[act], out=y)
        want, bound = ref.norm_fwd(x_, w_ if weight else np.ones(n), c_ if bias else np.zeros(n), eps, act, half(dtype))
        ref.assert_within(y, want, bound, act)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,n", NORM + [(30000, 64), (20000, 9)])
def test_norm_backward(rows, n, dtype):
    (x, x_), (w, w_), (c, c_), (g, g_) = draw(rows + n, dtype, (rows, n), (n,), (n,), (rows, n), scale=(1.5, 1, 0.5, 1))
    for act, weight, bias in [("none", True, True), ("silu", True, False), ("tanh", False, True), ("gelu", False, False)]:
        got = e3j.e3j_layer_norm_bwd(x, w if weight else None, c if bias else None, g, 1e-5, ref.ACTS[act])
        want, bounds = ref.norm_bwd(x_, w_ if weight else np.ones(n), c_ if bias else np.zeros(n), g_, 1e-5, act, half(dtype))
        for t, v, e, what in zip(got, want, bounds, ("grad_x", "grad_weight", "grad_bias")):
            ref.assert_within(t, v, e, f"{act} {what}")
        again = e3j.e3j_layer_norm_bwd(x, w if weight else None, c if bias else None, g, 1e-5, ref.ACTS[act])
        assert all(torch.equal(p, q) for p, q in zip(got, again))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n_in,n_out", [(64, 64), (33, 129), (130, 40)])
@pytest.mark.parametrize("real", [0, 1, 128, 200, 389, -3, 1000])
def test_padded_rows(real, n_in, n_out, dtype):
    rows, kept = 389, min(max(real, 0), 389)
    (x, x_), (W, W_), (b, b_), (r, r_) = draw(real + n_in, dtype, (rows, n_in), (n_in, n_out), (n_out,), (rows, n_out),
                                               scale=(1, n_in ** -0.5, 0.5, 1))
    (w, w_), (c, c_) = draw(5, dtype, (n_in,), (n_in,))
    (gn, gn_),  = draw(6, dtype, (rows, n_in))
    for t in (x, r, gn):
        t[kept:] = float("nan")
    count = torch.tensor([7, real], dtype=torch.int32, device="cuda")[1:]
    nan = lambda *shape: torch.full(shape, float("nan"), dtype=dtype, device="cuda")
    x_, r_, gn_ = x_[:kept], r_[:kept], gn_[:kept]

    def check(t, want, bound, what):
        ref.assert_within(t[:kept], want, bound, what)
        assert (t[kept:] == 0).all(), what

    y = e3j.e3j_linear_fwd(x, W, b, r, 1, n_real=count, out=nan(rows, n_out))
    check(y, *ref.linear_fwd(x_, W_, b_, r_, "silu", half(dtype)), "y")
    for act in ("silu", "none"):
        got = e3j.e3j_linear_bwd(x, W, b, r, ref.ACTS[act], n_real=count, grad_x=nan(rows, n_in), grad_W=nan(n_in, n_out), grad_b=nan(n_out))
        want, bounds = ref.linear_bwd(x_, W_, b_, r_, act, half(dtype))
        check(got[0], want[0], bounds[0], "grad_x")
        ref.assert_within(got[1], want[1], bounds[1], "grad_W")
        ref.assert_within(got[2], want[2], bounds[2], "grad_b")
    y = e3j.e3j_layer_norm_fwd(x, w, c, act=3, n_real=count, out=nan(rows, n_in))
    check(y, *ref.norm_fwd(x_, w_, c_, 1e-5, "gelu", half(dtype)), "norm")
    got = e3j.e3j_layer_norm_bwd(x, w, c, gn, act=3, n_real=count, grad_x=nan(rows, n_in))
    want, bounds = ref.norm_bwd(x_, w_, c_, gn_, 1e-5, "gelu", half(dtype))
    check(got[0], want[0], bounds[0], "norm grad_x")
    ref.assert_within(got[1], want[1], bounds[1], "grad_weight")
    ref.assert_within(got[2], want[2], bounds[2], "grad_bias")


def test_no_rows():
    W, b = torch.ones(5, 7, device="cuda"), torch.ones(7, device="cuda")
    x, g = torch.empty(0, 5, device="cuda"), torch.empty(0, 7, device="cuda")
    assert e3j.e3j_linear_fwd(x, W, b).shape == (0, 7)
    gx, gW, gb = e3j.e3j_linear_bwd(x, W, b, g, 1)
    assert gx.shape == (0, 5) and gW.shape == (5, 7) and (gW == 0).all() and gb.shape == (7,) and (gb == 0).all()
    assert e3j.e3j_layer_norm_fwd(x).shape == (0, 5)
    gx, gw, gc = e3j.e3j_layer_norm_bwd(x, None, None, x)
    assert gx.shape == (0, 5) and (gw == 0).all() and (gc == 0).all() and gw.shape == (5,)
