"""The hidden layers as they are used (GPU): in a radial network in front of the convolution, through autograd, on other streams,
in graphs, at once, on views, beyond 2^31 elements; what they refuse."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import layer_util as ref
import paper_2609_35099_b200 as e3j
from oracle import conv as oconv
from paper_2609_35099_b200 import workloads
from paper_2609_35099_b200.autograd import Graph, conv_radial, layer_norm, linear

pytestmark = pytest.mark.gpu
SILU, GELU = e3j.E3J_ACT_SILU, e3j.E3J_ACT_GELU


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def radial_network(rbf, p, lin, norm, silu):
    """rbf -> linear + silu -> linear -> layer norm + silu -> linear + silu with a residual"""
    h1 = lin(rbf, p[0], p[1], None, True)
    h2 = norm(lin(h1, p[2], p[3], None, False), p[4], p[5])
    return lin(h2, p[6], p[7], h2, True)


def test_a_radial_network_in_front_of_the_convolution():
    """Forward and all gradients against the float64 oracle behind float64 layers.  The convolution is held to 1e-5 of a block's largest
    value elsewhere; the three layers and the norm add at most some 60 u of sums of magnitudes each (layer_util.py), which
    here are up to about 8 times the results: 4 * 60 * 8 * 2^-24 = 1.2e-4 of the largest value."""
    c = workloads.CONFIGS[2]
    wl = workloads.make_graph(2, 192)
    plan = e3j.e3j_plan_create(c["irreps_in"], c["sh_lmax"], c["irreps_out"], c["out_lmax"])
    cp = oconv.Coupling(c["irreps_in"], c["sh_lmax"], c["irreps_out"], c["out_lmax"])
    x, y, _, g = workloads.make_features(wl, plan.n_paths, plan.d_out, with_weights=False)
    _, W = workloads.make_radial(wl, plan.n_paths, 64)
    rng = np.random.default_rng(5)
    rbf = rng.standard_normal((wl.n_edges, 8)).astype(np.float32)
    shapes = [(8, 64), (64,), (64, 64), (64,), (64,), (64,), (64, 64), (64,)]
    params = [(rng.standard_normal(s) * (s[0] ** -0.5 if len(s) == 2 else 0.3) + (k == 4)).astype(np.float32) for k, s in enumerate(shapes)]

    p64 = [torch.from_numpy(a).double().requires_grad_() for a in params]
    rbf64 = torch.from_numpy(rbf).double().requires_grad_()
    silu64 = lambda z: z * torch.sigmoid(z)
    lin64 = lambda t, W, b, r, act: (silu64(t @ W + b) if act else t @ W + b) + (0 if r is None else r)
    norm64 = lambda t, w, b: silu64((t - t.mean(1, keepdim=True)) / torch.sqrt(t.var(1, unbiased=False, keepdim=True) + 1e-5) * w + b)
    h64 = radial_network(rbf64, p64, lin64, norm64, silu64)
    want = oconv.conv_radial_fwd(cp, x, y, h64.detach().numpy(), W, wl.senders, wl.receivers)
    wx, wy, wh, wW = oconv.conv_radial_bwd(cp, x, y, h64.detach().numpy(), W, wl.senders, wl.receivers, g)
    want_p = torch.autograd.grad(h64, [rbf64, *p64], torch.from_numpy(np.asarray(wh, dtype=np.float64)))

    graph = Graph(wl.n_nodes, cuda(wl.senders), cuda(wl.receivers))
    leaves = [cuda(a).requires_grad_() for a in (x, y, W, rbf, *params)]
    lin = lambda t, W, b, r, act: linear(t, W, b, r, SILU if act else 0)
    h = radial_network(leaves[3], leaves[4:], lin, lambda t, w, b: layer_norm(t, w, b, act=SILU), None)
    out = conv_radial(plan, graph, leaves[0], leaves[1], h, leaves[2])
    grads = torch.autograd.grad(out, leaves, cuda(g))
    for got, w in zip((out, *grads), (want, wx, wy, wW, *want_p)):
        w = np.asarray(w.detach() if isinstance(w, torch.Tensor) else w, dtype=np.float64)
        err = np.abs(got.detach().cpu().numpy().astype(np.float64) - w).max()
        assert err <= 1.2e-4 * np.abs(w).max(), (err, np.abs(w).max())
    assert e3j.e3j_plan_device_status(plan) == 0 and e3j.e3j_linear_status() == 0


@pytest.mark.parametrize("act", [0, 1, 2, 3])
def test_gradients_against_differences(act):
    """A directional derivative in float64 from float32 results: differences of a sum of the results along a random direction, step e.
    The results lose up to 60 u of magnitudes of about 4 each, in random directions over the R elements of the sum: below
    1e-6 sqrt(R) altogether, doubled and divided by 2 e; the third derivative adds e^2 / 6 of about 4 sqrt(R) |direction|^3 / sqrt(n)."""
    rng = np.random.default_rng(act)
    rows, n_in, n_out, e = 40, 24, 20, 1e-2
    x, W, b, g = rng.standard_normal((rows, n_in)), rng.standard_normal((n_in, n_out)) / n_in ** 0.5, rng.standard_normal(n_out), rng.standard_normal((rows, n_out))
    w, c = rng.standard_normal(n_out), rng.standard_normal(n_out)
    arrays = [a.astype(np.float32) for a in (x, W, b, w, c)]
    steps = [(rng.standard_normal(a.shape) / a.size ** 0.5).astype(np.float32) for a in arrays]

    def value(*t):
        return layer_norm(linear(t[0], t[1], t[2], act=act), t[3], t[4], act=act)

    leaves = [cuda(a).requires_grad_() for a in arrays]
    grads = torch.autograd.grad(value(*leaves), leaves, cuda(g.astype(np.float32)))
    along = sum((p.double() * cuda(s).double()).sum().item() for p, s in zip(grads, steps))
    at = [(value(*[cuda((a.astype(np.float64) + k * e * s).astype(np.float32)) for a, s in zip(arrays, steps)]).double() * cuda(g)).sum().item() for k in (1, -1)]
    bound = 1e-6 * (rows * n_out) ** 0.5 * 4 / e + 4 * e * e * (rows * n_out) ** 0.5
    assert abs((at[0] - at[1]) / (2 * e) - along) <= bound, (along, at, bound)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_autograd_with_padding(dtype):
    rows, real = 300, 210
    x, r, g = (torch.randn(rows, 40, device="cuda").to(dtype) for _ in range(3))
    for t in (x, r, g):
        t[real:] = float("nan")
    W, b = torch.randn(40, 40, device="cuda").to(dtype), torch.randn(40, device="cuda").to(dtype)
    count = torch.tensor([real], dtype=torch.int32, device="cuda")
    for t in (x, r, W, b):
        t.requires_grad_()
    y = layer_norm(linear(x, W, b, r, SILU, count), n_real=count)
    gx, gr, gW, gb = torch.autograd.grad(y, (x, r, W, b), g)
    assert all(torch.isfinite(t.float()).all() for t in (y, gx, gr, gW, gb))
    assert (y[real:] == 0).all() and (gx[real:] == 0).all() and (gr[real:] == 0).all()
    x2, r2 = (t.detach()[:real].clone().requires_grad_() for t in (x, r))
    y2 = layer_norm(linear(x2, W, b, r2, SILU))
    gx2, gr2 = torch.autograd.grad(y2, (x2, r2), g[:real])
    assert torch.equal(y[:real], y2) and torch.equal(gx[:real], gx2) and torch.equal(gr[:real], gr2)


def test_only_what_is_wanted_and_where_it_is_wanted():
    x, W, b, g = torch.randn(700, 30, device="cuda"), torch.randn(30, 90, device="cuda"), torch.randn(90, device="cuda"), torch.randn(700, 90, device="cuda")
    for rows, cols in ((700, 90), (700, 50), (200, 90), (3000, 50)):
        xs = torch.randn(rows, 30, device="cuda")
        gs, Ws, bs = torch.randn(rows, cols, device="cuda"), W[:, :cols].contiguous(), b[:cols].contiguous()
        full = e3j.e3j_linear_bwd(xs, Ws, bs, gs, SILU)
        for which in range(8):
            flags = [bool(which >> k & 1) for k in range(3)]
            got = e3j.e3j_linear_bwd(xs, Ws, bs, gs, SILU, grad_x=flags[0], grad_W=flags[1], grad_b=flags[2])
            for k in range(3):
                assert (got[k] is None) == (not flags[k]) and (got[k] is None or torch.equal(got[k], full[k]))
    n = torch.randn(90, device="cuda")
    full = e3j.e3j_layer_norm_bwd(g, n, b, g, act=GELU)
    for which in range(8):
        flags = [bool(which >> k & 1) for k in range(3)]
        out = [torch.empty_like(t) if f else None for t, f in zip(full, flags)]
        got = e3j.e3j_layer_norm_bwd(g, n, b, g, 1e-5, GELU, None, *out)
        assert all(a is o and (a is None or torch.equal(a, w)) for a, o, w in zip(got, out, full))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n_in,n_out", [(64, 64), (64, 160), (33, 130)])
def test_arrays_off_their_boundaries_and_rows_behind_them(dtype, n_in, n_out):
    """Views that start one element into their storage: the same values (to the bits where the same kernel runs), and nothing
    written before or behind."""
    rows = 333
    make = lambda *shape: torch.randn(shape, device="cuda").to(dtype)
    x, W, b, r, w = make(rows, n_in), make(n_in, n_out) / 8, make(n_out), make(rows, n_out), make(n_in)

    def shifted(t):
        room = torch.full((t.numel() + 9,), 7.0, dtype=dtype, device="cuda")
        room[1:1 + t.numel()] = t.reshape(-1)
        return room, room[1:1 + t.numel()].view(t.shape)

    def fenced(*shape):
        room, view = shifted(torch.full(shape, float("nan"), dtype=dtype, device="cuda"))
        return room, view

    def check(room, view, want):
        assert torch.equal(view, want) and (room[0] == 7).all() and (room[1 + view.numel():] == 7).all()

    (_, x1), (_, W1), (_, b1), (_, r1), (_, w1) = map(shifted, (x, W, b, r, w))
    want = e3j.e3j_linear_fwd(x, W, b, r, SILU)
    room, y = fenced(rows, n_out)
    e3j.e3j_linear_fwd(x1, W1, b1, r1, SILU, out=y)
    check(room, y, want)
    want = e3j.e3j_linear_bwd(x, W, b, r, SILU)
    outs = [fenced(*t.shape) for t in want]
    e3j.e3j_linear_bwd(x1, W1, b1, r1, SILU, None, *(o[1] for o in outs))
    for (room, view), t in zip(outs, want):
        check(room, view, t)
    close = dict(rtol=0, atol=0.1) if dtype == torch.bfloat16 else dict(rtol=0, atol=1e-3)   # (another order of the sums; the values are held to float64 elsewhere)
    want = e3j.e3j_layer_norm_bwd(x, w, w, x, act=GELU)
    outs = [fenced(*t.shape) for t in want]
    e3j.e3j_layer_norm_bwd(x1, w1, w1, x1, 1e-5, GELU, None, *(o[1] for o in outs))
    for (room, view), t in zip(outs, want):
        assert torch.allclose(view.float(), t.float(), **close) and room[0] == 7 and (room[1 + view.numel():] == 7).all()


def test_another_stream_and_its_workspace():
    x, W, b, g = (torch.randn(*s, device="cuda") for s in ((20000, 96), (96, 70), (70,), (20000, 70)))
    w = torch.randn(96, device="cuda")
    want = *e3j.e3j_linear_bwd(x, W, b, g, SILU), *e3j.e3j_layer_norm_bwd(x, w, w, x)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    got = *e3j.e3j_linear_bwd(x, W, b, g, SILU, stream=side), *e3j.e3j_layer_norm_bwd(x, w, w, x, stream=side)
    junk = [torch.zeros(e3j.e3j_linear_bwd_workspace_bytes(20000, 96, 70, 1), dtype=torch.uint8, device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    assert len(junk) == 3 and all(torch.equal(a, b) for a, b in zip(got, want))


def test_captured_and_at_once():
    shapes = [(1000, 64, 64), (5000, 64, 64), (4000, 100, 130)]
    sides = [torch.cuda.Stream() for _ in shapes]
    data, want = [], []
    for rows, n_in, n_out in shapes:
        t = [torch.randn(*s, device="cuda") for s in ((rows, n_in), (n_in, n_out), (n_out,), (rows, n_out), (n_in,))]
        data.append(t)
        want.append((e3j.e3j_linear_fwd(*t[:3], act=GELU), *e3j.e3j_linear_bwd(*t[:4], GELU), *e3j.e3j_layer_norm_bwd(t[0], t[4], t[4], t[0])))
    torch.cuda.synchronize()
    for _ in range(5):   # three at once
        got = []
        for t, side in zip(data, sides):
            with torch.cuda.stream(side):
                got.append((e3j.e3j_linear_fwd(*t[:3], act=GELU), *e3j.e3j_linear_bwd(*t[:4], GELU), *e3j.e3j_layer_norm_bwd(t[0], t[4], t[4], t[0])))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for p, q in zip(got, want) for a, b in zip(p, q))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [(e3j.e3j_linear_fwd(*t[:3], act=GELU), *e3j.e3j_linear_bwd(*t[:4], GELU), *e3j.e3j_layer_norm_bwd(t[0], t[4], t[4], t[0])) for t in data]
    for t in data:
        t[0].mul_(2)
    want = [(e3j.e3j_linear_fwd(*t[:3], act=GELU), *e3j.e3j_linear_bwd(*t[:4], GELU), *e3j.e3j_layer_norm_bwd(t[0], t[4], t[4], t[0])) for t in data]
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for p, q in zip(got, want) for a, b in zip(p, q))


def test_a_captured_backward():
    x = torch.randn(800, 64, device="cuda", requires_grad=True)
    W, w = torch.randn(64, 64, device="cuda", requires_grad=True), torch.randn(64, device="cuda", requires_grad=True)
    g = torch.randn(800, 64, device="cuda")
    step = lambda: torch.autograd.grad(layer_norm(linear(x, W, act=SILU), w), (x, W, w), g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = [t.clone() for t in step()]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_padding_does_not_change_the_bits_of_rows():
    """A row's results do not depend on how many rows, real or not, are behind it."""
    for dtype in (torch.float32, torch.bfloat16):
        x, W, b = (torch.randn(*s, device="cuda").to(dtype) for s in ((1500, 64), (64, 100), (100,)))
        y, z = e3j.e3j_linear_fwd(x, W, b, act=SILU), e3j.e3j_layer_norm_fwd(x, act=SILU)
        for rows in (1, 129, 1000):
            assert torch.equal(e3j.e3j_linear_fwd(x[:rows], W, b, act=SILU), y[:rows])
            assert torch.equal(e3j.e3j_layer_norm_fwd(x[:rows], act=SILU), z[:rows])


def test_more_than_2_to_the_31_elements():
    rows, n = 34_000_007, 64
    x = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
    x[:1000].normal_()
    x[1000:-1000] = 0.5
    x[-1000:] = x[:1000]
    W, b = (torch.randn(n, n, device="cuda") / 8).bfloat16(), torch.randn(n, device="cuda").bfloat16()
    for call in (lambda t: e3j.e3j_linear_fwd(t, W, b, act=SILU), lambda t: e3j.e3j_layer_norm_fwd(t, b, b, act=SILU),
                 lambda t: e3j.e3j_linear_bwd(t, W, b, t, SILU, grad_W=False, grad_b=False)[0],
                 lambda t: e3j.e3j_layer_norm_bwd(t, b, b, t, grad_weight=False, grad_bias=False)[0]):
        y = call(x)
        assert torch.equal(y[-1000:], call(x[:1000])) and torch.equal(y[:1000], y[-1000:])
        del y
        torch.cuda.empty_cache()


def test_infinities_and_the_largest_values():
    x = torch.randn(200, 64, device="cuda")
    W = torch.eye(64, device="cuda")
    want = e3j.e3j_linear_fwd(x, W)
    assert torch.equal(want, x)                                        # three terms are the whole of a float32
    x[3, 5], x[130, 0], x[77, 63] = float("inf"), float("nan"), float("-inf")
    y = e3j.e3j_linear_fwd(x, W)
    rows = torch.tensor([3, 77, 130], device="cuda")
    other = torch.ones(200, dtype=torch.bool, device="cuda")
    other[rows] = False
    assert torch.equal(y[other], want[other]) and not torch.isfinite(y[rows]).all(1).any()
    big = torch.full((5, 64), 3.4e38, device="cuda")
    assert torch.equal(e3j.e3j_linear_fwd(big, W), big)
    for act, low, high in ((SILU, 0.0, 200.0), (GELU, 0.0, 200.0), (e3j.E3J_ACT_TANH, -1.0, 1.0)):
        z = torch.tensor([[-200.0, 200.0]], device="cuda")
        assert torch.equal(e3j.e3j_linear_fwd(z, torch.eye(2, device="cuda"), act=act), torch.tensor([[low, high]], device="cuda"))


def test_refusals():
    x, W = torch.randn(10, 4, device="cuda"), torch.randn(4, 6, device="cuda")
    with pytest.raises(ValueError, match="W has shape"):
        e3j.e3j_linear_fwd(x, torch.randn(5, 6, device="cuda"))
    with pytest.raises(ValueError, match="b has shape"):
        e3j.e3j_linear_fwd(x, W, torch.randn(4, device="cuda"))
    with pytest.raises(TypeError, match="x must be float32 or bfloat16"):
        e3j.e3j_linear_fwd(x.double(), W.double())
    with pytest.raises(TypeError, match="W must be contiguous"):
        e3j.e3j_linear_fwd(x, W.bfloat16())
    with pytest.raises(TypeError, match="x must be contiguous"):
        e3j.e3j_layer_norm_fwd(W.t())
    with pytest.raises(TypeError, match="b must be a CUDA tensor"):
        e3j.e3j_linear_fwd(x, W, torch.randn(6))
    with pytest.raises(ValueError, match="x has shape"):
        e3j.e3j_layer_norm_fwd(x[None])
    with pytest.raises(TypeError, match="n_real must be contiguous"):
        e3j.e3j_layer_norm_fwd(x, n_real=torch.zeros(1, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError, match="n_real has shape"):
        e3j.e3j_layer_norm_fwd(x, n_real=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(e3j.E3JError, match="e3j_linear_fwd: invalid argument"):
        e3j.e3j_linear_fwd(x, W, act=9)
    with pytest.raises(e3j.E3JError, match="e3j_layer_norm_fwd: invalid argument"):
        e3j.e3j_layer_norm_fwd(x, eps=-1.0)
    with pytest.raises(e3j.E3JError):
        e3j.e3j_layer_norm_fwd(torch.randn(2, 5000, device="cuda"))
    big, g = torch.randn(5000, 64, device="cuda"), torch.randn(5000, 64, device="cuda")
    with pytest.raises(ValueError, match="workspace"):
        e3j.e3j_linear_bwd(big, torch.randn(64, 64, device="cuda"), None, g, workspace=torch.empty(100, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("rows,n_in,n_out", [(300, 1030, 70), (130, 70, 1030), (200, 4096, 100), (150, 600, 513)])
def test_long_contractions_keep_float32_accuracy(rows, n_in, n_out):
    """Values of one sign, for which every addition of the tensor cores cuts off in the same direction: a chain is 16 of them, each up to 2 u
    of a partial sum that grows evenly (so 16 u on average over the chain), chains and terms are rounded: below 32 u = 2e-6 of
    the result, against 4096 / 16 * u = 1.5e-5 in one chain."""
    x, W, g = (torch.rand(*s, device="cuda") for s in ((rows, n_in), (n_in, n_out), (rows, n_out)))
    for got, want in ((e3j.e3j_linear_fwd(x, W), x.double() @ W.double()),
                      (e3j.e3j_linear_bwd(x, W, None, g, grad_W=False, grad_b=False)[0], g.double() @ W.double().T)):
        assert ((got.double() - want).abs() / want).max() <= 2e-6
    (xs, x_), (Ws, W_), (bs, b_), (gs, g_) = [(t.cuda(), t.double().numpy()) for t in (torch.randn(rows, n_in), torch.randn(n_in, n_out) / n_in ** 0.5, torch.randn(n_out), torch.randn(rows, n_out))]
    ref.assert_within(e3j.e3j_linear_fwd(xs, Ws, bs, gs, SILU), *ref.linear_fwd(x_, W_, b_, g_, "silu", 2.0 ** -24), "y")
    want, bounds = ref.linear_bwd(x_, W_, b_, g_, "gelu", 2.0 ** -24)
    for t, v, e in zip(e3j.e3j_linear_bwd(xs, Ws, bs, gs, GELU), want, bounds):
        ref.assert_within(t, v, e)


@pytest.mark.parametrize("n_in,n_out,act", [(128, 96, SILU), (8, 64, 0), (200, 200, 0), (72, 130, GELU)])
def test_large_padded_calls_in_bfloat16(n_in, n_out, act):
    """Large enough for operands to come as boxes, NaN behind the last real row (inside a tile): the rows of the short call to the
    bits, and the gradients within their bounds."""
    rows, real = 61_003, 40_007
    x, W, b, r = ((torch.randn(*s, device="cuda") * k).bfloat16() for s, k in (((rows, n_in), 1), ((n_in, n_out), n_in ** -0.5), ((n_out,), 1), ((rows, n_out), 1)))
    x[real:], r[real:] = float("nan"), float("nan")
    count = torch.tensor([real], dtype=torch.int32, device="cuda")
    y = e3j.e3j_linear_fwd(x, W, b, r, act, n_real=count)
    assert (y[real:] == 0).all() and torch.equal(y[:real], e3j.e3j_linear_fwd(x[:real], W, b, r[:real], act))
    got = e3j.e3j_linear_bwd(x, W, b, r, act, n_real=count)
    assert (got[0][real:] == 0).all()
    name = {0: "none", 1: "silu", 3: "gelu"}[act]
    x_, W_, b_, g_ = (t.double().cpu().numpy() for t in (x[:real], W, b, r[:real]))
    ref.assert_within(y[:real], *ref.linear_fwd(x_, W_, b_, g_, name, 2.0 ** -8))
    want, bounds = ref.linear_bwd(x_, W_, b_, g_, name, 2.0 ** -8)
    for t, v, e in zip((got[0][:real], *got[1:]), want, bounds):
        ref.assert_within(t, v, e)
    assert e3j.e3j_linear_status() == 0
