"""How exact the float32 linear layer's sums are (GPU): chains of the tensor cores' additions, every term product of the gradients of W, sums over
many rows."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import layer_util as ref
import paper_2609_35099_b200 as e3j

pytestmark = pytest.mark.gpu
U = 2.0 ** -24   # half a step of float32


@pytest.mark.parametrize("k", [257, 400, 512, 513, 1024])
def test_contractions_of_every_length_are_cut_into_chains(k):
    """The first product is 1 and the others, positive, add up to less than 0.13 (0.26 for 1024), so every partial sum of the first chain is between 1
    and 2.  An instruction adds 16 products to it; it cuts each off at a multiple of u / 4, which loses u / 8 on average, and the sum at a multiple of
    2 u, which loses u on average: 3 u (measured on chains of 1, 2, 4 .. instructions: 2.9, 6.1, 12.1 .. u).  A chain has 16 of them: 48 u.  Each
    of up to three later chains is a sum below 0.07: 48 u of that, 10 u in all; they and the smaller terms are added rounding, half up and
    half down: 1 u.  In relation to the results, at least 1.06 with 257 products and 1.25 with 1024: below 52 u on average.  In one chain 512 would
    lose 32 * 3 u / 1.12 = 86 u, 400 71 u."""
    rng = np.random.default_rng(k)
    a, w = rng.random((600, k)), rng.random((k, 200)) * 2.0 ** -10
    a[:, 0], w[0] = 1, 1
    x, W = torch.from_numpy(a).float().cuda(), torch.from_numpy(w).float().cuda()
    forward, want = e3j.e3j_linear_fwd(x, W), x.double() @ W.double()
    grad_x = e3j.e3j_linear_bwd(x[:, :200].contiguous(), W.t().contiguous(), None, x, grad_W=False, grad_b=False)[0]
    for got in (forward, grad_x):
        assert abs(((got.double() - want) / want).mean().item()) <= 52 * U


@pytest.mark.parametrize("n_in", [32, 64, 96, 300, 520])
@pytest.mark.parametrize("n_out", [64, 129, 160, 192, 257, 288])
def test_a_tile_s_width_does_not_change_bits(n_in, n_out):
    """Tiles are 64 or 128 columns wide by rules on sizes, rows and what the results meet; a result's sums are the same in both."""
    x, W, b = torch.randn(20000, n_in, device="cuda"), torch.randn(n_in, n_out, device="cuda"), torch.randn(n_out, device="cuda")
    y = e3j.e3j_linear_fwd(x, W, b)
    assert torch.equal(y, e3j.e3j_linear_fwd(x, W, b, torch.zeros_like(y)))
    assert torch.equal(y[:100], e3j.e3j_linear_fwd(x[:100], W, b))
    if n_out % 64 == 0:
        room = torch.empty(y.numel() + 1, device="cuda")[1:].view(y.shape)   # (rows off 16 bytes)
        assert torch.equal(y, e3j.e3j_linear_fwd(x, W, b, out=room))


def terms(rng, n):
    """n times three values of 8 significant bits, 2^-8 of one another: the leading terms of a float32 and what is behind them."""
    return [(rng.integers(128, 256, n) * rng.choice([-1, 1], n)).astype(np.float64) * 2.0 ** (-8 * k - 7) for k in range(3)]


@pytest.mark.parametrize("product", ["hi hi", "hi mid", "mid hi", "mid mid", "hi lo", "lo hi"])
@pytest.mark.parametrize("rows,n_in,n_out", [(300, 64, 64), (20000, 64, 64), (1500, 33, 47), (300, 128, 96), (5000, 97, 161), (9000, 300, 64), (700, 40, 200)])
def test_grad_W_has_every_term_product(rows, n_in, n_out, product):
    """Two or four neighbouring rows whose leading products cancel, zeros elsewhere: what is left is the named product of terms, exact in
    float32 (16 bits), and so is every partial sum (multiples of the smallest product, less than 2^24 of them), as long as the rows are in
    one chain: they share a group of 16.  The result has to be that product to the bit."""
    rng = np.random.default_rng(n_in + n_out)
    H, M, L = terms(rng, n_in)
    sign = np.sign(H)
    M, L = np.abs(M) * sign, np.abs(L) * sign       # (the parts of one value have its sign)
    G, N, O = terms(rng, n_out)
    sign = np.sign(G)
    N, O = np.abs(N) * sign, np.abs(O) * sign
    x_of, g_of, want = {
        "hi hi": ([H], [G], (H, G)),
        "hi mid": ([H, -H], [G + N, G], (H, N)),
        "mid hi": ([H + M, -H], [G, G], (M, G)),
        "mid mid": ([H + M, -H, -(H + M), H], [G + N, G + N, G, G], (M, N)),
        "hi lo": ([H, -H], [G + N + O, G + N], (H, O)),
        "lo hi": ([H + M + L, -(H + M)], [G, G], (L, G)),
    }[product]
    want = np.outer(*want)
    W = torch.randn(n_in, n_out, device="cuda")
    for at in (0, 16 * ((rows - 16) // 16), 16 * (rows // 32) + 7):   # the first rows, the last whole group, the middle of one
        x, g = torch.zeros(rows, n_in), torch.zeros(rows, n_out)
        for i, (a, b) in enumerate(zip(x_of, g_of)):
            x[at + i], g[at + i] = torch.from_numpy(a).float(), torch.from_numpy(b).float()
        got = e3j.e3j_linear_bwd(x.cuda(), W, None, g.cuda())[1].cpu().double().numpy()
        assert np.array_equal(got, want), (at, np.abs(got - want).max() / np.abs(want).max())


@pytest.mark.parametrize("rows,n_in,n_out", [(2500, 64, 64), (20000, 64, 64), (160900, 64, 64), (2500, 128, 96), (9000, 40, 96), (60001, 97, 161)])
def test_sums_over_rows_keep_float32_accuracy(rows, n_in, n_out):
    """2-norms over normal values, whose partial sums grow as the square root of their number.  A chain is at most 24 additions of 16 rows, each
    cutting off less than 2 u of the partial sum: 2 u (4 + 4 sqrt 2 + .. + 4 sqrt 24) = 2 u * 4 * 82 = 656 u at most for a chain whose own size is
    sqrt(384) = 19.6, so 33.5 u of it; chains are independent, so this is the sum's too.  The products' three missing terms are 9 u of a
    product, independent too, and adding up to 440 chains and shares rounds: sqrt(440 / 2) u = 15 u if one after the other.  Altogether
    below 60 u = 3.6e-6; without one of the products of weight 2^-16, about 2^-17 = 128 u would be missing."""
    x, W, g = (torch.randn(*s, device="cuda") for s in ((rows, n_in), (n_in, n_out), (rows, n_out)))
    _, gW, gb = e3j.e3j_linear_bwd(x, W, None, g)
    for got, want in ((gW, x.double().T @ g.double()), (gb, g.double().sum(0))):
        assert (got.double() - want).norm() <= 60 * U * want.norm()


@pytest.mark.parametrize("rows,n", [(1500, 64), (30000, 64), (160900, 64), (20000, 9), (9001, 385), (5000, 1024), (300, 4096)])
def test_layer_norm_s_sums_keep_float32_accuracy(rows, n):
    """2-norms again.  Adding n rounded values of random sign one after the other loses u sqrt(n / 2) of the sum.  A lane, its warp, the blocks and their
    shares are at most 1100 (160 900 rows: 296 blocks and 32 slots, 17 rows a slot) additions: 24 u; the elements gz and gz xh lose 1 u and, through
    mean and variance of up to 4096 columns added pairwise over lanes, 16 to 32 at a time in a row, below 16 u: 40 u = 2.4e-6."""
    x, w, g = torch.randn(rows, n, device="cuda") * 2 + 1, torch.randn(n, device="cuda"), torch.randn(rows, n, device="cuda")
    _, gw, gc = e3j.e3j_layer_norm_bwd(x, w, None, g)
    x64 = x.double()
    d = x64 - x64.mean(1, keepdim=True)
    xh = d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5)
    for got, want in ((gw, (g.double() * xh).sum(0)), (gc, g.double().sum(0))):
        assert (got.double() - want).norm() <= 40 * U * want.norm()


@pytest.mark.parametrize("rows,real", [(20003, None), (20003, 12345), (389, 200), (389, 1), (389, 0)])
@pytest.mark.parametrize("n_in,n_out", [(300, 161), (512, 256), (400, 64), (257, 130), (64, 320), (97, 401)])
def test_two_chains_over_many_tiles_and_padded(rows, real, n_in, n_out):
    """More than one tile a block, and lists that end inside one, where the forward's or grad_x's contraction is two chains."""
    rng = np.random.default_rng(n_in)
    kept = rows if real is None else real
    arrays = [rng.standard_normal(s) * k for s, k in (((rows, n_in), 1), ((n_in, n_out), n_in ** -0.5), ((n_out,), 0.5), ((rows, n_out), 1))]
    x, W, b, g = (torch.from_numpy(a).float().cuda() for a in arrays)
    x_, W_, b_, g_ = (t.double().cpu().numpy() for t in (x[:kept], W, b, g[:kept]))
    x[kept:], g[kept:] = float("nan"), float("nan")
    count = None if real is None else torch.tensor([real], dtype=torch.int32, device="cuda")
    y = e3j.e3j_linear_fwd(x, W, b, g, ref.ACTS["silu"], n_real=count)
    ref.assert_within(y[:kept], *ref.linear_fwd(x_, W_, b_, g_, "silu", U), "y")
    got = e3j.e3j_linear_bwd(x, W, b, g, ref.ACTS["gelu"], n_real=count)
    want, bounds = ref.linear_bwd(x_, W_, b_, g_, "gelu", U)
    for t, v, e, what in zip((got[0][:kept], *got[1:]), want, bounds, ("grad_x", "grad_W", "grad_b")):
        ref.assert_within(t, v, e, what)
    assert (y[kept:] == 0).all() and (got[0][kept:] == 0).all() and e3j.e3j_linear_status() == 0
