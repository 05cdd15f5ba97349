"""How exact the float32 linear layer's sums are (GPU): chains of the tensor cores' additions, every term product of the gradients of W, sums over
many rows."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

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
