"""What the hidden layers rely on besides their inputs (GPU): the count of real rows until the backward, workspaces, what else is on the GPU."""
import pytest

torch = pytest.importorskip("torch")

import paper_2609_35099_b200 as e3j
from paper_2609_35099_b200.autograd import layer_norm, linear

pytestmark = pytest.mark.gpu
SILU, GELU = e3j.E3J_ACT_SILU, e3j.E3J_ACT_GELU


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_count_of_real_rows_is_the_forward_s(dtype):
    """A count that is rewritten for the next padded list before the backward of this one: by torch, and by a call of the library."""
    rows, real = 500, 300
    x, W, b, r, g, w = (torch.randn(*s, device="cuda").to(dtype).requires_grad_() for s in ((rows, 40), (40, 70), (70,), (rows, 70), (rows, 70), (70,)))
    with torch.no_grad():
        x[real:], r[real:], g[real:] = float("nan"), float("nan"), float("nan")

    def by_torch(count):
        count.fill_(450)

    def by_the_library(count):   # (a row of four words; the count is the first of them)
        words = torch.full((1, 4), 450, dtype=torch.int32, device="cuda").view(torch.float32)
        e3j.e3j_rows_gather(count._base.view(torch.float32).view(1, 4), words, torch.zeros(1, dtype=torch.int32, device="cuda"))

    def both(count, rewrite):
        y = layer_norm(linear(x, W, b, r, SILU, count), w, act=GELU, n_real=count)
        rewrite(count)
        return torch.autograd.grad(y, (x, W, b, r, w), g)

    count = lambda: torch.tensor([real] * 4, dtype=torch.int32, device="cuda")[:1]
    want = both(count(), lambda c: None)
    assert all(torch.isfinite(t.float()).all() for t in want)
    for rewrite in (by_torch, by_the_library):
        c = count()
        got = both(c, rewrite)
        assert c.item() == 450
        assert all(torch.equal(p, q) for p, q in zip(got, want)), rewrite.__name__


def test_clusters_on_several_streams():
    """Backward calls of few rows, one cluster each, on eight streams: more clusters at once than blocks of one that an SM could hold."""
    shapes = [(1000, 64, 64), (900, 40, 64), (700, 64, 24), (1024, 8, 64)]
    for dtype in (torch.bfloat16, torch.float32):
        data = [[torch.randn(*s, device="cuda").to(dtype) for s in ((rows, n_in), (n_in, n_out), (n_out,), (rows, n_out))] for rows, n_in, n_out in shapes]
        want = [e3j.e3j_linear_bwd(*t, SILU) for t in data]
        torch.cuda.synchronize()
        sides, got = [torch.cuda.Stream() for _ in range(8)], []
        for k in range(200):
            with torch.cuda.stream(sides[k % 8]):
                got.append(e3j.e3j_linear_bwd(*data[k % 4], SILU))
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for k, t in enumerate(got) for p, q in zip(t, want[k % 4]))
    assert e3j.e3j_linear_status() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,n_in,n_out,act", [(377, 104, 140, SILU), (377, 104, 140, 0), (1218, 96, 200, GELU), (3000, 33, 130, 0)])
def test_sums_beside_grad_x_see_this_call_s_gradients(rows, n_in, n_out, act, dtype):
    """Calls that follow one another with the same workspace and the same arrays, rewritten in between on the stream: the sums over rows,
    which run beside grad_x's product, are those of the call without grad_x."""
    x, W, g = (torch.empty(*s, device="cuda", dtype=dtype) for s in ((rows, n_in), (n_in, n_out), (rows, n_out)))
    W.normal_()
    room = torch.empty(max(1, e3j.e3j_linear_bwd_workspace_bytes(rows, n_in, n_out, act, int(dtype == torch.bfloat16))), dtype=torch.uint8, device="cuda")
    xs, gs = [torch.randn_like(x) for _ in range(4)], [torch.randn_like(g) for _ in range(5)]
    got, want = [], []
    for k in range(60):
        x.copy_(xs[k % 4])
        g.copy_(gs[k % 5])
        got.append(e3j.e3j_linear_bwd(x, W, None, g, act, workspace=room)[1:])
    for k in range(20):
        want.append(e3j.e3j_linear_bwd(xs[k % 4], W, None, gs[k % 5], act, grad_x=False)[1:])
    assert all(torch.equal(p, q) for k in range(60) for p, q in zip(got[k], want[k % 20]))


def bwd_without_room(x, W, g, act, gx, dtype):
    """The C entry point with no workspace, for grad_x alone."""
    rows, n_in = x.shape
    return e3j._load().e3j_linear_bwd(dtype, rows, n_in, W.shape[1], x.data_ptr(), W.data_ptr(), None, g.data_ptr(), act, None, gx.data_ptr(),
                                      None, None, None, 0, torch.cuda.current_stream().cuda_stream)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,n_in,n_out,act", [(5000, 64, 64, SILU), (5000, 30, 17, 0), (200, 64, 64, GELU), (5000, 100, 70, 0), (40000, 64, 64, GELU)])
def test_grad_x_alone_needs_no_room_for_shares(rows, n_in, n_out, act, dtype):
    x, W, g = (torch.randn(*s, device="cuda").to(dtype) for s in ((rows, n_in), (n_in, n_out), (rows, n_out)))
    want = e3j.e3j_linear_bwd(x, W, None, g, act)[0]
    gx = torch.full_like(x, float("nan"))
    assert bwd_without_room(x, W, g, act, gx, int(dtype == torch.bfloat16)) == 0
    assert torch.equal(gx, want)
    gx.fill_(float("nan"))
    before = torch.cuda.memory_stats()["allocation.all.allocated"]
    e3j.e3j_linear_bwd(x, W, None, g, act, grad_x=gx, grad_W=False, grad_b=False)
    e3j.e3j_layer_norm_bwd(x, None, None, x, grad_x=gx, grad_weight=False, grad_bias=False)
    assert torch.cuda.memory_stats()["allocation.all.allocated"] == before
    e3j.e3j_linear_bwd(x, W, None, g, act, grad_x=gx, grad_W=False, grad_b=False)
    assert torch.equal(gx, want)


def test_with_an_activation_beyond_64_columns_room_for_gz_is_still_asked_for():
    x, W, g = torch.randn(5000, 100, device="cuda"), torch.randn(100, 70, device="cuda"), torch.randn(5000, 70, device="cuda")
    gx = torch.empty_like(x)
    assert bwd_without_room(x, W, g, SILU, gx, 0) == e3j.E3J_ERR_WORKSPACE
    assert torch.equal(e3j.e3j_linear_bwd(x, W, None, g, SILU, grad_W=False, grad_b=False)[0], e3j.e3j_linear_bwd(x, W, None, g, SILU)[0])


def test_a_missing_or_flat_W_is_named():
    x, g = torch.randn(5, 4, device="cuda"), torch.randn(5, 3, device="cuda")
    for W in (None, [1.0], torch.randn(12, device="cuda"), torch.tensor(1.0, device="cuda")):
        for call in (lambda: e3j.e3j_linear_fwd(x, W), lambda: e3j.e3j_linear_bwd(x, W, None, g)):
            with pytest.raises(TypeError, match="W must be a CUDA tensor"):
                call()
