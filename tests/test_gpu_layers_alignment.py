"""Layer norm on arrays that do not start on 16 bytes (GPU): every width's kernels, forward and backward, against float64."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import layer_util as ref
import paper_2609_35099_b200 as e3j

pytestmark = pytest.mark.gpu


def moved(a, dtype, by):
    """(its storage, a view with those values that starts `by` elements into it), 7 before and behind."""
    t = torch.from_numpy(np.asarray(a, dtype=np.float64)).to(dtype)
    room = torch.full((t.numel() + 16,), 7.0, dtype=dtype, device="cuda")
    room[by:by + t.numel()] = t.reshape(-1).cuda()
    return room, room[by:by + t.numel()].view(t.shape)


def untouched(room, by, n):
    return (room[:by] == 7).all() and (room[by + n:] == 7).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 7, 33, 64, 97, 130, 256, 257, 385, 512, 1000, 1024, 2047, 2050, 4096])
@pytest.mark.parametrize("rows,by", [(3, 1), (301, 1), (301, 3)])
def test_norm_off_16_bytes(rows, by, n, dtype):
    rng = np.random.default_rng(rows + n)
    half = torch.finfo(dtype).eps / 2
    arrays = [rng.standard_normal(s) * k for s, k in (((rows, n), 1.5), ((n,), 1), ((n,), 0.5), ((rows, n), 1))]
    (_, x), (_, w), (_, c), (_, g) = (moved(a, dtype, by) for a in arrays)
    x_, w_, c_, g_ = (t.double().cpu().numpy() for t in (x, w, c, g))
    out = lambda *shape: moved(np.full(shape, np.nan), dtype, by)
    for act, weight, bias in (("silu", True, True), ("gelu", False, True), ("none", True, False)):
        one, none = w_ if weight else np.ones(n), c_ if bias else np.zeros(n)
        room, y = out(rows, n)
        e3j.e3j_layer_norm_fwd(x, w if weight else None, c if bias else None, 1e-5, ref.ACTS[act], out=y)
        ref.assert_within(y, *ref.norm_fwd(x_, one, none, 1e-5, act, half), act)
        assert untouched(room, by, rows * n)
        outs = [out(rows, n), out(n), out(n)]
        e3j.e3j_layer_norm_bwd(x, w if weight else None, c if bias else None, g, 1e-5, ref.ACTS[act], None, *(o[1] for o in outs))
        want, bounds = ref.norm_bwd(x_, one, none, g_, 1e-5, act, half)
        for (room, t), v, e, what in zip(outs, want, bounds, ("grad_x", "grad_weight", "grad_bias")):
            ref.assert_within(t, v, e, f"{act} {what}")
            assert untouched(room, by, t.numel())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [64, 385, 1024])
def test_padded_rows_off_16_bytes(n, dtype):
    rows, real = 200, 131
    rng = np.random.default_rng(n)
    half = torch.finfo(dtype).eps / 2
    (_, x), (_, g) = (moved(rng.standard_normal((rows, n)), dtype, 1) for _ in range(2))
    x[real:], g[real:] = float("nan"), float("nan")
    x_, g_ = (t[:real].double().cpu().numpy() for t in (x, g))
    count = torch.tensor([real], dtype=torch.int32, device="cuda")
    (room, y), (room_x, gx) = (moved(np.full((rows, n), np.nan), dtype, 1) for _ in range(2))
    e3j.e3j_layer_norm_fwd(x, act=1, n_real=count, out=y)
    _, gw, gc = e3j.e3j_layer_norm_bwd(x, None, None, g, act=1, n_real=count, grad_x=gx)
    assert (y[real:] == 0).all() and (gx[real:] == 0).all() and untouched(room, 1, rows * n) and untouched(room_x, 1, rows * n)
    one, none = np.ones(n), np.zeros(n)
    ref.assert_within(y[:real], *ref.norm_fwd(x_, one, none, 1e-5, "silu", half), "y")
    want, bounds = ref.norm_bwd(x_, one, none, g_, 1e-5, "silu", half)
    for t, v, e in zip((gx[:real], gw, gc), want, bounds):
        ref.assert_within(t, v, e)
