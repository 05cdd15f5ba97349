"""The hidden layers' refusals, sizes and marshalling, as far as they need no device."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

import paper_2609_35099_b200 as e3j

LIB = e3j._load()
BAD, UNSUPPORTED, NO_ROOM = e3j.E3J_ERR_INVALID_ARG, e3j.E3J_ERR_UNSUPPORTED, e3j.E3J_ERR_WORKSPACE
P = 1 << 20   # stands for a device address: none of these calls gets as far as using it


def linear_fwd(dtype=0, rows=5, n_in=4, n_out=3, x=P, W=P, b=P, residual=None, act=1, n_real=None, y=P):
    return LIB.e3j_linear_fwd(dtype, rows, n_in, n_out, x, W, b, residual, act, n_real, y, None)


def linear_bwd(dtype=0, rows=5, n_in=4, n_out=3, x=P, W=P, b=P, grad_y=P, act=1, gx=P, gW=P, gb=P, ws=None, size=0):
    return LIB.e3j_linear_bwd(dtype, rows, n_in, n_out, x, W, b, grad_y, act, None, gx, gW, gb, ws, size, None)


def norm_fwd(dtype=0, rows=5, n=4, x=P, w=P, b=P, eps=1e-5, act=1, y=P):
    return LIB.e3j_layer_norm_fwd(dtype, rows, n, x, w, b, eps, act, None, y, None)


def norm_bwd(dtype=0, rows=5, n=4, x=P, w=P, b=P, grad_y=P, eps=1e-5, act=1, gx=P, gw=P, gb=P, ws=None, size=0):
    return LIB.e3j_layer_norm_bwd(dtype, rows, n, x, w, b, grad_y, eps, act, None, gx, gw, gb, ws, size, None)


@pytest.mark.parametrize("call", [linear_fwd, linear_bwd, norm_fwd, norm_bwd])
def test_types_activations_and_sizes(call):
    wide = {"n_in": 4097} if "linear" in call.__name__ else {"n": 4097}
    none = {"n_in": 0} if "linear" in call.__name__ else {"n": 0}
    assert call(dtype=2) == call(dtype=-1) == BAD
    assert call(act=4) == call(act=-1) == BAD
    assert call(rows=-1) == call(**none) == BAD
    assert call(**wide) == UNSUPPORTED and call(rows=(1 << 31) - 1) == UNSUPPORTED
    assert call(x=None) == BAD and call(x=P + 2) == BAD and call(dtype=1, x=P + 1) == BAD


def test_linear_arguments():
    assert linear_fwd(n_out=0) == BAD and linear_fwd(n_out=4097) == UNSUPPORTED
    assert linear_fwd(W=None) == BAD and linear_fwd(y=None) == BAD
    for name in ("W", "b", "residual", "y"):
        assert linear_fwd(**{name: P + 1}) == BAD
    assert linear_bwd(W=None) == BAD and linear_bwd(grad_y=None) == BAD
    for name in ("W", "b", "grad_y", "gx", "gW", "gb"):
        assert linear_bwd(**{name: P + 2}) == BAD
    assert linear_fwd(rows=0, x=None, y=None) == 0                       # nothing to do
    assert linear_bwd(gx=None, gW=None, gb=None) == 0


def test_norm_arguments():
    for call in (norm_fwd, norm_bwd):
        assert call(eps=-1e-9) == BAD and call(eps=float("nan")) == BAD
        assert call(w=P + 1) == BAD and call(b=P + 2) == BAD
    assert norm_fwd(y=None) == BAD and norm_bwd(grad_y=None) == BAD
    assert norm_fwd(rows=0, x=None, y=None) == 0 and norm_bwd(gx=None, gw=None, gb=None) == 0


def test_workspaces():
    assert e3j.e3j_linear_bwd_workspace_bytes(1000, 64, 64, 1) == 0      # one cluster: none is needed
    need = e3j.e3j_linear_bwd_workspace_bytes(5000, 64, 64, 1)
    assert need > 0 and need % 256 == 0
    kw = dict(rows=5000, n_in=64, n_out=64)
    assert linear_bwd(**kw) == NO_ROOM and linear_bwd(**kw, ws=P, size=need - 1) == NO_ROOM
    assert linear_bwd(**kw, ws=P + 128, size=need) == NO_ROOM
    gz = e3j.e3j_linear_bwd_workspace_bytes(100, 10, 70, 1)              # gz in memory: rows of 72 float32
    assert gz == -(-100 * 72 * 4 // 256) * 256 and e3j.e3j_linear_bwd_workspace_bytes(100, 10, 70, 0) == 0
    assert e3j.e3j_layer_norm_bwd_workspace_bytes(1000, 64) == 0
    need = e3j.e3j_layer_norm_bwd_workspace_bytes(50000, 64)
    assert need > 0 and norm_bwd(rows=50000, n=64) == NO_ROOM and norm_bwd(rows=50000, n=64, ws=P, size=need - 256) == NO_ROOM
    for bad in ((0, 5, 0, 3, 0), (0, -1, 4, 3, 0), (2, 5, 4, 3, 0)):
        assert LIB.e3j_linear_bwd_workspace_bytes(*bad) == 0
    assert LIB.e3j_layer_norm_bwd_workspace_bytes(0, 5, 5000) == 0


def test_status_wants_a_place():
    assert LIB.e3j_linear_status(None) == BAD


def test_the_binding_names_what_is_wrong():
    x = torch.zeros(4, 3)
    for call in (lambda: e3j.e3j_linear_fwd(x, x), lambda: e3j.e3j_linear_bwd(x, x, None, x), lambda: e3j.e3j_layer_norm_fwd(x),
                 lambda: e3j.e3j_layer_norm_bwd(x, None, None, x), lambda: e3j.e3j_linear_fwd([1.0], x)):
        with pytest.raises(TypeError, match="x must be a CUDA tensor"):
            call()


def test_a_double_arrives_wherever_it_stands():
    e3j._torch()
    if e3j._native is None:
        pytest.skip("_marshal was not built")
    seen = []
    kinds = [ctypes.c_int, ctypes.c_int64, ctypes.c_void_p, ctypes.c_double, ctypes.c_int] + [ctypes.c_void_p] * 6 + [ctypes.c_size_t]
    f = ctypes.CFUNCTYPE(ctypes.c_int, *kinds)(lambda *a: seen.append(a) or -3)
    address = ctypes.cast(f, ctypes.c_void_p).value
    assert e3j._native.call_real(1e-5, address, 1, -7, None, 2, *range(11, 17), 99) == -3
    assert seen == [(1, -7, None, 1e-5, 2, 11, 12, 13, 14, 15, 16, 99)]
    for bad in (("x", address), (1.0,), (1.0, 2.0), (1.0, address, 1.5)):
        with pytest.raises(TypeError):
            e3j._native.call_real(*bad)
    assert e3j._native.same_device(torch.zeros(3), None) == -1 and e3j._native.same_device(1) == -1


def test_a_count_of_real_rows_off_its_alignment():
    for n_real in (P + 1, P + 2):
        assert linear_fwd(n_real=n_real) == BAD
        assert LIB.e3j_linear_bwd(0, 5, 4, 3, P, P, P, P, 1, n_real, P, P, P, None, 0, None) == BAD
        assert LIB.e3j_layer_norm_fwd(0, 5, 4, P, P, P, 1e-5, 1, n_real, P, None) == BAD
        assert LIB.e3j_layer_norm_bwd(0, 5, 4, P, P, P, P, 1e-5, 1, n_real, P, P, P, None, 0, None) == BAD
