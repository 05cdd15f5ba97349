"""The radial network's hidden layers: what is measured of the linear layer and of layer norm, and their plain forms.

A radial network maps every edge's distance embedding to the hidden activations h that e3j_conv_radial_* takes: linear
layers with bias and activation, some with a residual, some followed by a layer norm whose output goes through the
activation.  Rows are edges (or nodes, for the read-out of node scalars).  A case names one call:

  linear_fwd   y = act(x W + b) + residual
  linear_bwd   (grad_x, grad_W, grad_b) from x, W, b and grad_y
  norm_fwd     y = act(layer_norm(x) weight + bias)
  norm_bwd     (grad_x, grad_weight, grad_bias) from x, weight, bias and grad_y

rows, n_in and n_out are the sizes; n_real < rows makes the list a padded one: the count of real rows is on the device, the
rows behind it hold NaN and come back as zeros.  Inputs are N(0, 1) (grad_y too), W is N(0, 1 / n_in), layer norm's rows have
means and spreads of their own.
"""
import math

import torch

own = False

EPS = 1e-5
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}


def listed():
    return [
        # First layer of the network on a batch of small molecules: 8 radial basis functions to 64 hidden; latency.
        dict(name="linear_first_small", kind="linear_fwd", rows=1201, n_real=1201, n_in=8, n_out=64, act="silu", bias=True,
             residual=False, dtype="float32"),
        # The same size, backward of a hidden layer: a training step of a toy potential.
        dict(name="linear_bwd_small", kind="linear_bwd", rows=1201, n_real=1201, n_in=64, n_out=64, act="silu", bias=True,
             residual=False, dtype="float32"),
        # Hidden layer on all edges of the 3000-atom water box.
        dict(name="linear_hidden_water", kind="linear_fwd", rows=160900, n_real=160900, n_in=64, n_out=64, act="silu",
             bias=True, residual=False, dtype="float32"),
        # Its backward.
        dict(name="linear_hidden_water_bwd", kind="linear_bwd", rows=160900, n_real=160900, n_in=64, n_out=64, act="silu",
             bias=True, residual=False, dtype="float32"),
        # A wide residual block of a network trained in bfloat16.
        dict(name="linear_wide_bf16", kind="linear_fwd", rows=78000, n_real=78000, n_in=512, n_out=512, act="gelu", bias=True,
             residual=True, dtype="bfloat16"),
        # Odd widths and a padded edge list (fixed capacity, fewer real edges), backward in float32.
        dict(name="linear_padded_odd_bwd", kind="linear_bwd", rows=49157, n_real=41003, n_in=97, n_out=161, act="tanh",
             bias=True, residual=False, dtype="float32"),
        # Layer norm of one small molecule's edges; latency.
        dict(name="norm_small", kind="norm_fwd", rows=1201, n_real=1201, n_in=64, act="silu", affine=True, dtype="float32"),
        # Its backward.
        dict(name="norm_bwd_small", kind="norm_bwd", rows=1201, n_real=1201, n_in=64, act="silu", affine=True, dtype="float32"),
        # Layer norm and SiLU behind the hidden layer on the water box.
        dict(name="norm_water", kind="norm_fwd", rows=160900, n_real=160900, n_in=64, act="silu", affine=True, dtype="float32"),
        # Its backward, with the reduction of the weight's and the bias's gradients over all edges.
        dict(name="norm_water_bwd", kind="norm_bwd", rows=160900, n_real=160900, n_in=64, act="silu", affine=True,
             dtype="float32"),
        # A wide norm in bfloat16 over an odd number of rows.
        dict(name="norm_wide_bf16", kind="norm_fwd", rows=78001, n_real=78001, n_in=1024, act="none", affine=True,
             dtype="bfloat16"),
        # Odd width, padded list, backward in bfloat16.
        dict(name="norm_padded_odd_bwd", kind="norm_bwd", rows=49157, n_real=41003, n_in=385, act="gelu", affine=True,
             dtype="bfloat16"),
    ]


def _between(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    """Rows from one edge to a large box; widths from a single radial function to wide blocks, three in four of them whole
    multiples of 8; both types, all activations, with and without what is optional, a quarter of the lists padded."""
    kind = rng.choice(["linear_fwd", "linear_bwd", "norm_fwd", "norm_bwd"])
    linear = kind.startswith("linear")

    def width(low, high):
        n = _between(rng, low, high)
        return max(8, n // 8 * 8) if rng.random() < 0.75 else n

    while True:
        rows = _between(rng, 1, 160900)
        case = dict(kind=kind, rows=rows, n_real=rows if rng.random() < 0.75 else rng.randint(0, rows),
                    n_in=width(4, 512) if linear else width(8, 1024), act=rng.choice(["none", "silu", "tanh", "gelu"]),
                    dtype=rng.choice(["float32", "bfloat16"]))
        if linear:
            case |= dict(n_out=width(4, 512), bias=rng.random() < 0.75, residual=kind == "linear_fwd" and rng.random() < 0.5)
        else:
            case |= dict(affine=rng.random() < 0.75)
        need = work(case)
        if need["bytes"] <= 1.2e8 and need["flops"] <= 2e10:
            return case


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + 11)
    dtype, rows, n_in = TYPES[case["dtype"]], case["rows"], case["n_in"]
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    s = {"kind": case["kind"], "act": case["act"]}
    if case["kind"].startswith("linear"):
        n_out = case["n_out"]
        s["x"] = normal(rows, n_in)
        s["W"] = (normal(n_in, n_out) / math.sqrt(n_in)).to(dtype)
        s["b"] = (0.5 * normal(n_out)).to(dtype) if case["bias"] else None
        s["residual"] = normal(rows, n_out) if case["residual"] else None
        s["grad_y"] = normal(rows, n_out) if case["kind"] == "linear_bwd" else None
    else:
        s["x"] = normal(rows, n_in) * torch.exp(0.5 * normal(rows, 1)) + normal(rows, 1)
        s["weight"] = (1 + 0.3 * normal(n_in)).to(dtype) if case["affine"] else None
        s["bias"] = (0.3 * normal(n_in)).to(dtype) if case["affine"] else None
        s["grad_y"] = normal(rows, n_in) if case["kind"] == "norm_bwd" else None
    for name in ("x", "residual", "grad_y"):
        if s.get(name) is not None:
            s[name] = s[name].to(dtype)
            s[name][case["n_real"]:] = float("nan")
    s["n_real"] = torch.tensor([case["n_real"]], dtype=torch.int32, device="cuda") if case["n_real"] < rows else None
    return s


def _activation(z, name):
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "tanh":
        return torch.tanh(z)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _slope(z, name):
    if name == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if name == "tanh":
        return 1 - torch.square(torch.tanh(z))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def _plain(s):
    """The call in elementary operations, in 32 bits, rounded to the inputs' type at the end."""
    dtype = s["x"].dtype
    real = None if s["n_real"] is None else (torch.arange(s["x"].shape[0], device="cuda") < s["n_real"]).unsqueeze(1)

    def rows(t):   # padding rows as zeros
        return t.float() if real is None else torch.where(real, t.float(), 0.0)

    def wide(t):
        return None if t is None else t.float()

    x = rows(s["x"])
    if s["kind"].startswith("linear"):
        W, b = wide(s["W"]), wide(s["b"])
        if s["kind"] == "linear_fwd" or s["act"] != "none":
            z = x @ W
            z = z if b is None else z + b
        if s["kind"] == "linear_fwd":
            y = _activation(z, s["act"])
            y = y if s["residual"] is None else y + s["residual"].float()
            return rows(y).to(dtype)
        gz = rows(s["grad_y"]) if s["act"] == "none" else rows(s["grad_y"]) * _slope(z, s["act"])
        return (gz @ W.T).to(dtype), (x.T @ gz).to(dtype), None if b is None else gz.sum(0).to(dtype)
    weight, bias = wide(s["weight"]), wide(s["bias"])
    centred = x - x.mean(1, keepdim=True)
    inverse = torch.rsqrt(torch.square(centred).mean(1, keepdim=True) + EPS)
    xh = centred * inverse
    z = xh if weight is None else xh * weight + bias
    if s["kind"] == "norm_fwd":
        return rows(_activation(z, s["act"])).to(dtype)
    gz = rows(s["grad_y"]) if s["act"] == "none" else rows(s["grad_y"]) * _slope(z, s["act"])
    u = gz if weight is None else gz * weight
    gx = (u - u.mean(1, keepdim=True) - xh * (u * xh).mean(1, keepdim=True)) * inverse
    if weight is None:
        return rows(gx).to(dtype), None, None
    return rows(gx).to(dtype), (gz * xh).sum(0).to(dtype), gz.sum(0).to(dtype)


def run(state):
    s = state
    if not own:
        return _plain(s)
    import paper_2609_35099_b200 as e3j
    act = {"none": e3j.E3J_ACT_NONE, "silu": e3j.E3J_ACT_SILU, "tanh": e3j.E3J_ACT_TANH, "gelu": e3j.E3J_ACT_GELU}[s["act"]]
    if s["kind"] == "linear_fwd":
        return e3j.e3j_linear_fwd(s["x"], s["W"], s["b"], s["residual"], act, n_real=s["n_real"])
    if s["kind"] == "linear_bwd":
        return e3j.e3j_linear_bwd(s["x"], s["W"], s["b"], s["grad_y"], act, n_real=s["n_real"], grad_b=s["b"] is not None)
    if s["kind"] == "norm_fwd":
        return e3j.e3j_layer_norm_fwd(s["x"], s["weight"], s["bias"], EPS, act, n_real=s["n_real"])
    affine = s["weight"] is not None
    return e3j.e3j_layer_norm_bwd(s["x"], s["weight"], s["bias"], s["grad_y"], EPS, act, n_real=s["n_real"],
                                  grad_weight=affine, grad_bias=affine)


def work(case):
    """Each input that the real rows need read once, each output (padding rows too) written once; the products' operations,
    and about 10 (forward) and 25 (backward) an element for layer norm."""
    size = 4 if case["dtype"] == "float32" else 2
    rows, real, n_in = case["rows"], case["n_real"], case["n_in"]
    if case["kind"].startswith("linear"):
        n_out = case["n_out"]
        weights = n_in * n_out + (n_out if case["bias"] else 0)
        if case["kind"] == "linear_fwd":
            values = real * (n_in + (n_out if case["residual"] else 0)) + weights + rows * n_out
            return {"bytes": size * values, "flops": 2 * real * n_in * n_out}
        values = real * (n_in + n_out) + 2 * weights + rows * n_in
        return {"bytes": size * values, "flops": (4 if case["act"] == "none" else 6) * real * n_in * n_out}
    back = case["kind"] == "norm_bwd"
    values = real * n_in * (2 if back else 1) + rows * n_in + ((4 if back else 2) * n_in if case["affine"] else 0)
    return {"bytes": size * values, "flops": (25 if back else 10) * real * n_in}


def exact(case, seed):
    """The definitions in 64 bits: activations through the logistic function and the complementary error function, layer norm
    through two moments about the mean, gradients as products with the Jacobians."""
    s = prepare(case, seed)
    real, rows, n_in = case["n_real"], case["rows"], case["n_in"]
    f64 = torch.float64
    cut = {k: s[k][:real].to(f64) for k in ("x", "residual", "grad_y") if s.get(k) is not None}
    full = {k: s[k].to(f64) for k in ("W", "b", "weight", "bias") if s.get(k) is not None}

    def act(z):
        return {"none": lambda: z, "silu": lambda: z * torch.sigmoid(z), "tanh": lambda: 2 * torch.sigmoid(2 * z) - 1,
                "gelu": lambda: 0.5 * z * torch.erfc(-z / math.sqrt(2.0))}[case["act"]]()

    def slope(z):
        if case["act"] == "silu":
            return torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)
        if case["act"] == "tanh":
            return 1 / torch.cosh(z) ** 2
        if case["act"] == "gelu":
            return 0.5 * torch.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        return torch.ones_like(z)

    def padded(t):
        out = torch.zeros(rows, t.shape[1], dtype=f64, device=t.device)
        out[:real] = t
        return out

    x = cut["x"]
    if case["kind"].startswith("linear"):
        z = torch.einsum("rk,km->rm", x, full["W"]) + (full["b"] if "b" in full else 0)
        if case["kind"] == "linear_fwd":
            return padded(act(z) + (cut["residual"] if "residual" in cut else 0))
        gz = cut["grad_y"] * slope(z)
        return (padded(torch.einsum("rm,km->rk", gz, full["W"])), torch.einsum("rk,rm->km", x, gz),
                gz.sum(0) if "b" in full else None)
    mean = x.sum(1, keepdim=True) / n_in
    spread = torch.sqrt(((x - mean) ** 2).sum(1, keepdim=True) / n_in + EPS)
    xh = (x - mean) / spread
    weight = full.get("weight", torch.ones(n_in, dtype=f64, device=x.device))
    z = torch.addcmul(full["bias"], xh, weight) if "bias" in full else xh
    if case["kind"] == "norm_fwd":
        return padded(act(z))
    gz = cut["grad_y"] * slope(z)
    u = gz * weight
    along = torch.einsum("rk,rk->r", u, xh).unsqueeze(1) / n_in
    gx = (u - u.sum(1, keepdim=True) / n_in - along * xh) / spread
    affine = case["affine"]
    return padded(gx), (gz * xh).sum(0) if affine else None, gz.sum(0) if affine else None
