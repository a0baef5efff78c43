"""Microscaled 4-bit linears and the layer norm in front of them, with their gradients, as a program that runs or tunes a
UNet of this family calls them.

A microscaled 4-bit (MXFP4) matrix holds every 32 consecutive values of a row as e2m1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and
their negatives) times one power of two: the exponent of the block's largest magnitude less 2, -127 at least; a code is
the nearest value, ties to the even code, magnitudes past 6 become 6.  A block that holds an infinity or a NaN stands for NaN.

Widths, token counts and distributions are those of the repository's own benchmark (channel levels 320 / 640 / 1280, a text
context of 77 x 2048, activations N(0, 1) with one entry in a hundred ten times as large, weights N(0, 0.02^2)); what lies
beyond them is generic.  A case is one of these kinds:

  store    a 16-bit tensor written down in MXFP4 and read back, as a skip connection that is kept in 4 bits
  linear   y = mx(x) mx(W)^T + bias (+ residual): the activations are quantised in the call, the weights once before it
  norm     the same behind a layer norm, whose output goes into MXFP4 directly
  grad     the gradient of that linear with respect to its input, the quantiser of x passed straight through: dx = dy mx(W)
  train    layer norm for training: the forward pass, and dx (+ the skip connection's gradient), dweight and dbias
"""
import math

import torch

own = False

EPS = 1e-5
DT = {"f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # first linear of the time embedding for one image: the smallest call, all latency
        dict(name="linear_1_row_320_1280", kind="linear", M=1, K=320, N=1280, dtype="f16", residual=False),
        # eight rows against a large weight: the weight is read once from memory
        dict(name="linear_8_rows_5120_20480_bf16", kind="linear", M=8, K=5120, N=20480, dtype="bf16", residual=False),
        # output projection of an attention at the 1280-channel level, four images, skip connection added
        dict(name="linear_4096_1280_1280_res", kind="linear", M=4096, K=1280, N=1280, dtype="f16", residual=True),
        # a large product: the matrix units are the limit
        dict(name="linear_8192_8192_8192_bf16", kind="linear", M=8192, K=8192, N=8192, dtype="bf16", residual=False),
        # norm and feed-forward projection at the 640-channel level, four images: the limit is what is written
        dict(name="norm_16384_640_5120", kind="norm", M=16384, K=640, N=5120, dtype="f16", params="f16"),
        # norm and stacked q, k, v of three images of 26 x 38 positions, norm parameters kept in 32 bits
        dict(name="norm_2964_1280_3840_bf16", kind="norm", M=2964, K=1280, N=3840, dtype="bf16", params="f32"),
        # gradient through the feed-forward projection at the 1280-channel level
        dict(name="grad_4096_1280_10240_bf16", kind="grad", M=4096, K=1280, N=10240, dtype="bf16"),
        # gradient through the K projection of a text context of four prompts
        dict(name="grad_308_2048_640", kind="grad", M=308, K=2048, N=640, dtype="f16"),
        # a skip connection of the 640-channel level, four images
        dict(name="store_16384_640", kind="store", M=16384, K=640, dtype="f16"),
        # an odd number of rows, a width that is no multiple of 64
        dict(name="store_1001_1952_bf16", kind="store", M=1001, K=1952, dtype="bf16"),
        # norm of the 640-channel level, four images
        dict(name="train_16384_640", kind="train", M=16384, K=640, dtype="f16", params="f32", residual=True),
        # norm of the 1280-channel level, three images of 26 x 38 positions
        dict(name="train_2964_1280_bf16", kind="train", M=2964, K=1280, dtype="bf16", params="bf16", residual=False),
    ]


def _log(rng, lo, hi, step):
    """A multiple of `step` between lo and hi, spread over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return int(min(max(round(v / step) * step, -(-lo // step) * step), hi // step * step))


def draw(rng):
    most = max(work(c)["flops"] for c in listed())
    moved = max(work(c)["bytes"] for c in listed())
    while True:
        kind = rng.choice(("linear", "linear", "linear", "norm", "norm", "grad", "grad", "store", "train", "train"))
        dtype = rng.choice(("f16", "bf16"))
        if kind in ("linear", "norm", "grad"):
            c = dict(kind=kind, M=_log(rng, 1, 16384, 1), K=_log(rng, 64, 8192, 32), N=_log(rng, 32, 20480, rng.choice((1, 8, 32))), dtype=dtype)
            if kind == "linear":
                c["residual"] = rng.random() < 0.5
        elif kind == "store":
            c = dict(kind=kind, M=_log(rng, 1, 32768, 1), K=_log(rng, 32, 8192, 32), dtype=dtype)
        else:
            c = dict(kind=kind, M=_log(rng, 1, 32768, 1), K=_log(rng, 8, 8192, rng.choice((1, 8))), dtype=dtype, residual=rng.random() < 0.5)
        if kind in ("norm", "train"):
            c["params"] = rng.choice((dtype, "f32"))
        w = work(c)
        if w["flops"] <= most and w["bytes"] <= moved:
            return c


# ---------------------------------------------------------------------------------------------------------- inputs

def _inputs(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    dt = DT[case["dtype"]]
    M, K = case["M"], case["K"]

    def normal(*shape, std=1.0, mean=0.0):
        return torch.randn(*shape, generator=gen, device=dev) * std + mean

    def acts(*shape):
        x = normal(*shape)
        x[torch.rand(*shape, generator=gen, device=dev) < 0.01] *= 10.0
        return x.to(dt)

    s = {}
    if case["kind"] == "grad":
        s["dy"] = acts(M, case["N"])
    else:
        s["x"] = acts(M, K)
    if case["kind"] in ("linear", "norm", "grad"):
        s["w16"] = normal(case["N"], K, std=0.02).to(dt)
    if case["kind"] in ("linear", "norm"):
        s["bias"] = normal(case["N"], std=0.01).to(dt)
    if case["kind"] in ("norm", "train"):
        pt = torch.float32 if case["params"] == "f32" else dt
        s["gain"], s["shift"] = normal(K, std=0.1, mean=1.0).to(pt), normal(K, std=0.1).to(pt)
    if case["kind"] == "train":
        s["dy"] = acts(M, K)
    if case.get("residual"):
        s["res"] = acts(M, case["N"] if case["kind"] == "linear" else K)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["kind"] = case["kind"]
    if "w16" in s:
        w = s.pop("w16")  # the layer's weights, quantised when the model is loaded
        if own:
            import paper_2405_17873_amd as mq
            s["w"] = mq.mx_quantize_weights(w)
        else:
            s["w"] = _mx(w.float())
    return s


# ------------------------------------------------------------------------------------------------- plain forms, 32 bits

def _mx(v):
    """What a float32 matrix stands for after quantisation to MXFP4."""
    b = v.reshape(v.shape[0], -1, 32)
    top = b.abs().amax(-1, keepdim=True)
    e = top.view(torch.int32) >> 23                      # biased exponent: 0 for zero and subnormal, 255 for infinity and NaN
    s = (e - 2).clamp(min=0)
    q = b * ((254 - s) << 23).view(torch.float32)        # times 2^(127 - s), exact
    a = q.abs().clamp(max=6.0)
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    a = torch.round(a / step) * step
    scale = torch.where(s > 0, (s << 23).view(torch.float32), 2.0 ** -127)
    r = torch.where(q < 0, -a, a) * scale
    return torch.where(e == 255, float("nan"), r).reshape(v.shape)


def _norm(x, gain, shift):
    mean = x.mean(-1, keepdim=True)
    d = x - mean
    rstd = torch.rsqrt((d * d).mean(-1, keepdim=True) + EPS)
    return d * rstd, rstd, d * rstd * gain + shift


def _plain(s):
    kind = s["kind"]
    if kind == "store":
        return _mx(s["x"].float()).to(s["x"].dtype)
    if kind in ("linear", "norm"):
        x = s["x"].float()
        if kind == "norm":
            x = _norm(x, s["gain"].float(), s["shift"].float())[2]
        y = torch.matmul(_mx(x), s["w"].t()) + s["bias"].float()
        return (y + s["res"].float() if "res" in s else y).to(s["x"].dtype)
    if kind == "grad":
        return torch.matmul(s["dy"].float(), s["w"]).to(s["dy"].dtype)
    gain, dy = s["gain"].float(), s["dy"].float()
    xhat, rstd, y = _norm(s["x"].float(), gain, s["shift"].float())
    g = dy * gain
    dx = rstd * (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True))
    if "res" in s:
        dx = dx + s["res"].float()
    return dict(y=y.to(s["x"].dtype), dx=dx.to(s["x"].dtype), dweight=(dy * xhat).sum(0), dbias=dy.sum(0))


def run(s):
    if not own:
        return _plain(s)
    import paper_2405_17873_amd as mq
    kind = s["kind"]
    if kind == "store":
        return mq.mx_dequantize(mq.mx_quantize(s["x"]), s["x"].dtype)
    if kind == "linear":
        return mq.mx_linear(s["x"], s["w"], s["bias"], residual=s.get("res"))
    if kind == "norm":
        return mq.mx_linear(mq.layer_norm_mx(s["x"], s["gain"], s["shift"], EPS), s["w"], s["bias"], dtype=s["x"].dtype)
    if kind == "grad":
        return mq.mx_linear_grad(s["dy"], s["w"])
    y, mean, rstd = mq.layer_norm(s["x"], s["gain"], s["shift"], EPS, want_stats=True)
    dx, dweight, dbias = mq.layer_norm_grad(s["dy"], s["x"], s["gain"], mean, rstd, residual=s.get("res"))
    return dict(y=y, dx=dx, dweight=dweight, dbias=dbias)


def work(case):
    M, K, kind = case["M"], case["K"], case["kind"]
    if kind == "store":
        return {"bytes": 4 * M * K, "flops": 4 * M * K}
    if kind == "train":
        p = 4 if case["params"] == "f32" else 2
        # the forward pass reads x and writes y, the backward pass reads x, dy (and the skip's gradient) and writes dx
        return {"bytes": M * K * (10 + (2 if case["residual"] else 0)) + 2 * p * K + 8 * K, "flops": 24 * M * K}
    N = case["N"]
    weights = N * K // 2 + N * K // 32
    if kind == "grad":
        return {"bytes": 2 * M * N + weights + 2 * M * K, "flops": 2 * M * N * K}
    params = 2 * K * (4 if case["params"] == "f32" else 2) if kind == "norm" else 0
    return {"bytes": 2 * M * K + weights + 2 * N + 2 * M * N * (2 if case.get("residual") else 1) + params, "flops": 2 * M * N * K}


# ---------------------------------------------------------------------------------------------------------- 64 bits

def _exact_mx(v):
    """MXFP4 values of a float64 matrix, from the definition: the block's exponent by frexp, the codes by their borders."""
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=v.device)
    border = (grid[1:] + grid[:-1]) / 2
    b = v.reshape(v.shape[0], -1, 32)
    top = b.abs().amax(-1, keepdim=True)
    e = (torch.frexp(top)[1] - 3).clamp(min=-127)
    e = torch.where(top == 0, -127, e)
    unit = torch.ldexp(torch.ones_like(top), e)
    a = b.abs() / unit
    below, above = torch.bucketize(a, border), torch.bucketize(a, border, right=True)
    r = grid[torch.where(below == above, below, torch.where(below % 2 == 0, below, above))]  # between two: the even code
    r = torch.where(torch.isfinite(top), torch.where(b < 0, -r, r) * unit, float("nan"))
    return r.reshape(v.shape)


def exact(case, seed):
    s = _inputs(case, seed)
    f = {k: v.double() for k, v in s.items()}
    kind = case["kind"]
    if kind == "store":
        return _exact_mx(f["x"])
    if kind == "grad":
        return f["dy"] @ _exact_mx(f["w16"])
    if kind in ("norm", "train"):
        x = f["x"]
        var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
        rstd = 1.0 / torch.sqrt(var + EPS)
        xhat = (x - mean) * rstd
        y = xhat * f["gain"] + f["shift"]
    if kind != "train":
        out = _exact_mx(y if kind == "norm" else f["x"]) @ _exact_mx(f["w16"]).T + f["bias"]
        return out + f["res"] if "res" in f else out
    g = f["dy"] * f["gain"]
    K = case["K"]
    dx = (g - (g.sum(1, keepdim=True) + xhat * (g * xhat).sum(1, keepdim=True)) / K) * rstd
    if "res" in f:
        dx = dx + f["res"]
    return dict(y=y, dx=dx, dweight=torch.einsum("mk,mk->k", f["dy"], xhat), dbias=f["dy"].sum(0))
