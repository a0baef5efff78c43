"""What a transformer block has around its microscaled 4-bit linears, with gradients, as a program that runs or tunes such a network calls it.

  heads        norm of every query and key head and the rotation by position, in one pass over the stacked output of the q, k (, v) linear
  heads_train  the same and its gradient: dx, and the norm weights' sums over rows and heads
  act          a linear with MXFP4 weights whose epilogue has bias, activation and residual, or a gated activation (value * act(gate))
  act_train    the same for training, one microbatch forward, the one before it backward: the linear's own result is kept; from the kept one come the gradient
               behind the activation and the bias' gradient
  experts      rows sorted by expert, each times its own expert's MXFP4 weights; the number of rows of each is known on the GPU alone
  experts_train  the same without an activation, and the gradient with respect to the rows

Widths, token counts and distributions are those of the repository's own benchmark (channel levels 320 / 640 / 1280, heads of 64, a text context of 77 x 2048,
images of 64 x 64 and 32 x 32 positions or 26 x 38; activations N(0, 1) with one entry in a hundred ten times as large, weights N(0, 0.02^2)); what lies
beyond them is generic.  Frequencies of a rotation are theta^(-i/n) over the n pairs of an axis; positions are whole numbers.  MXFP4: 32 consecutive values of a row
as e2m1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) times one power of two, the exponent of the block's largest magnitude less 2, -127 at least;
nearest value, ties to the even code, magnitudes past 6 become 6; a block that holds an infinity or a NaN stands for NaN.
"""
import math

import torch

own = False

EPS = 1e-6
THETA = 10000.0
DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one new token of a sequence far along: the smallest call, all latency
        dict(name="heads_1_row_20_20_64", kind="heads", M=1, q=20, k=20, D=64, sections="32", interleaved=False, far=100000, dtype="bf16", params="bf16"),
        # eight frames of 64 x 64 positions at the 1280-channel width, three axes of positions
        dict(name="heads_32768_20_20_64_3_axes", kind="heads", M=32768, q=20, k=20, D=64, sections="8,12,12", interleaved=True, far=0, dtype="bf16", params="f32"),
        # training at 64 x 64 positions, four query heads to a key head, half-split pairs
        dict(name="heads_train_4096_32_8_128", kind="heads_train", M=4096, q=32, k=8, D=128, sections="64", interleaved=False, far=0, dtype="bf16", params="f32"),
        # three images of 26 x 38 positions, heads of 80 of which 64 turn, two axes
        dict(name="heads_train_2964_16_16_80", kind="heads_train", M=2964, q=16, k=16, D=80, sections="16,16", interleaved=True, far=0, dtype="f16", params="f16"),
        # eight rows through a linear and its activation: latency and the weights
        dict(name="act_8_1280_5120_gelu", kind="act", M=8, K=1280, N=5120, act="gelu", gated=False, residual=False, dtype="f16"),
        # gated feed-forward projection at the 640-channel level, four images
        dict(name="act_16384_640_5120_geglu", kind="act", M=16384, K=640, N=5120, act="gelu", gated=True, residual=False, dtype="f16"),
        # a large gated projection: the matrix units are the limit
        dict(name="act_8192_4096_16384_swiglu_bf16", kind="act", M=8192, K=4096, N=16384, act="silu", gated=True, residual=False, dtype="bf16"),
        # three images of 26 x 38 positions, activation and residual
        dict(name="act_train_2964_1280_1280_res", kind="act_train", M=2964, K=1280, N=1280, act="gelu_tanh", gated=False, residual=True, dtype="bf16"),
        # tuning through the gated projection of the 1280-channel level, four images
        dict(name="act_train_4096_1280_10240_geglu", kind="act_train", M=4096, K=1280, N=10240, act="gelu", gated=True, residual=False, dtype="bf16"),
        # eight tokens, four experts each out of 32: a row or two for an expert, the weights are what counts
        dict(name="experts_32_of_32_2048_2560", kind="experts", M=32, E=32, K=2048, N=2560, act="silu", gated=True, dtype="bf16"),
        # a batch of prompts, eight experts, ragged
        dict(name="experts_16384_of_8_2048_8192", kind="experts", M=16384, E=8, K=2048, N=8192, act="silu", gated=True, dtype="bf16"),
        # tuning through experts, many of them short
        dict(name="experts_train_4001_of_16_1280_2048", kind="experts_train", M=4001, E=16, K=1280, N=2048, act="", gated=False, dtype="f16"),
    ]


def _log(rng, lo, hi, step):
    """A multiple of `step` between lo and hi, spread over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return int(min(max(round(v / step) * step, -(-lo // step) * step), hi // step * step))


def _sections(rng, D):
    """Pairs of each axis: a multiple of four in all, no more than a head has."""
    pairs = rng.choice((D // 2 // 4, D // 2 // 4, max(1, D // 4 // 4))) * 4
    axes = rng.choice((1, 1, 2, 3))
    cuts = sorted(rng.randrange(pairs + 1) for _ in range(axes - 1))
    return ",".join(str(b - a) for a, b in zip([0] + cuts, cuts + [pairs]))


def draw(rng):
    cases = listed()
    most = max(work(c)["flops"] for c in cases)
    moved = max(work(c)["bytes"] for c in cases)
    while True:
        kind = rng.choice(("heads", "heads_train", "act", "act_train", "experts", "experts_train"))
        dtype = rng.choice(("f16", "bf16"))
        if kind in ("heads", "heads_train"):
            D = rng.choice((32, 40, 64, 64, 72, 80, 96, 128, 128, 160, 256))
            k = rng.choice((1, 2, 5, 8, 10, 16, 20))
            c = dict(kind=kind, M=_log(rng, 1, 32768, 1), q=k * rng.choice((1, 1, 2, 4, 7)), k=k, D=D, sections=_sections(rng, D), interleaved=rng.random() < 0.5,
                     far=rng.choice((0, 0, 5000, 1000000)), dtype=dtype, params=rng.choice((dtype, "f32")))
        else:
            gated = kind != "experts_train" and rng.random() < 0.5
            c = dict(kind=kind, K=_log(rng, 64, 8192, 32), act=rng.choice(("gelu", "gelu_tanh", "silu")), gated=gated, dtype=dtype)
            if kind in ("act", "act_train"):
                c.update(M=_log(rng, 1, 16384, 1), N=_log(rng, 64, 20480, 64 if gated else rng.choice((1, 8, 32))), residual=not gated and rng.random() < 0.5)
            else:
                c.update(M=_log(rng, 1, 16384, 1), E=rng.choice((1, 4, 8, 16, 32, 64)), N=_log(rng, 64, 8192, 64 if gated else 32))
                if kind == "experts_train" or rng.random() < 0.3:
                    c.update(act="", gated=False)
        w = work(c)
        if w["flops"] <= most and w["bytes"] <= moved and c.get("E", 1) * c.get("N", 1) * c.get("K", 1) <= 1 << 29:
            return c


# ---------------------------------------------------------------------------------------------------------- inputs

def _inputs(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    dt = DT[case["dtype"]]
    M, kind = case["M"], case["kind"]

    def normal(*shape, std=1.0, mean=0.0):
        return torch.randn(*shape, generator=gen, device=dev) * std + mean

    def acts(*shape):
        x = normal(*shape)
        x[torch.rand(*shape, generator=gen, device=dev) < 0.01] *= 10.0
        return x.to(dt)

    s = {}
    if kind in ("heads", "heads_train"):
        width = (case["q"] + case["k"]) * case["D"]
        s["x"] = acts(M, width)
        pt = DT[case["params"]]
        s["qw"], s["kw"] = normal(case["D"], std=0.1, mean=1.0).to(pt), normal(case["D"], std=0.1, mean=1.0).to(pt)
        axes = case["sections"].count(",") + 1
        row = torch.arange(M, device=dev)
        side = max(1, math.isqrt(M // 8 if axes == 3 else M))
        at = {1: [row], 2: [row // side, row % side], 3: [row // (side * side), row // side % side, row % side]}[axes]
        start = torch.randint(case["far"], 2 * case["far"], (1,), generator=gen, device=dev) if case["far"] else 0
        s["pos"] = (torch.stack(at, 1) + start).to(torch.int32)
        if kind == "heads_train":
            s["dy"] = acts(M, width)
        return s
    K, N, E = case["K"], case["N"], case.get("E", 1)
    s["x"] = acts(M, K)
    s["w16"] = normal(E * N, K, std=0.02 if K > 1000 else K ** -0.5).to(dt)
    s["bias"] = normal(E, N, std=0.01).to(dt)
    if "E" in case:
        # shares of the experts as a router gives them: uneven, some without a row
        share = torch.rand(E, generator=gen, device=dev).double() ** 2
        to = torch.multinomial(share, M, replacement=True, generator=gen)
        s["sizes"] = torch.bincount(to, minlength=E)
    if kind == "act_train":
        s["dy"] = acts(M, N // 2 if case["gated"] else N)
        s["kept"] = acts(M, N)
    if kind == "experts_train":
        s["dy"] = acts(M, N)
    if case.get("residual"):
        s["res"] = acts(M, N)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    kind = case["kind"]
    if own:
        import paper_2405_17873_amd as mq
    if kind in ("heads", "heads_train"):
        sections = [int(n) for n in case["sections"].split(",")]
        if own:
            s["rotary"] = mq.rotary(sections, THETA, interleaved=case["interleaved"], device=s["x"].device)
        else:
            f = [THETA ** (-i / n) for n in sections for i in range(n)]
            s["freq"] = torch.tensor(f, dtype=torch.float64, device=s["x"].device)
            s["axis"] = torch.tensor([a for a, n in enumerate(sections) for _ in range(n)], device=s["x"].device)
        return s
    w = s.pop("w16")  # the weights, quantised when the model is loaded
    if "E" in case:
        s["offsets"] = torch.nn.functional.pad(s["sizes"].cumsum(0), (1, 0)).to(torch.int32)
        if own:
            s["w"] = mq.mx_quantize_experts(w.view(case["E"], case["N"], case["K"]))
        else:
            s["w"] = _mx(w.float()).view(case["E"], case["N"], case["K"])
            s["ends"] = s["offsets"].tolist()
    else:
        s["bias"] = s["bias"][0].clone()
        s["w"] = mq.mx_quantize_weights(w) if own else _mx(w.float())
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


def _act(a, name):
    """(act(a), its slope)"""
    if name == "gelu":
        below = 0.5 * (1.0 + torch.erf(a * math.sqrt(0.5)))
        return a * below, below + a * torch.exp(-0.5 * a * a) * (1.0 / math.sqrt(2.0 * math.pi))
    c, d = (1.0, 0.0) if name == "silu" else (2.0 * math.sqrt(2.0 / math.pi), 2.0 * math.sqrt(2.0 / math.pi) * 0.044715)
    s = 1.0 / (1.0 + torch.exp(-a * (c + d * a * a)))
    return a * s, s + a * s * (1.0 - s) * (c + 3.0 * d * a * a)


def _turn(u, cos, sin, interleaved):
    """u [M, heads, D]: its first 2 P values in pairs, turned; cos, sin [M, 1, P]."""
    P = cos.shape[-1]
    a, b = (u[..., 0:2 * P:2], u[..., 1:2 * P:2]) if interleaved else (u[..., :P], u[..., P:2 * P])
    c, d = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((c, d), -1).flatten(-2) if interleaved else torch.cat((c, d), -1)
    return torch.cat((turned, u[..., 2 * P:]), -1)


def _plain_heads(s, case):
    x, M, q = s["x"], case["M"], case["q"]
    angle = s["pos"][:, s["axis"]].double() * s["freq"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    v = x.float().view(M, -1, case["D"])
    rstd = torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)
    xhat = v * rstd
    w = torch.cat((s["qw"].float().expand(q, -1), s["kw"].float().expand(case["k"], -1)))
    y = _turn(xhat * w, cos, sin, case["interleaved"]).reshape(M, -1).to(x.dtype)
    if case["kind"] == "heads":
        return y
    g = _turn(s["dy"].float().view(M, -1, case["D"]), cos, -sin, case["interleaved"])
    dw = (g * xhat).sum(0)
    g = g * w
    dx = rstd * (g - xhat * (g * xhat).mean(-1, keepdim=True))
    return dict(y=y, dx=dx.reshape(M, -1).to(x.dtype), dq_weight=dw[:q].sum(0), dk_weight=dw[q:].sum(0))


def _activated(a, case):
    if not case["act"]:
        return a
    if not case["gated"]:
        return _act(a, case["act"])[0]
    v, g = a.chunk(2, -1)
    return v * _act(g, case["act"])[0]


def _plain(s):
    case, dt = s["case"], s["x"].dtype
    kind = case["kind"]
    if kind in ("heads", "heads_train"):
        return _plain_heads(s, case)
    x = _mx(s["x"].float())
    if kind in ("experts", "experts_train"):
        ends, rows = s["ends"], []
        for e in range(case["E"]):
            rows.append(_activated(torch.matmul(x[ends[e]:ends[e + 1]], s["w"][e].t()) + s["bias"][e].float(), case))
        y = torch.cat(rows).to(dt)
        if kind == "experts":
            return y
        return dict(y=y, dx=torch.cat([torch.matmul(s["dy"][ends[e]:ends[e + 1]].float(), s["w"][e]) for e in range(case["E"])]).to(dt))
    a = torch.matmul(x, s["w"].t()) + s["bias"].float()
    y = _activated(a, case)
    if "res" in s:
        y = y + s["res"].float()
    if kind == "act":
        return y.to(dt)
    kept, dy = s["kept"].float(), s["dy"].float()
    if case["gated"]:
        v, g = kept.chunk(2, -1)
        f, slope = _act(g, case["act"])
        da = torch.cat((dy * f, dy * v * slope), -1)
    else:
        da = dy * _act(kept, case["act"])[1]
    return dict(y=y.to(dt), pre=a.to(dt), da=da.to(dt), dbias=da.sum(0))


def run(s):
    if not own:
        return _plain(s)
    import paper_2405_17873_amd as mq
    case = s["case"]
    kind = case["kind"]
    if kind in ("heads", "heads_train"):
        args = dict(q_heads=case["q"], k_heads=case["k"], q_weight=s["qw"], k_weight=s["kw"], rotary=s["rotary"], positions=s["pos"], eps=EPS)
        y = mq.qk_norm_rope(s["x"], **args)
        if kind == "heads":
            return y
        dx, dq, dk = mq.qk_norm_rope_grad(s["dy"], s["x"], **args)
        return dict(y=y, dx=dx, dq_weight=dq, dk_weight=dk)
    if kind in ("experts", "experts_train"):
        y = mq.mx_linear_grouped(s["x"], s["w"], s["offsets"], s["bias"], act=case["act"] or None, gated=case["gated"])
        return y if kind == "experts" else dict(y=y, dx=mq.mx_linear_grouped_grad(s["dy"], s["w"], s["offsets"]))
    if kind == "act":
        return mq.mx_linear(s["x"], s["w"], s["bias"], residual=s.get("res"), act=case["act"], gated=case["gated"])
    y, pre = mq.mx_linear(s["x"], s["w"], s["bias"], residual=s.get("res"), act=case["act"], gated=case["gated"], want_pre=True)
    da, dbias = mq.act_grad(s["dy"], s["kept"], case["act"], gated=case["gated"])
    return dict(y=y, pre=pre, da=da, dbias=dbias)


def work(case):
    M, kind = case["M"], case["kind"]
    if kind in ("heads", "heads_train"):
        width = (case["q"] + case["k"]) * case["D"]
        p = 2 * case["D"] * (4 if case["params"] == "f32" else 2) + 4 * M * (case["sections"].count(",") + 1)
        # the forward pass reads x and writes y, the backward pass reads x and dy and writes dx
        return {"bytes": 4 * M * width + p, "flops": 8 * M * width} if kind == "heads" else {"bytes": 10 * M * width + p + 8 * case["D"], "flops": 26 * M * width}
    K, N, E = case["K"], case["N"], case.get("E", 1)
    # experts that have a row, on average: an expert's share is the square of a number between 0 and 1, times 3 / E
    live = E * sum(1.0 - (1.0 - 3.0 / max(E, 3) * ((i + 0.5) / 64) ** 2) ** M for i in range(64)) / 64 if E > 1 else 1
    weights = int(live * (N * K // 2 + N * K // 32 + 2 * N))
    out = N // 2 if case["gated"] else N
    moved = 2 * M * K + weights + 2 * M * out
    if kind == "act_train":  # the forward pass also writes the linear's own result; the backward pass reads it and dy and writes da
        moved += 2 * M * N + 2 * M * out + 4 * M * N + 4 * N
    if case.get("residual"):
        moved += 2 * M * N
    if kind == "experts_train":
        moved += 2 * M * K + weights + 2 * M * N
    return {"bytes": moved, "flops": 2 * M * N * K * (2 if kind == "experts_train" else 1)}


# ---------------------------------------------------------------------------------------------------------- 64 bits

def _exact_mx(v):
    """MXFP4 values of a float64 matrix, from the definition: the block's exponent by frexp, the codes by their borders."""
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=v.device)
    border = (grid[1:] + grid[:-1]) / 2
    b = v.reshape(v.shape[0], -1, 32)
    top = b.abs().amax(-1, keepdim=True)
    e = (torch.frexp(top)[1] - 3).clamp(min=-127)
    e = torch.where(top == 0, -127, e)
    unit = ((e.long() + 1023) << 52).view(torch.float64)  # 2^e
    a = b.abs() / unit
    below, above = torch.bucketize(a, border), torch.bucketize(a, border, right=True)
    r = grid[torch.where(below == above, below, torch.where(below % 2 == 0, below, above))]  # between two: the even code
    r = torch.where(torch.isfinite(top), torch.where(b < 0, -r, r) * unit, float("nan"))
    return r.reshape(v.shape)


def _exact_act(a, name):
    if name == "gelu":
        return a * 0.5 * torch.special.erfc(-a / math.sqrt(2.0))
    if name == "silu":
        return a / (1.0 + torch.exp(-a))
    return 0.5 * a * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (a + 0.044715 * a ** 3)))


def _exact_slope(a, name):
    if name == "gelu":
        return 0.5 * torch.special.erfc(-a / math.sqrt(2.0)) + a * torch.exp(-a * a / 2.0) / math.sqrt(2.0 * math.pi)
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-a))
        return s * (1.0 + a * (1.0 - s))
    k = math.sqrt(2.0 / math.pi)
    t = torch.tanh(k * (a + 0.044715 * a ** 3))
    return 0.5 * (1.0 + t) + 0.5 * a * (1.0 - t * t) * k * (1.0 + 3 * 0.044715 * a * a)


def _exact_heads(f, s, case):
    M, q, D = case["M"], case["q"], case["D"]
    heads = q + case["k"]
    sections = [int(n) for n in case["sections"].split(",")]
    P = sum(sections)
    # a matrix of a turn as a complex number for each row and pair
    parts = [s["pos"][:, a:a + 1].double() * torch.pow(torch.tensor(THETA, dtype=torch.float64, device=s["pos"].device), -torch.arange(n, device=s["pos"].device).double() / n)
             for a, n in enumerate(sections) if n]
    unit = torch.polar(torch.ones(M, P, dtype=torch.float64, device=s["pos"].device), torch.cat(parts, 1)) if P else None
    i = torch.arange(P, device=s["pos"].device)
    re, im = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + P)

    def turned(u, by):
        z = torch.complex(u[..., re], u[..., im]) * by[:, None]
        o = u.clone()
        o[..., re], o[..., im] = z.real, z.imag
        return o

    x = f["x"].view(M, heads, D)
    r = 1.0 / torch.sqrt(torch.einsum("mhd,mhd->mh", x, x)[..., None] / D + EPS)
    w = torch.cat((f["qw"].repeat(q, 1), f["kw"].repeat(case["k"], 1)))
    y = turned(x * r * w, unit).reshape(M, -1)
    if case["kind"] == "heads":
        return y
    g = turned(f["dy"].view(M, heads, D), unit.conj())
    dw = torch.einsum("mhd,mhd->hd", g, x * r)
    inner = torch.einsum("mhd,mhd->mh", g * w, x)[..., None]
    dx = r * g * w - x * r ** 3 * inner / D
    return dict(y=y, dx=dx.reshape(M, -1), dq_weight=dw[:q].sum(0), dk_weight=dw[q:].sum(0))


def exact(case, seed):
    s = _inputs(case, seed)
    f = {k: v.double() for k, v in s.items() if k not in ("pos", "sizes")}
    kind = case["kind"]
    if kind in ("heads", "heads_train"):
        return _exact_heads(f, s, case)
    N, E, gated, act = case["N"], case.get("E", 1), case["gated"], case["act"]
    x, w = _exact_mx(f["x"]), _exact_mx(f["w16"]).view(E, N, case["K"])
    sizes = s["sizes"].tolist() if "sizes" in s else [case["M"]]
    a = torch.cat([p @ w[e].T + f["bias"][e] for e, p in enumerate(x.split(sizes))])
    if act and gated:
        y = a[:, :N // 2] * _exact_act(a[:, N // 2:], act)
    else:
        y = _exact_act(a, act) if act else a
    if "res" in f:
        y = f["res"] + y
    if kind in ("act", "experts"):
        return y
    if kind == "experts_train":
        return dict(y=y, dx=torch.cat([p @ w[e] for e, p in enumerate(f["dy"].split(sizes))]))
    if gated:
        v, g = f["kept"][:, :N // 2], f["kept"][:, N // 2:]
        da = torch.cat((f["dy"] * _exact_act(g, act), f["dy"] * v * _exact_slope(g, act)), 1)
    else:
        da = f["dy"] * _exact_slope(f["kept"], act)
    return dict(y=y, pre=a, da=da, dbias=torch.einsum("mn->n", da))
