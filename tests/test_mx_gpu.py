"""Microscaled 4-bit linears, layer norm and their gradients on the GPU, against the float64 oracle.

Codes, scales and dequantised values are exact.  Other bounds count roundings: a 16-bit result is off by half a step of its type at most, an fp32
operation by U = 2^-24 of its result, and an addition inside a matrix instruction, which may cut off, by 2 U."""
import numpy as np
import pytest
import torch

from oracle import mx as omx

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
TYPES = (F16, BF16)


@pytest.fixture(scope="module")
def mq():
    import paper_2405_17873_amd as m
    m.load()
    assert torch.cuda.is_available()
    return m


def f64(t):
    return t.detach().cpu().double().numpy()


def half_step(y, dtype):
    """Largest rounding error of a 16-bit value (subnormals of fp16: half of 2^-24)."""
    return torch.finfo(dtype).eps / 2 * np.abs(y) + (2.0 ** -25 if dtype == F16 else 2.0 ** -133)


def rand(shape, dtype, seed, std=1.0, mean=0.0, outliers=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * std + mean
    if outliers:
        x[torch.rand(shape, generator=g) < 0.02] *= 12.0
    return x.to(dtype).cuda()


def spread(t, pad, offset=0):
    """The same matrix with rows `pad` further apart, `offset` elements into an allocation."""
    M, K = t.shape
    flat = torch.full((M * (K + pad) + offset + 8,), float("nan"), dtype=t.dtype, device=t.device)
    v = flat[offset:offset + M * (K + pad)].view(M, K + pad)[:, :K]
    v.copy_(t)
    return v


def within(got, want, bound, what="", dtype=None):
    """dtype: of a rounded result; what lies past its largest value is infinite."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    if dtype is not None:
        big = torch.finfo(dtype).max * (1 + torch.finfo(dtype).eps / 4)  # halfway to the next step
        past = np.abs(want) >= big
        assert np.array_equal(got[past], np.copysign(np.inf, want[past])), what
        got, want = np.where(past, 0.0, got), np.where(past, 0.0, want)
    assert got.shape == want.shape
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    ok = np.isnan(want) | (np.abs(got - want) <= bound)
    assert ok.all(), f"{what}: {np.count_nonzero(~ok)} of {ok.size}, first at {np.argwhere(~ok)[0]}, worst {np.nanmax(np.abs(got - want) / np.maximum(bound, 1e-300)):.2f} bounds"


# ---------------------------------------------------------------------------------------------------------- conversion

def check_quantize(mq, x):
    t = mq.mx_quantize(x)
    codes, scales = (v.cpu().numpy() for v in mq.mx_unpack(t))
    c, s = omx.quantize(f64(x))
    assert np.array_equal(scales, s)
    assert np.array_equal(codes, omx.flat(c))
    for dtype in TYPES:
        v = mq.mx_dequantize(t, dtype)
        with np.errstate(over="ignore"):
            want = torch.from_numpy(omx.decode(c, s)).to(dtype)
        assert torch.equal(torch.nan_to_num(v.cpu(), nan=12345.0), torch.nan_to_num(want, nan=12345.0))
    return t


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K", ((1, 32), (1, 320), (2, 64), (31, 96), (32, 256), (33, 288), (77, 2048), (130, 352), (257, 1952)))
def test_quantize_exact(mq, M, K, dtype):
    check_quantize(mq, rand((M, K), dtype, M * 1000 + K))


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_every_pattern(mq, dtype):
    """All 65536 bit patterns, each under several largest values of its block: borders, ties, subnormals, zeros of both signs, infinities and NaN."""
    p = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dtype).float()
    p = p[torch.isfinite(p)]
    blocks = []
    for top in (1.0, 1.5, 6.0, 7.5, 2.0 ** -14, 2.0 ** -20, 0.0):
        q = p[p.abs() <= (top if top else 1e38)]
        q = torch.cat([q, torch.zeros(-len(q) % 31)]).view(-1, 31)
        blocks.append(torch.cat([torch.full((len(q), 1), top), q], 1))
    x = torch.cat(blocks).to(dtype)
    x[5, 3], x[6, 0], x[7, 31] = float("inf"), float("-inf"), float("nan")
    x[8] = 0.0
    x[9] = -0.0
    check_quantize(mq, x.cuda())
    check_quantize(mq, x[:len(x) // 64 * 64].reshape(-1, 2048).cuda())


@pytest.mark.parametrize("pad,offset", ((0, 1), (1, 0), (8, 8), (3, 5), (40, 4)))
def test_quantize_views(mq, pad, offset):
    x = rand((37, 160), F16, 3)
    v = spread(x, pad, offset)
    t = check_quantize(mq, v)
    out = spread(torch.zeros(37, 160, dtype=F16, device="cuda"), pad, offset)
    mq.mx_dequantize(t, F16, out=out)
    assert torch.equal(out, mq.mx_dequantize(t, F16))


def test_pack_round_trip_and_top(mq):
    rng = np.random.default_rng(4)
    codes = torch.from_numpy(rng.integers(0, 256, (45, 80), dtype=np.uint8)).cuda()
    scales = torch.from_numpy(rng.integers(90, 140, (45, 5), dtype=np.uint8)).cuda()
    scales[3, 2], scales[:, 4] = 255, 255
    t = mq.mx_pack(codes, scales)
    c, s = mq.mx_unpack(t)
    assert torch.equal(s, scales)
    nan = (scales == 255).repeat_interleave(16, 1)
    assert torch.equal(c, torch.where(nan, 0, codes))
    finite = np.where(scales.cpu().numpy() == 255, 0, scales.cpu().numpy())
    assert np.array_equal(t.top.cpu().numpy(), finite.max(0))


def test_quantize_many_rows(mq):
    """More groups of 32 rows than one grid dimension holds."""
    M = 65535 * 32 + 37
    x = torch.zeros(M, 32, dtype=F16, device="cuda")
    tail = rand((64, 32), F16, 5)
    x[-64:] = tail
    t = mq.mx_quantize(x)
    v = mq.mx_dequantize(t, F16)
    assert torch.equal(v[-64:].cpu(), torch.from_numpy(omx.values(f64(tail))).half())
    assert not v[:-64].any()


# ------------------------------------------------------------------------------------------------------------- linear

def check_linear(mq, x, w, bias=None, res=None, out=None, packed=False):
    wq = mq.mx_quantize_weights(w)
    if packed:
        y = mq.mx_linear(mq.mx_quantize(x), wq, bias, residual=res, dtype=x.dtype, out=out)
    else:
        y = mq.mx_linear(x, wq, bias, residual=res, out=out)
    r64 = None if res is None else f64(res)
    want, mag = omx.linear(omx.values(f64(x)), omx.values(f64(w)), None if bias is None else f64(bias), r64)
    K = x.shape[1]
    acc = (K + 4) * 2 * U * mag
    within(f64(y), want, acc + half_step(np.abs(want) + acc, x.dtype), f"{tuple(x.shape)} x {w.shape[0]}", x.dtype)
    return y


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,N", ((1, 32, 1), (1, 320, 1280), (1, 64, 33), (2, 96, 8), (3, 5120, 40), (8, 2048, 640), (16, 352, 64), (17, 256, 130),
                                   (32, 1280, 96), (33, 288, 31), (64, 640, 320), (77, 2048, 100), (100, 480, 257), (129, 128, 129), (260, 1952, 520),
                                   (513, 320, 384), (700, 64, 1000)))
def test_linear(mq, M, K, N, dtype):
    x, w, b = rand((M, K), dtype, M + K + N), rand((N, K), dtype, N, 0.02), rand((N,), dtype, 9, 0.1)
    check_linear(mq, x, w, b)
    check_linear(mq, x, w, None, rand((M, N), dtype, 10), packed=True)


@pytest.mark.parametrize("M,K,N", ((8200, 704, 4104), (33000, 320, 1032), (2400, 640, 1944), (1190, 992, 4200), (6000, 1280, 1600)))
def test_linear_tiles(mq, M, K, N):
    """Several tiles for a workgroup, large ones and ones of another shape, last ones that are cut off on both sides; every element, with and without a
    residual, in place too."""
    x, w, b, r = rand((M, K), F16, 11), rand((N, K), F16, 12, 0.02), rand((N,), F16, 13, 0.1), rand((M, N), F16, 14)
    wq, xq = mq.mx_quantize_weights(w), mq.mx_quantize(x)
    xv, wv = mq.mx_dequantize(xq, BF16).double(), mq.mx_dequantize(wq, BF16).double()  # (exact: two significant bits)
    want, mag = xv @ wv.T + b.double(), xv.abs() @ wv.abs().T + b.double().abs()
    for res in (None, r):
        if res is not None:
            want, mag = want + res.double(), mag + res.double().abs()
        y = mq.mx_linear(xq, wq, b, residual=res, dtype=F16)
        acc = (K + 4) * 2 * U * mag
        bound = acc + torch.finfo(F16).eps / 2 * (want.abs() + acc) + 2.0 ** -25
        assert int(((y.double() - want).abs() > bound).sum()) == 0
    o = r.clone()
    assert torch.equal(mq.mx_linear(xq, wq, b, residual=o, dtype=F16, out=o), y)


@pytest.mark.parametrize("M", (1, 5, 40, 200))
def test_linear_views(mq, M):
    """Strides and alignments of every operand; the residual as the output itself; the output over the activations."""
    K, N = 160, 72
    x, w, b, r = rand((M, K), F16, 1), rand((N, K), F16, 2, 0.05), rand((N,), F16, 3), rand((M, N), F16, 4)
    want = check_linear(mq, x, w, b, r)
    wq = mq.mx_quantize_weights(w)
    for pad, offset in ((8, 8), (1, 0), (5, 3), (16, 4)):
        o = spread(torch.zeros_like(r), pad, offset)
        base = o._base if o._base is not None else o
        mq.mx_linear(spread(x, pad, offset), wq, spread(b.view(1, -1), pad, offset)[0], out=o, residual=spread(r, pad, offset))
        assert torch.equal(o, want)
        assert int(torch.isnan(base).sum()) == base.numel() - M * N  # nothing beside the result
    o = r.clone()
    assert mq.mx_linear(x, wq, b, out=o, residual=o) is o and torch.equal(o, want)
    both = torch.zeros(M, K, dtype=F16, device="cuda")
    both.copy_(x)
    mq.mx_linear(both, wq, b, residual=r, out=both[:, 8:8 + N])
    assert torch.equal(both[:, 8:8 + N], want)


@pytest.mark.parametrize("M", (1, 20, 150))
def test_linear_special_values(mq, M):
    K, N = 320, 64
    x, w = rand((M, K), F16, 6), rand((N, K), F16, 7, 0.02)
    x[0] = 0.0
    if M > 4:
        x[1, 5], x[2, 319], x[3] = float("nan"), float("inf"), 60000.0
        x[4, 64:96] = 2.0 ** -24
    w[3], w[5, 40] = 0.0, float("nan")
    y = f64(check_linear(mq, x, w))
    assert np.isnan(y[:, 5]).all() and (y[0, 3] == 0.0)
    if M > 4:
        assert np.isnan(y[1]).all() and np.isnan(y[2]).all() and np.isfinite(y[4, :5]).all()


def test_linear_deterministic_and_independent_of_neighbours(mq):
    """The same bits twice; a row's result does not depend on the rows beside it."""
    x, w = rand((70, 640), BF16, 8), rand((200, 640), BF16, 9, 0.02)
    wq = mq.mx_quantize_weights(w)
    y = mq.mx_linear(x, wq)
    assert torch.equal(y, mq.mx_linear(x, wq))
    x2 = x.clone()
    x2[1:] = float("nan")
    assert torch.equal(mq.mx_linear(x2, wq)[0], y[0])


def test_empty(mq):
    w = mq.mx_quantize_weights(rand((8, 64), F16, 1))
    x = torch.empty(0, 64, dtype=F16, device="cuda")
    assert mq.mx_linear(x, w).shape == (0, 8)
    assert mq.mx_linear(mq.mx_quantize(x), w).shape == (0, 8)
    assert mq.mx_linear_grad(torch.empty(0, 8, dtype=F16, device="cuda"), w).shape == (0, 64)
    y, mean, rstd = mq.layer_norm(x, want_stats=True)
    assert y.shape == (0, 64) and mean.shape == (0,)
    dx, dw, db = mq.layer_norm_grad(x, x, None, mean, rstd)
    assert dx.shape == (0, 64) and not dw.any() and not db.any() and dw.shape == (64,)
    assert mq.mx_dequantize(mq.layer_norm_mx(x)).shape == (0, 64)


def test_linear_offsets_past_32_bits(mq):
    """An output of more than 2^31 elements, and activations of more than 2^32 bytes: rows from both ends and the middle."""
    M, K, N = 70001, 32768, 32768
    x = torch.empty(M, K, dtype=F16, device="cuda")
    rows = [0, 1, 32767, 32768, 65535, 65536, 70000]
    x.fill_(1.0)
    some = rand((len(rows), K), F16, 11)
    x[rows] = some
    w = rand((N, K), F16, 12, 0.02)
    wq = mq.mx_quantize_weights(w)
    y = mq.mx_linear(x, wq)
    cols = torch.arange(0, N, 257)
    want, mag = omx.linear(omx.values(f64(some)), omx.values(f64(w[cols.cuda()])))
    acc = (K + 4) * 2 * U * mag
    within(f64(y[rows][:, cols.cuda()]), want, acc + half_step(np.abs(want) + acc, F16))
    dx = mq.mx_linear_grad(y, wq)
    g = f64(y[rows])
    kk = torch.cat([torch.arange(k, k + 32) for k in (0, 1024, K // 2, K - 32)])  # whole blocks
    want, mag = omx.linear_grad(g, omx.values(f64(w[:, kk.cuda()])))
    acc = (N + 8) * 2 * U * mag
    within(f64(dx[rows][:, kk.cuda()]), want, acc + half_step(np.abs(want) + acc, F16))


# --------------------------------------------------------------------------------------------------- gradient of linear

def check_grad(mq, dy, w, out=None):
    wq = mq.mx_quantize_weights(w)
    dx = mq.mx_linear_grad(dy, wq, out=out)
    v = omx.values(f64(w))
    want, mag = omx.linear_grad(f64(dy), v)
    top = np.nanmax(np.abs(v).reshape(v.shape[0], -1, 32), axis=(0, 2), initial=0.0)
    # products exact in fp32, N additions; what lies 2^-37 below a block column's largest may be missing (64 times that: 6 units against the scale)
    acc = (w.shape[0] + 8) * 2 * U * mag + np.abs(f64(dy)).sum(1, keepdims=True) * np.repeat(top, 32)[None] * 2.0 ** -36
    within(f64(dx), want, acc + half_step(np.abs(want) + acc, dy.dtype), f"{tuple(dy.shape)} x {w.shape[1]}", dy.dtype)
    return dx


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,N", ((1, 32, 1), (1, 1280, 320), (2, 64, 7), (31, 96, 33), (33, 352, 64), (64, 64, 65), (77, 2048, 100), (130, 320, 640),
                                   (257, 480, 130), (300, 160, 1001),
                                   (1, 160, 9000), (20, 608, 4104), (50, 1280, 5000), (100, 96, 8200), (400, 2080, 1320)))
def test_linear_grad(mq, M, K, N, dtype):
    check_grad(mq, rand((M, N), dtype, M + N), rand((N, K), dtype, K, 0.02))


@pytest.mark.parametrize("dtype", TYPES)
def test_linear_grad_scales(mq, dtype):
    """Weights from the smallest scale to the largest, in one column of blocks and across them."""
    w = rand((96, 256), dtype, 20)
    e = torch.linspace(-20, 8, 96).round() if dtype == F16 else torch.linspace(-120, 100, 96).round()
    w[:, :128] *= 2.0 ** e.view(-1, 1).to(dtype).cuda()
    w[:, 128:160] *= 2.0 ** -14 if dtype == F16 else 2.0 ** -125
    w[:, 160:192] = 0.0
    w[:, 192:224] *= 1000.0 if dtype == F16 else 1e30
    dy = rand((40, 96), dtype, 21)
    if dtype == BF16:
        dy *= 2.0 ** -10
    check_grad(mq, dy, w)


def test_linear_grad_views_and_special_values(mq):
    M, K, N = 45, 160, 72
    dy, w = rand((M, N), F16, 22), rand((N, K), F16, 23, 0.05)
    want = check_grad(mq, dy, w)
    wq = mq.mx_quantize_weights(w)
    for pad, offset in ((8, 8), (1, 0), (5, 3)):
        o = spread(torch.zeros(M, K, dtype=F16, device="cuda"), pad, offset)
        mq.mx_linear_grad(spread(dy, pad, offset), wq, out=o)  # (what lies between the rows is NaN)
        assert torch.equal(o, want)
        assert int(torch.isnan(o._base).sum()) == o._base.numel() - M * K
    dy[3], dy[7, 5], w[9, 40] = 0.0, float("nan"), float("inf")
    dx = f64(check_grad(mq, dy, w))
    assert np.isnan(dx[7]).all() and np.isnan(dx[:, 32:64]).all() and (dx[3, :32] == 0).all()


@pytest.mark.parametrize("M,K,N", ((1, 64, 650), (45, 160, 650), (9, 96, 2100), (300, 352, 1003)))
def test_linear_grad_rows_copied(mq, M, K, N):
    """Reductions of any length over rows at any distance: nothing beside a row gets into it."""
    dy, w = rand((M, N), F16, 24), rand((N, K), F16, 25, 0.05)
    want = check_grad(mq, dy, w)
    wq = mq.mx_quantize_weights(w)
    for pad, offset in ((0, 0), (8, 8), (1, 0), (5, 3)):
        assert torch.equal(mq.mx_linear_grad(spread(dy, pad, offset), wq), want)
    if M > 8:
        dy[4, N - 1], dy[8, 0] = float("nan"), float("inf")
        dx = f64(check_grad(mq, dy, w))
        assert np.isnan(dx[4]).all() and np.isfinite(dx[5:8]).all()


def test_linear_grad_wants_top(mq):
    with pytest.raises(ValueError):
        mq.mx_linear_grad(rand((2, 8), F16, 1), mq.mx_quantize(rand((8, 64), F16, 1)))


# ---------------------------------------------------------------------------------------------------------- layer norm

def depth(C):
    """Additions on the way of one value into a row's sum: up to 64 in a lane, 6 over lanes, 3 over waves."""
    return 64 + 9


def norm_bounds(x, w, eps):
    """(mean, rstd, bound of mean, relative bound of rstd) of the fp32 statistics."""
    mean, rstd = omx.norm_stats(x, eps)
    dm = (depth(x.shape[1]) + 2) * U * np.abs(x).mean(-1, keepdims=True)
    var = 1.0 / rstd ** 2
    dv = ((depth(x.shape[1]) + 5) * U * (var - eps) + dm ** 2) / var
    return mean, rstd, dm, 0.5 * dv + 4 * U


def norm_error(x, w, b, eps):
    """(exact normalised values, bound of their fp32 form)."""
    mean, rstd, dm, dr = norm_bounds(x, w, eps)
    d = x - mean
    y = d * rstd * w + b
    err = np.abs(w) * rstd * (dm + np.abs(d) * (dr + 4 * U)) + U * (np.abs(y) + np.abs(b) + np.abs(d * rstd * w))
    return y, err


def params(C, kind, dtype, seed):
    if kind == "none":
        return None, None
    t = F32 if kind == "f32" else dtype
    return rand((C,), F32, seed, 0.2, 1.0, False).to(t), rand((C,), F32, seed + 1, 0.2, 0.0, False).to(t)


def p64(w, b, C):
    return (np.ones(C) if w is None else f64(w)), (np.zeros(C) if b is None else f64(b))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,C", ((1, 1), (1, 320), (3, 8), (5, 33), (2, 255), (33, 512), (7, 520), (4, 1000), (9, 1280), (5, 1529), (6, 2048), (3, 2056),
                                 (2, 4099), (3, 8192), (2, 16384), (70, 640)))
@pytest.mark.parametrize("kind", ("16", "f32", "none"))
def test_layer_norm(mq, M, C, dtype, kind):
    x = rand((M, C), dtype, M + C, 1.0, 0.5)
    w, b = params(C, kind, dtype, 30)
    y, mean, rstd = mq.layer_norm(x, w, b, 1e-5, want_stats=True)
    X = f64(x)
    want, err = norm_error(X, *p64(w, b, C), 1e-5)
    within(f64(y), want, err + half_step(np.abs(want) + err, dtype))
    m, r, dm, dr = norm_bounds(X, None, 1e-5)
    within(f64(mean)[:, None], m, dm)
    within(f64(rstd)[:, None], r, r * dr)


def test_layer_norm_views_and_special_rows(mq):
    M, C = 9, 168
    x = rand((M, C), F16, 31)
    x[1] = 3.0          # no variance
    x[2] = 0.0
    x[3, 7], x[4, 0] = float("nan"), float("inf")
    x[5] = 60000.0
    x[5, ::2] = -60000.0
    x[6] = 2.0 ** -24
    w, b = params(C, "16", F16, 32)
    y = mq.layer_norm(x, w, b, 1e-5)
    Y = f64(y)
    assert np.isnan(Y[3]).all() and np.isnan(Y[4]).all()
    ok = [0, 1, 2, 5, 6, 7, 8]
    want, err = norm_error(f64(x)[ok], *p64(w, b, C), 1e-5)
    within(Y[ok], want, err + half_step(np.abs(want) + err, F16))
    for pad, offset in ((8, 8), (1, 0), (5, 3)):
        o = spread(torch.zeros_like(x), pad, offset)
        mq.layer_norm(spread(x, pad, offset), spread(w.view(1, -1), 0, offset)[0], spread(b.view(1, -1), 0, offset)[0], 1e-5, out=o)
        assert torch.equal(torch.nan_to_num(o), torch.nan_to_num(y))
    z = x.clone()
    mq.layer_norm(z, w, b, 1e-5, out=z)
    assert torch.equal(torch.nan_to_num(z), torch.nan_to_num(y))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,C,kind", ((1, 32, "16"), (1, 320, "f32"), (31, 96, "none"), (33, 640, "16"), (40, 1280, "f32"), (5, 2080, "16"), (3, 4096, "f32"),
                                      (2, 8224, "none"), (2, 16384, "16"), (65, 512, "16")))
def test_layer_norm_mx(mq, M, C, kind, dtype):
    """The kernel quantises fp32 values that lie within `err` of the exact ones: its scale is that of some such block, its codes lie between those
    of the interval's ends under that scale."""
    x = rand((M, C), dtype, M + C, 1.0, 0.3)
    w, b = params(C, kind, dtype, 33)
    t, mean, rstd = mq.layer_norm_mx(x, w, b, 1e-5, want_stats=True)
    codes, scales = (v.cpu().numpy() for v in mq.mx_unpack(t))
    y, err = norm_error(f64(x), *p64(w, b, C), 1e-5)
    lo, hi = np.maximum(np.abs(y) - err, 0.0), np.abs(y) + err
    assert (scales >= omx.scale_bytes(lo)).all() and (scales <= omx.scale_bytes(hi)).all()
    got = omx.decode(omx.unflat(codes), scales)
    assert (got >= omx.decode(omx.encode(y - err, scales), scales)).all() and (got <= omx.decode(omx.encode(y + err, scales), scales)).all()
    _, m2, r2 = mq.layer_norm(x, w, b, 1e-5, want_stats=True)
    assert torch.equal(mean, m2) and torch.equal(rstd, r2)
    # what is padding adds nothing to a product: the whole buffer beyond the real blocks is zero
    data = t.data.cpu().numpy()
    assert np.count_nonzero(data) <= np.count_nonzero(codes) + np.count_nonzero(scales)


def test_layer_norm_mx_into_linear(mq):
    """Rows with NaN stay what they are, and spoil no other row."""
    x, w = rand((70, 640), F16, 34), rand((96, 640), F16, 35, 0.02)
    g, s = params(640, "16", F16, 36)
    wq = mq.mx_quantize_weights(w)
    clean = mq.mx_linear(mq.layer_norm_mx(x, g, s), wq)
    x[5, 9], x[69, 3] = float("nan"), float("inf")
    y = mq.mx_linear(mq.layer_norm_mx(x, g, s), wq)
    assert torch.isnan(y[[5, 69]]).all()
    rest = [i for i in range(70) if i not in (5, 69)]
    assert torch.equal(y[rest], clean[rest])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,C", ((1, 1), (1, 320), (3, 8), (5, 33), (33, 512), (7, 520), (4, 1000), (300, 1280), (6, 2048), (3, 2056), (2, 4099), (3, 8192),
                                 (2, 16384), (2500, 640), (5000, 40)))
@pytest.mark.parametrize("kind,residual", (("16", False), ("f32", True), ("none", True)))
def test_layer_norm_grad(mq, M, C, dtype, kind, residual):
    x, dy = rand((M, C), dtype, M + C, 1.0, 0.5), rand((M, C), dtype, M + C + 1)
    res = rand((M, C), dtype, 40) if residual else None
    w, b = params(C, kind, dtype, 41)
    _, mean, rstd = mq.layer_norm(x, w, b, 1e-5, want_stats=True)
    dx, dw, db = mq.layer_norm_grad(dy, x, w, mean, rstd, residual=res)
    W, _ = p64(w, b, C)
    X, DY, mu, r = f64(x), f64(dy), f64(mean)[:, None], f64(rstd)[:, None]  # the statistics are inputs, taken as they are
    wantx, wantw, wantb = omx.norm_grad(DY, X, W, mu, r, None if res is None else f64(res))
    xh, g = (X - mu) * r, DY * W
    exh = 3 * U * (np.abs(X) + np.abs(mu)) * r
    n = depth(C)
    m1, m2 = np.abs(g).mean(-1, keepdims=True), (np.abs(g) * (np.abs(xh) + exh)).mean(-1, keepdims=True)
    e1, e2 = (n + 4) * U * m1, (n + 6) * U * m2 + (np.abs(g) * exh).mean(-1, keepdims=True)
    err = r * (6 * U * (np.abs(g) + m1 + np.abs(xh) * m2) + e1 + np.abs(xh) * e2 + exh * m2) + (2 * U * np.abs(f64(res)) if residual else 0) + 2 * U * np.abs(wantx)
    within(f64(dx), wantx, err + half_step(np.abs(wantx) + err, dtype), "dx")
    # rows of a workgroup's walk (M / 2048 of them, or all), 4 waves, then up to 32 workgroups in a run and 16 runs
    rows = M / 256 + 64
    within(f64(dw), wantw, ((rows + 2) * U * np.abs(DY * xh) + np.abs(DY) * exh).sum(0) + 2.0 ** -126, "dweight")
    within(f64(db), wantb, rows * U * np.abs(DY).sum(0) + 2.0 ** -126, "dbias")


def test_layer_norm_grad_views_and_aliases(mq):
    M, C = 50, 168
    x, dy, res = rand((M, C), F16, 42), rand((M, C), F16, 43), rand((M, C), F16, 44)
    w, b = params(C, "16", F16, 45)
    _, mean, rstd = mq.layer_norm(x, w, b, want_stats=True)
    want = mq.layer_norm_grad(dy, x, w, mean, rstd, residual=res)
    for pad, offset in ((8, 8), (1, 0), (5, 3)):
        o = spread(torch.zeros_like(x), pad, offset)
        got = mq.layer_norm_grad(spread(dy, pad, offset), spread(x, pad, offset), w, mean, rstd, residual=spread(res, pad, offset), out=o)
        assert all(torch.equal(a, c) for a, c in zip(got, want))
    for alias in ("dy", "res"):
        d, r = dy.clone(), res.clone()
        got = mq.layer_norm_grad(d, x, w, mean, rstd, residual=r, out=d if alias == "dy" else r)
        assert all(torch.equal(a, c) for a, c in zip(got, want))


# ------------------------------------------------------------------------------------------------- streams and graphs

def step(mq, x, gain, shift, wq, bias, dy, res):
    """Forward and backward of a norm and the linear behind it."""
    t, mean, rstd = mq.layer_norm_mx(x, gain, shift, want_stats=True)
    y = mq.mx_linear(t, wq, bias, dtype=x.dtype)
    dn = mq.mx_linear_grad(dy, wq)
    return (y,) + tuple(mq.layer_norm_grad(dn, x, gain, mean, rstd, residual=res)) + (mq.mx_linear(x, wq, bias, residual=dy),)


def test_graph_replays_and_side_stream(mq):
    M, C, N = 130, 320, 264
    make = lambda s: (rand((M, C), F16, s), rand((M, N), F16, s + 1), rand((M, C), F16, s + 2))
    gain, shift = params(C, "f32", F16, 50)
    wq, bias = mq.mx_quantize_weights(rand((N, C), F16, 51, 0.02)), rand((N,), F16, 52)
    x, dy, res = make(60)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        eager = step(mq, x, gain, shift, wq, bias, dy, res)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for a, c in zip(eager, step(mq, x, gain, shift, wq, bias, dy, res)):
        assert torch.equal(a, c)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(mq, x, gain, shift, wq, bias, dy, res)
    for s in (60, 70, 80, 60):
        for t, v in zip((x, dy, res), make(s)):
            t.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(captured, step(mq, x, gain, shift, wq, bias, dy, res)):
            assert torch.equal(a, c)


# ------------------------------------------------------------------------------------------------------------ together

def test_example_tunes_norms(mq):
    """The operators as a training loop uses them: the error against the 16-bit blocks falls."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "tune_norms.py")
    spec = importlib.util.spec_from_file_location("tune_norms", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    losses = m.tune(rows=500, width=160, hidden=608, blocks=2, steps=40, say=lambda *a, **k: None)
    assert all(np.isfinite(losses)) and np.mean(losses[-5:]) < np.mean(losses[:5])


# ------------------------------------------------------------------------------------------------------------ refusals

def test_overlapping_rows_are_refused(mq):
    """A broadcast gradient, rows that lie over one another, as every matrix operand."""
    M, K, N = 6, 64, 64
    w = mq.mx_quantize_weights(rand((N, K), F16, 80, 0.05))
    x = rand((M, K), F16, 81)
    _, mean, rstd = mq.layer_norm(x, want_stats=True)
    v = rand((256,), F16, 82)
    for t in (v[:64].expand(M, K), v.as_strided((M, K), (16, 1))):
        for call in (lambda: mq.mx_quantize(t), lambda: mq.mx_linear(t, w), lambda: mq.mx_linear(x, w, residual=t), lambda: mq.mx_linear(x, w, out=t),
                     lambda: mq.mx_linear(mq.mx_quantize(x), w, residual=t), lambda: mq.mx_linear_grad(t, w), lambda: mq.mx_linear_grad(x, w, out=t),
                     lambda: mq.layer_norm(t), lambda: mq.layer_norm(x, out=t), lambda: mq.layer_norm_mx(t), lambda: mq.layer_norm_grad(t, x, None, mean, rstd),
                     lambda: mq.layer_norm_grad(x, t, None, mean, rstd), lambda: mq.layer_norm_grad(x, x, None, mean, rstd, residual=t),
                     lambda: mq.layer_norm_grad(x, x, None, mean, rstd, out=t), lambda: mq.mx_dequantize(w, F16, out=t)):
            with pytest.raises(ValueError):
                call()
        assert torch.equal(mq.mx_linear_grad(t.contiguous(), w), mq.mx_linear_grad(t.clone(memory_format=torch.contiguous_format), w))


def test_buffers_are_looked_at(mq):
    """Microscaled matrices, column scales and workspaces on the host, too short, of another type or not contiguous: the call raises instead of launching."""
    import dataclasses
    M, K, N = 5, 64, 64
    w, x = mq.mx_quantize_weights(rand((N, K), F16, 80, 0.05)), rand((M, K), F16, 81)
    xq, (_, mean, rstd), n = mq.mx_quantize(x), mq.layer_norm(x, want_stats=True), mq.mx_bytes(N, K)
    part = torch.zeros(2 * n, dtype=torch.uint8, device="cuda")
    for data in (w.data.cpu(), w.data[:n - 1], w.data.view(torch.int8), part[::2], part[:1].expand(n)):
        t = dataclasses.replace(w, data=data)
        for call in (lambda: mq.mx_linear(x, t), lambda: mq.mx_linear(x, t, out=torch.empty_like(x)), lambda: mq.mx_linear(xq, t), lambda: mq.mx_linear(t, w),
                     lambda: mq.mx_linear_grad(x, t), lambda: mq.mx_linear_grad(x, t, out=torch.empty_like(x)), lambda: mq.mx_dequantize(t),
                     lambda: mq.mx_dequantize(t, out=torch.empty(N, K, dtype=BF16, device="cuda")), lambda: mq.mx_unpack(t)):
            with pytest.raises(ValueError):
                call()
    for top, error in ((w.top.cpu(), ValueError), (w.top[:1], ValueError), (w.top.to(torch.int8), TypeError), (part[::2][:2], ValueError)):
        with pytest.raises(error):
            mq.mx_linear_grad(x, dataclasses.replace(w, top=top))
    for ws in (torch.zeros(1 << 20, dtype=torch.uint8), torch.zeros(1 << 21, dtype=torch.uint8, device="cuda")[::2]):
        for call in (lambda: mq.mx_linear(x, w, ws=ws), lambda: mq.mx_linear_grad(x, w, ws=ws), lambda: mq.layer_norm_grad(x, x, None, mean, rstd, ws=ws)):
            with pytest.raises(ValueError):
                call()
    for call in (lambda: mq.mx_linear(x, w, residual=x.cpu()), lambda: mq.mx_linear(x, w, out=x.cpu()), lambda: mq.layer_norm_grad(x.cpu(), x, None, mean, rstd),
                 lambda: mq.layer_norm_grad(x, x, None, mean.cpu(), rstd)):
        with pytest.raises(ValueError):
            call()


# ---------------------------------------------------------------------------------------------- norms: rows without variance, far values

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C", (3, 96, 320, 333, 448, 640, 896, 1000, 1001, 1120, 2709, 4099, 8191))
def test_layer_norm_constant_rows(mq, C, dtype):
    """Rows of one value: up to 2^13 of 11 significant bits add up exactly in float32 in any order, so the mean is the value, what is left of the row
    is zero, and the output is the bias; likewise the gradient of a constant dY, which is zero."""
    x = torch.tensor([1000.0, 60000.0, 0.1, -7.7, 3e-5, 1.0 / 3.0, -65504.0], dtype=dtype, device="cuda").view(-1, 1).repeat(1, C)
    w, b = params(C, "f32", dtype, 90)
    y, mean, rstd = mq.layer_norm(x, w, b, 1e-5, want_stats=True)
    assert torch.equal(mean, x[:, 0].float())
    assert torch.equal(y, b.to(dtype).expand_as(y))
    dx, dw, _ = mq.layer_norm_grad(x, x, None, mean, rstd)
    assert not dx.any() and not dw.any()
    if C % 32 == 0:
        v = mq.mx_dequantize(mq.layer_norm_mx(x, w, b, 1e-5), BF16)
        assert np.array_equal(f64(v), np.repeat(omx.values(f64(b)[None]), len(x), 0))


@pytest.mark.parametrize("C", (8, 24, 33, 328, 1288, 4104))
def test_layer_norm_grad_far_mean(mq, C):
    """Means near the end of bfloat16's range under small variances: lanes that have no columns must not turn 0 times infinity into the row's sum."""
    M = 3
    x = torch.full((M, C), 1e37, dtype=BF16, device="cuda")
    dy, res = rand((M, C), BF16, 91), rand((M, C), BF16, 92)
    for kind in ("16", "none"):
        w, _ = params(C, kind, BF16, 93)
        mean, rstd = x[:, 0].float().contiguous(), torch.full((M,), 316.0, device="cuda")
        dx, dw, db = mq.layer_norm_grad(dy, x, w, mean, rstd, residual=res)
        g = f64(dy) * (1.0 if w is None else f64(w))
        want = 316.0 * (g - g.mean(-1, keepdims=True)) + f64(res)  # xhat is zero
        m1 = np.abs(g).mean(-1, keepdims=True)
        err = 316.0 * (6 * U * (np.abs(g) + m1) + (depth(C) + 4) * U * m1) + 2 * U * np.abs(f64(res)) + 2 * U * np.abs(want)
        within(f64(dx), want, err + half_step(np.abs(want) + err, BF16))
        assert not dw.any()
        within(f64(db), f64(dy).sum(0), (M + 70) * U * np.abs(f64(dy)).sum(0))


# ----------------------------------------------------------------------------------------------- gradient: the ends of bfloat16's range

@pytest.mark.parametrize("M,K,N", ((5, 64, 64), (45, 160, 72), (300, 352, 650), (9, 96, 71), (2, 1280, 9000)))
def test_linear_grad_large_dy(mq, M, K, N):
    """dY near the end of bfloat16's range, weights of ordinary size: results are finite, and so are the sums on the way."""
    dy, w = rand((M, N), BF16, 94, 1.0, 0.0, False), rand((N, K), BF16, 95, 0.02, 0.0, False)
    dy = (dy.float() * 2.0 ** 124).to(BF16)
    dy[-1], dy[-1, 0] = 0.0, 3.3e38
    check_grad(mq, dy, w)
    dx = mq.mx_linear_grad(dy, mq.mx_quantize_weights(w))
    assert torch.isfinite(dx).all()


def test_linear_grad_far_scales(mq):
    """Weights at both ends of bfloat16's range in one column of blocks, dY only on those at the lower one: they count for what they are."""
    N, K = 64, 96
    w = rand((N, K), BF16, 96, 1.0, 0.0, False)
    w[:32] *= 2.0 ** 120
    w[32:] *= 2.0 ** -110
    dy = torch.zeros(6, N, dtype=BF16, device="cuda")
    dy[:, 32:] = rand((6, 32), BF16, 97) * 2.0 ** 20
    wq = mq.mx_quantize_weights(w)
    v = omx.values(f64(w))
    want, mag = omx.linear_grad(f64(dy), v)
    acc = (N + 8) * 2 * U * mag
    for rows in (1, 6):
        within(f64(mq.mx_linear_grad(dy[:rows], wq)), want[:rows], acc[:rows] + half_step(np.abs(want[:rows]) + acc[:rows], BF16))


@pytest.mark.parametrize("M,K,N", ((5, 64, 64), (9, 96, 71), (300, 352, 650)))
def test_linear_grad_small_dy(mq, M, K, N):
    """dY and results near the lower end, subnormal ones among them: a product of the matrix instructions below 2^-149 may go, a result is off by half a
    step."""
    w = rand((N, K), BF16, 98, 0.02)
    for e in (-118, -122, -126):
        dy = (rand((M, N), BF16, 99).float() * 2.0 ** e).to(BF16)
        v = omx.values(f64(w))
        want, mag = omx.linear_grad(f64(dy), v)
        acc = (N + 8) * 2 * U * mag + (N + 8) * 2.0 ** -149
        within(f64(mq.mx_linear_grad(dy, mq.mx_quantize_weights(w))), want, acc + half_step(np.abs(want) + acc, BF16))


def test_graphs_are_refused(mq):
    """Operands that require a gradient: refused where autograd is on, the same bits as without where it is off, and in a torch.autograd.Function."""
    M, K, N = 40, 64, 96
    x, w, b, r = rand((M, K), F16, 100), mq.mx_quantize_weights(rand((N, K), F16, 101, 0.05)), rand((N,), F16, 102), rand((M, N), F16, 103)
    gain, shift = params(K, "f32", F16, 104)
    _, mean, rstd = mq.layer_norm(x, want_stats=True)
    xq = mq.mx_quantize(x)
    g = lambda t: t.clone().requires_grad_()
    calls = ((lambda x: mq.mx_linear(x, w, b), x), (lambda b: mq.mx_linear(x, w, b), b), (lambda r: mq.mx_linear(x, w, b, residual=r), r),
             (lambda b: mq.mx_linear(xq, w, b), b), (lambda r: mq.mx_linear(xq, w, b, residual=r), r), (lambda x: mq.layer_norm(x, gain, shift), x),
             (lambda p: mq.layer_norm(x, p, shift), gain), (lambda p: mq.layer_norm(x, gain, p), shift), (lambda p: mq.layer_norm_mx(x, p, shift).data, gain),
             (lambda d: mq.mx_linear_grad(d, w), r), (lambda d: mq.layer_norm_grad(d, x, gain, mean, rstd)[0], x))
    for call, t in calls:
        with pytest.raises(RuntimeError, match="graph"):
            call(g(t))
        with torch.no_grad():
            assert torch.equal(call(g(t)), call(t))

    class Linear(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            return mq.mx_linear(x, w, b)

        @staticmethod
        def backward(ctx, dy):
            return mq.mx_linear_grad(dy, w)

    leaf = g(x)
    Linear.apply(leaf).backward(r)
    assert torch.equal(leaf.grad, mq.mx_linear_grad(r, w))


def test_outputs_over_operands(mq):
    """Outputs whose rows lie between those of an operand are as any other; ones over an operand are refused."""
    M, K, N = 37, 64, 64
    w = mq.mx_quantize_weights(rand((N, K), F16, 110, 0.05))
    x, r = rand((M, K), F16, 111), rand((M, N), F16, 112)
    _, mean, rstd = mq.layer_norm(x, want_stats=True)
    both = lambda t: (lambda b: (b[:, :64], b[:, 64:]))(torch.cat([t, torch.zeros_like(t)], 1))
    for rows in (1, 5, M):
        a, out = both(r[:rows])
        assert torch.equal(mq.mx_linear_grad(a, w, out=out), mq.mx_linear_grad(r[:rows], w))
        for t in (x[:rows], mq.mx_quantize(x[:rows])):
            a, out = both(r[:rows])
            assert torch.equal(mq.mx_linear(t, w, residual=a, out=out), mq.mx_linear(t, w, residual=r[:rows]))
        a, out = both(x[:rows])
        assert torch.equal(mq.mx_linear(a, w, out=out), mq.mx_linear(x[:rows], w))
        a, out = both(x[:rows])
        assert torch.equal(mq.layer_norm(a, out=out), mq.layer_norm(x[:rows]))
        a, out = both(r[:rows])
        for got, want in zip(mq.layer_norm_grad(a, x[:rows], None, mean[:rows], rstd[:rows], out=out), mq.layer_norm_grad(r[:rows], x[:rows], None, mean[:rows], rstd[:rows])):
            assert torch.equal(got, want)
    b = torch.cat([x, x], 0)
    for call in (lambda: mq.mx_linear_grad(b[:M], w, out=b[:M]), lambda: mq.mx_linear_grad(b[:M], w, out=b[1:M + 1]), lambda: mq.mx_linear(x, w, residual=b[:M], out=b[1:M + 1]),
                 lambda: mq.mx_linear(mq.mx_quantize(x), w, residual=b[1:M + 1], out=b[:M]), lambda: mq.layer_norm(b[:M], out=b[3:M + 3]),
                 lambda: mq.layer_norm_grad(b[:M], x, None, mean, rstd, out=b[1:M + 1])):
        with pytest.raises(mq.MixdqError):
            call()


# --------------------------------------------------------------------------------------------------- many rows, many tiles

# Rows of 640 columns are walked 16 at a time by each of 256 workgroups, 1280 8, 4096 one, 33 columns 32: a walk of two or three turns, the last one cut off.
# (637 and 2049 columns, and rows that start anywhere, take the form that loads value by value.)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,C,per,kind", ((9001, 640, 16, "f32"), (4500, 1280, 8, "16"), (700, 4096, 1, "16"), (2100, 2560, 4, "f32"), (16500, 320, 32, "16"),
                                          (5001, 637, 16, "f32"), (1100, 2049, 4, "16"), (8300, 33, 32, "none")))
def test_layer_norm_grad_many_rows(mq, M, C, per, kind, dtype):
    assert M > 256 * per  # a second turn
    x, dy, res = rand((M, C), dtype, M + C, 1.0, 0.5), rand((M, C), dtype, M + C + 1), rand((M, C), dtype, 120)
    w, b = params(C, kind, dtype, 121)
    _, mean, rstd = mq.layer_norm(x, w, b, 1e-5, want_stats=True)
    W, _ = p64(w, b, C)
    X, DY, R, mu, r = f64(x), f64(dy), f64(res), f64(mean)[:, None], f64(rstd)[:, None]
    xh, g = (X - mu) * r, DY * W
    exh = 3 * U * (np.abs(X) + np.abs(mu)) * r
    n = depth(C)
    m1, m2 = np.abs(g).mean(-1, keepdims=True), (np.abs(g) * (np.abs(xh) + exh)).mean(-1, keepdims=True)
    e1, e2 = (n + 4) * U * m1, (n + 6) * U * m2 + (np.abs(g) * exh).mean(-1, keepdims=True)
    # additions of a column's sum: the turns of a walk, the rows of a workgroup that lie side by side, up to 8 workgroups in a run, 32 runs
    adds = -(-M // (256 * per)) + per + 8 + 32
    for res_, R_ in ((res, R), (None, None)):
        wantx, wantw, wantb = omx.norm_grad(DY, X, W, mu, r, R_)
        err = r * (6 * U * (np.abs(g) + m1 + np.abs(xh) * m2) + e1 + np.abs(xh) * e2 + exh * m2) + (0 if R_ is None else 2 * U * np.abs(R_)) + 2 * U * np.abs(wantx)

        def check(got):
            within(f64(got[0]), wantx, err + half_step(np.abs(wantx) + err, dtype), "dx")
            within(f64(got[1]), wantw, ((adds + 2) * U * np.abs(DY * xh) + np.abs(DY) * exh).sum(0) + 2.0 ** -126, "dweight")
            within(f64(got[2]), wantb, adds * U * np.abs(DY).sum(0) + 2.0 ** -126, "dbias")

        got = mq.layer_norm_grad(dy, x, w, mean, rstd, residual=res_)
        check(got)
        # dX over dY, over the residual: the same bits; in rows that start anywhere: another form, the same bounds
        d = dy.clone()
        assert all(torch.equal(a, c) for a, c in zip(mq.layer_norm_grad(d, x, w, mean, rstd, residual=res_, out=d), got))
        if res_ is not None:
            o = res.clone()
            assert all(torch.equal(a, c) for a, c in zip(mq.layer_norm_grad(dy, x, w, mean, rstd, residual=o, out=o), got))
        o = spread(torch.zeros_like(x), 5, 3)
        check(mq.layer_norm_grad(spread(dy, 3, 1), spread(x, 1, 0), w, mean, rstd, residual=None if res_ is None else spread(res, 5, 7), out=o))
        assert int(torch.isnan(o._base).sum()) == o._base.numel() - M * C


def exact_on_device(t):
    import paper_2405_17873_amd as m
    return m.mx_dequantize(t, BF16).double()  # (exact: two significant bits)


# Tiles of 128 rows x 128 columns in a whole round of 256 workgroups and a last round cut in two and four (6618, 6650, 4096), cut alone (4215) and whole (5557);
# of 64 rows in a whole round and four parts (5651, 5700), whole (4366); of 32 (1000, 20 in six parts).  Rows copied first where N is no multiple of eight.
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,N", ((6618, 544, 2066), (6650, 544, 2072), (4096, 1280, 10240), (4215, 32, 5107), (5557, 288, 40), (5651, 288, 4803), (5700, 288, 4808),
                                   (4366, 160, 32), (1000, 352, 640), (20, 5120, 20480)))
def test_linear_grad_tiles(mq, M, K, N, dtype):
    """Every element, against a float64 product."""
    dy, w = rand((M, N), dtype, M + N), rand((N, K), dtype, K, 0.02)
    wq = mq.mx_quantize_weights(w)
    v = exact_on_device(wq)
    d = dy.double()
    want, acc = d @ v, (d.abs() @ v.abs()) * ((N + 8) * 2 * U)
    top = v.abs().view(N, -1, 32).amax((0, 2)).repeat_interleave(32)
    acc += d.abs().sum(1, keepdim=True) * top * 2.0 ** -36
    bound = acc + torch.finfo(dtype).eps / 2 * (want.abs() + acc) + (2.0 ** -25 if dtype == F16 else 2.0 ** -133)
    for out in (None, spread(torch.zeros(M, K, dtype=dtype, device="cuda"), 8, 8)):
        dx = mq.mx_linear_grad(dy, wq, out=out)
        assert int(((dx.double() - want).abs() > bound).sum()) == 0
        if out is not None:
            assert int(torch.isnan(out._base).sum()) == out._base.numel() - M * K


@pytest.mark.parametrize("M,K,N", ((8200, 704, 4104), (33000, 320, 1032), (2400, 640, 1944), (1190, 992, 4200), (6000, 1280, 1600), (2100, 1280, 3848)))
def test_linear_tiles_bfloat16(mq, M, K, N):
    """The tiles of test_linear_tiles in the other type: 256 x 256, 128 x 160 and several of 128 x 128 to a workgroup, cut off on both sides; every element."""
    x, w, b, r = rand((M, K), BF16, 11), rand((N, K), BF16, 12, 0.02), rand((N,), BF16, 13, 0.1), rand((M, N), BF16, 14)
    wq, xq = mq.mx_quantize_weights(w), mq.mx_quantize(x)
    xv, wv = exact_on_device(xq), exact_on_device(wq)
    want, mag = xv @ wv.T + b.double(), xv.abs() @ wv.abs().T + b.double().abs()
    for res in (None, r):
        if res is not None:
            want, mag = want + res.double(), mag + res.double().abs()
        acc = (K + 4) * 2 * U * mag
        bound = acc + torch.finfo(BF16).eps / 2 * (want.abs() + acc) + 2.0 ** -133
        for t in (xq, x):
            y = mq.mx_linear(t, wq, b, residual=res, dtype=BF16)
            assert int(((y.double() - want).abs() > bound).sum()) == 0
    o = r.clone()
    assert torch.equal(mq.mx_linear(xq, wq, b, residual=o, dtype=BF16, out=o), y)
