"""What stands around the microscaled linears of a transformer block, on the GPU, against the float64 oracle.

Bounds count roundings: a 16-bit result is off by half a step of its type at most, an fp32 operation by U = 2^-24 of its result, an addition inside a matrix
instruction, which may cut off, by 2 U, the hardware's exponential, reciprocal and reciprocal root by 2 U, its sine and cosine by 2^-22 absolutely (which
includes the 2^-32 of a turn that the reduced angle is good to)."""
import numpy as np
import pytest
import torch

from oracle import block as ob, mx as omx
from test_mx_gpu import BF16, F16, F32, TYPES, U, f64, half_step, mq, rand, spread, within  # noqa: F401

pytestmark = pytest.mark.gpu

TRIG = 2.0 ** -22
ACTS = ("gelu", "gelu_tanh", "silu")


# --------------------------------------------------------------------------------------------------- norms and rotation

class Heads:
    """A case: sizes, weights, a rotation, positions; the bounds of its results."""

    def __init__(self, mq, M, q, k, D, sections, interleaved, dtype, kind="same", far=0, norm=True, eps=1e-6, pos_type=torch.int32, seed=0):
        self.mq, self.q, self.k, self.D, self.dtype, self.norm, self.eps, self.inter = mq, q, k, D, dtype, norm, eps, interleaved
        pt = {"same": dtype, "f32": F32, "none": None}[kind] if norm else None
        self.qw, self.kw = (None, None) if pt is None else (rand((D,), pt, seed + 1, 0.2, 1.0, False), rand((D,), pt, seed + 2, 0.2, 1.0, False))
        self.w = np.concatenate([np.repeat((np.ones(D) if w is None else f64(w))[None], n, 0) for w, n in ((self.qw, q), (self.kw, k))])
        self.rot = self.pos = None
        self.angle = np.zeros((M, 0))
        if sections:
            self.rot = mq.rotary(sections, interleaved=interleaved)
            g = torch.Generator().manual_seed(seed + 3)
            self.pos = torch.randint(-far, far + 60, (M, len(sections)), generator=g).to(pos_type).cuda()
            self.angle = ob.angles(self.pos.cpu().numpy(), *ob.frequencies(sections))
        self.args = dict(q_heads=q, k_heads=k, q_weight=self.qw, k_weight=self.kw, rotary=self.rot, positions=self.pos, eps=eps, norm=norm)

    def split(self, t):
        return f64(t).reshape(t.shape[0], self.q + self.k, self.D)

    def turned_magnitude(self, v):
        """For each value of a head: it and, where it turns, the other of its pair."""
        m = np.abs(v)
        P = self.angle.shape[1]
        a, b = ob.pairs(self.D, P, self.inter)
        o = m.copy()
        o[..., a] = o[..., b] = m[..., a] + m[..., b]
        return o

    def far_angle(self):
        """What the oracle's own product of a far position is off by."""
        return 0.0 if self.pos is None else float(self.pos.abs().max()) * 2.0 ** -52

    def check_forward(self, x, y):
        v = self.split(x)
        u = v * (1.0 / np.sqrt((v * v).mean(-1, keepdims=True) + self.eps) if self.norm else 1.0) * self.w
        want = ob.heads(v, self.w, self.angle, self.inter, self.eps, self.norm)
        # mean of D squares: (D + 2) U; its root half of that and 2 U; two products, two in the rotation
        err = self.turned_magnitude(u) * (TRIG + self.far_angle() + ((self.D + 2) / 2 + 8) * U)
        within(self.split(y), want, err + half_step(np.abs(want) + err, self.dtype), "y", self.dtype)

    def check_gradient(self, dy, x, dx, dq, dk):
        d, v = self.split(dy), self.split(x) if x is not None else None
        want, dw = ob.heads_grad(d, v, self.w, self.angle, self.inter, self.eps, self.norm)
        g = ob.turn(d, -self.angle, self.inter)
        e_g = self.turned_magnitude(d) * (TRIG + self.far_angle() + 3 * U)
        if not self.norm:
            within(self.split(dx), want, e_g + half_step(np.abs(want) + e_g, self.dtype), "dx", self.dtype)
            assert dq is None and dk is None
            return
        D, w, r = self.D, self.w, 1.0 / np.sqrt((v * v).mean(-1, keepdims=True) + self.eps)
        e_r = ((D + 2) / 2 + 4) * U  # of r, relative
        dot = (g * w * v).sum(-1, keepdims=True)
        e_dot = (e_g * np.abs(w * v)).sum(-1, keepdims=True) + (D + 3) * U * np.abs(g * w * v).sum(-1, keepdims=True)
        back = dot * r * r / D
        e_back = e_dot * r * r / D + np.abs(back) * (2 * e_r + 4 * U)
        t = g * w - v * back
        err = r * (e_g * np.abs(w) + U * np.abs(g * w) + np.abs(v) * e_back + 2 * U * np.abs(v * back) + U * np.abs(t)) + np.abs(r * t) * (e_r + 2 * U)
        within(self.split(dx), want, err + half_step(np.abs(want) + err, self.dtype), "dx", self.dtype)
        terms, e_terms = np.abs(g * v * r), (e_g * np.abs(v * r) + np.abs(g * v * r) * (e_r + 3 * U))
        for got, part in ((dq, slice(0, self.q)), (dk, slice(self.q, None))):
            n = terms[:, part].shape[0] * terms[:, part].shape[1]
            bound = e_terms[:, part].sum((0, 1)) + n * U * terms[:, part].sum((0, 1)) + 1e-37
            within(f64(got), dw[part].sum(0), bound, "dw")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", (False, True))
@pytest.mark.parametrize("M,q,k,D,sections,kind", ((1, 20, 20, 64, (32,), "same"), (1, 1, 0, 8, (4,), "f32"), (3, 0, 1, 16, None, "none"), (5, 3, 1, 40, (5, 7, 8), "f32"),
                                                  (33, 7, 2, 72, (16, 0, 20), "same"), (9, 5, 5, 80, (16, 16), "none"), (130, 4, 3, 96, (20, 28), "f32"),
                                                  (17, 8, 1, 128, (64,), "same"), (6, 2, 2, 160, (3, 5, 7, 13), "f32"), (4, 3, 2, 256, (128,), "same"),
                                                  (2, 1, 3, 512, (100, 156), "f32"), (700, 9, 4, 32, (16,), "same"), (5000, 3, 2, 64, (8, 12, 12), "same"),
                                                  (3, 70, 31, 24, (12,), "f32")))
def test_heads(mq, M, q, k, D, sections, kind, interleaved, dtype):
    c = Heads(mq, M, q, k, D, sections, interleaved, dtype, kind)
    x, dy = rand((M, (q + k) * D), dtype, 10), rand((M, (q + k) * D), dtype, 11)
    c.check_forward(x, mq.qk_norm_rope(x, **c.args))
    c.check_gradient(dy, x, *mq.qk_norm_rope_grad(dy, x, **c.args))


@pytest.mark.parametrize("interleaved", (False, True))
def test_heads_turn_alone(mq, interleaved):
    """Without the norm; what does not turn keeps its infinities, and turning back gives what went in up to the roundings."""
    c = Heads(mq, 40, 3, 2, 64, (8, 12), interleaved, F16, norm=False)
    x = rand((40, 320), F16, 12)
    y = mq.qk_norm_rope(x, **c.args)
    c.check_forward(x, y)
    dx, dq, dk = mq.qk_norm_rope_grad(x, None, **c.args)
    c.check_gradient(x, None, dx, dq, dk)
    x[3, 50], x[4, 60] = float("inf"), float("nan")  # head 0, columns 40 on do not turn
    y = mq.qk_norm_rope(x, **c.args)
    assert torch.equal(y[3, 40:64], x[3, 40:64]) and torch.equal(y[4, 40:60], x[4, 40:60]) and torch.isnan(y[4, 60])
    assert torch.isfinite(y[3, :40]).all() and torch.isfinite(y[3, 64:]).all()


@pytest.mark.parametrize("pos_type,far", ((torch.int32, 2 ** 30), (torch.int64, 2 ** 30), (torch.int64, 2 ** 44)))
def test_heads_far_positions(mq, pos_type, far):
    """Angles of far positions, negative ones among them.  The table is good to 2^-53 of a frequency (as the oracle's product is) and 2^-64 of a turn."""
    c = Heads(mq, 50, 2, 1, 64, (16, 16), False, F16, far=far, pos_type=pos_type)
    x = rand((50, 192), F16, 13)
    y = mq.qk_norm_rope(x, **c.args)
    if far < 2 ** 40:
        c.check_forward(x, y)
    else:  # (a double's product has lost its turn: a whole frequency in place)
        rot = mq.rotary((32,), freqs=[2 * np.pi / 4] * 32)  # a quarter turn; 2 pi / 4 is off by 2^-54: 2^44 positions by 2^-10
        pos = torch.full((50,), 2 ** 20 + 1, dtype=torch.int64, device="cuda")
        z = mq.qk_norm_rope(x, 2, 1, rotary=rot, positions=pos, norm=False)
        v, want = f64(x).reshape(50, 3, 64), f64(z).reshape(50, 3, 64)
        assert np.abs(want[..., :32] + v[..., 32:]).max() <= 2.0 ** -11 * np.abs(v).max() and torch.isfinite(y).all()


def test_heads_whole_turns(mq):
    """Frequencies of whole fractions of a turn: position p of 8 steps to a turn, at 2^40 + p, is position p exactly."""
    rot = mq.rotary((4, 4), freqs=[2 * np.pi / 8] * 8)
    rot.table[:, 0] = 0  # the fraction 1 / 8 itself
    rot.table[:, 1] = 1 << 29
    x = rand((8, 32), F16, 14)
    p = torch.arange(8, dtype=torch.int64, device="cuda")
    near, far = (torch.stack((q, 3 * q), 1) for q in (p, p + 2 ** 40))
    a = mq.qk_norm_rope(x, 1, 1, rotary=rot, positions=near, norm=False)
    assert torch.equal(a, mq.qk_norm_rope(x, 1, 1, rotary=rot, positions=far, norm=False))
    assert torch.equal(a, mq.qk_norm_rope(x, 1, 1, rotary=rot, positions=near.int(), norm=False))


@pytest.mark.parametrize("M", (1, 7, 300))
def test_heads_views(mq, M):
    """Strides and alignments, positions that lie apart, out over the input, the columns in front of a stacked q, k, v."""
    c = Heads(mq, M, 3, 2, 48, (10, 14), True, BF16, "f32")
    x, dy = rand((M, 240), BF16, 15), rand((M, 240), BF16, 16)
    y, (dx, dq, dk) = mq.qk_norm_rope(x, **c.args), mq.qk_norm_rope_grad(dy, x, **c.args)
    apart = torch.zeros(M, 7, dtype=torch.int32, device="cuda")
    apart[:, 2:4] = c.pos
    args = dict(c.args, positions=apart[:, 2:4])
    for pad, offset in ((8, 8), (1, 0), (5, 3), (16, 4)):
        o = spread(torch.zeros_like(x), pad, offset)
        base = o._base if o._base is not None else o
        mq.qk_norm_rope(spread(x, pad, offset), out=o, **args)
        assert torch.equal(o, y) and int(torch.isnan(base).sum()) == base.numel() - M * 240
        o = spread(torch.zeros_like(x), pad, offset)
        g = mq.qk_norm_rope_grad(spread(dy, pad, offset), spread(x, pad, offset), out=o, **args)
        assert torch.equal(o, dx) and torch.equal(g[1], dq) and torch.equal(g[2], dk)
    qkv = torch.cat((x, rand((M, 96), BF16, 17)), 1)
    values = qkv[:, 240:].clone()
    mq.qk_norm_rope(qkv[:, :240], out=qkv[:, :240], **c.args)
    assert torch.equal(qkv[:, :240], y) and torch.equal(qkv[:, 240:], values)
    for into in (dy.clone(), x.clone()):
        mq.qk_norm_rope_grad(into if torch.equal(into, dy) else dy, x if torch.equal(into, dy) else into, out=into, **c.args)
        assert torch.equal(into, dx)
    at = torch.arange(M, device="cuda")  # one axis: a line of positions
    rot = mq.rotary((24,))
    assert torch.equal(mq.qk_norm_rope(x, 3, 2, rotary=rot, positions=at), mq.qk_norm_rope(x, 3, 2, rotary=rot, positions=at.view(-1, 1).int()))


@pytest.mark.parametrize("kind", ("same", "f32"))
def test_heads_one_weight(mq, kind):
    """Weights of the queries or of the keys alone: the others' are 1."""
    for dtype in TYPES:
        c = Heads(mq, 33, 3, 2, 64, (32,), dtype == F16, dtype, kind)
        x, dy = rand((33, 320), dtype, 22), rand((33, 320), dtype, 23)
        both = c.w.copy()
        for only in ("q_weight", "k_weight"):
            args = dict(c.args, **{("k_weight" if only == "q_weight" else "q_weight"): None})
            c.w = both.copy()
            c.w[(slice(3, None) if only == "q_weight" else slice(0, 3))] = 1.0
            c.check_forward(x, mq.qk_norm_rope(x, **args))
            c.check_gradient(dy, x, *mq.qk_norm_rope_grad(dy, x, **args))


def test_heads_special_rows(mq):
    """Zeros, infinities and NaN stay in their heads; sums of the gradient take them only where they belong."""
    c = Heads(mq, 20, 2, 2, 64, (32,), False, F16, "f32")
    x, dy = rand((20, 256), F16, 18), rand((20, 256), F16, 19)
    x[0], x[1, 70] = 0.0, float("nan")  # a row of zeros; a NaN in head 1
    y = mq.qk_norm_rope(x, **c.args)
    assert not y[0].any() and torch.isnan(y[1, 64:128]).all() and torch.isfinite(y[1, :64]).all() and torch.isfinite(y[1, 128:]).all()
    dx, dq, dk = mq.qk_norm_rope_grad(dy, x, **c.args)
    assert torch.isnan(dx[1, 64:128]).all() and torch.isfinite(dx[1, 128:]).all() and torch.isnan(dq).any() and torch.isfinite(dk).all()
    one = Heads(mq, 3, 1, 0, 64, (32,), True, F16, "same", eps=0.0)  # no key heads, no eps
    z = rand((3, 64), F16, 20)
    one.check_forward(z, mq.qk_norm_rope(z, **one.args))
    _, dq, dk = mq.qk_norm_rope_grad(z, z, **one.args)
    assert torch.isfinite(dq).all() and not dk.any()


def test_heads_rows_past_32_bits(mq):
    """Rows whose offsets pass 32 bits, at both ends of a long matrix."""
    M, q, k, D = 140000, 121, 7, 128
    x = torch.empty(M, (q + k) * D, dtype=BF16, device="cuda").fill_(1.0)
    assert x.numel() > 2 ** 31
    rows = torch.tensor([0, 1, M // 2, M - 2, M - 1], device="cuda")
    some = rand((5, x.shape[1]), BF16, 21)
    x[rows] = some
    c = Heads(mq, M, q, k, D, (64,), False, BF16, far=1000)
    y = mq.qk_norm_rope(x, **c.args)
    c.angle, c.pos = c.angle[rows.cpu().numpy()], c.pos[rows]
    c.check_forward(some, y[rows])


def test_heads_empty(mq):
    rot = mq.rotary((32,))
    x, pos = torch.empty(0, 256, dtype=F16, device="cuda"), torch.empty(0, 1, dtype=torch.int32, device="cuda")
    w = torch.ones(64, device="cuda")
    assert mq.qk_norm_rope(x, 2, 2, w, w, rotary=rot, positions=pos).shape == (0, 256)
    dx, dq, dk = mq.qk_norm_rope_grad(x, x, 2, 2, w, w, rotary=rot, positions=pos)
    assert dx.shape == (0, 256) and not dq.any() and not dk.any()


# ---------------------------------------------------------------------------------------------------------- activations

def act_error(a, name, e_a):
    """(act, its slope, their errors) of an argument a that is off by e_a."""
    f, s = ob.act(a, name), ob.slope(a, name)
    with np.errstate(over="ignore", invalid="ignore"):
        if name == "gelu":
            t, g = ob.tail(a), ob.gauss(a)
            # the tail's polynomial is fitted to 3.3e-6 on [0, 6], its terms and the square are rounded; past 6 the product with 6 is good to 2 % down to -13
            # (and 0 further down), the tail itself to its factor of |a| / 6
            e_t = t * (3.4e-6 + (a * a + 30) * U) + 1e-38 + np.where(np.abs(a) > 6, 1.2 * t, 0)
            e_f = np.abs(a) * t * (3.4e-6 + (a * a + 30) * U) + np.where(np.abs(a) > 6, np.where(np.abs(a) > 13, 1.0, 0.021) * np.abs(a) * t, 0) + U * np.abs(f) + 1e-37
            e_s = e_t + U + np.abs(a) * g * (a * a + 8) * U + U * np.abs(s)
            curve = g * np.abs(2 - a * a)
        else:
            c, d = ob.logistic_terms(name)
            z = np.minimum(np.abs(c * a + d * a ** 3), 200.0)
            l, o, q = ob.logistic(c * a + d * a ** 3), ob.logistic(-(c * a + d * a ** 3)), c + 3 * d * a * a
            e_l = l * (o * (6 * z + 4) * U + 5 * U) + 1e-37
            e_o = e_l + U * np.maximum(o, 0)  # 1 - l
            e_f = np.abs(a) * e_l + U * np.abs(f)
            e_s = e_l + np.abs(q) * (o * e_f + np.abs(f) * e_o) + 5 * U * np.abs(q * f * o) + U * np.abs(s)
            curve = np.abs(2 * l * o * q + a * l * o * (o - l) * q * q + a * l * o * 6 * d * a)
    # second order: the slope changes by at most 1.2 per unit of a
    return f, s, e_f + np.abs(s) * e_a + 1.2 * e_a * e_a, e_s + curve * e_a + 4 * e_a * e_a


def check_act(mq, x, w, bias, name, gated, res=None, out=None, packed=False, want_pre=True):
    wq = mq.mx_quantize_weights(w)
    got = mq.mx_linear(mq.mx_quantize(x) if packed else x, wq, bias, residual=res, out=out, act=name, gated=gated, want_pre=want_pre, dtype=x.dtype if packed else None)
    y, pre = got if want_pre else (got, None)
    a, mag = omx.linear(omx.values(f64(x)), omx.values(f64(w)), None if bias is None else f64(bias))
    check_activated(y, pre, a, (x.shape[1] + 4) * 2 * U * mag, name, gated, x.dtype, res)
    return got


def check_activated(y, pre, a, e_a, name, gated, dtype, res=None):
    if pre is not None:
        within(f64(pre), a, e_a + half_step(np.abs(a) + e_a, dtype), "pre", dtype)
    if name is None:
        want, err = a, e_a
    elif gated:
        (v, g), (e_v, e_g) = ob.halves(a), ob.halves(e_a)
        f, _, e_f, _ = act_error(g, name, e_g)
        want = v * f
        err = np.abs(v) * e_f + e_v * (np.abs(f) + e_f) + U * np.abs(want)
    else:
        want, _, err, _ = act_error(a, name, e_a)
    if res is not None:
        want = want + f64(res)
        err = err + U * np.abs(want)
    within(f64(y), want, err + half_step(np.abs(want) + err, dtype), "y", dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("M,K,N", ((1, 32, 1), (1, 320, 1280), (3, 64, 33), (2, 6976, 40), (31, 2048, 65), (8, 1280, 96), (33, 288, 31), (64, 640, 72), (100, 480, 257), (130, 128, 130), (260, 544, 520),
                                   (513, 320, 384)))
def test_act(mq, M, K, N, name, dtype):
    x, w, b, r = rand((M, K), dtype, M + K), rand((N, K), dtype, N, 0.05), rand((N,), dtype, 9, 0.5), rand((M, N), dtype, 10)
    y, pre = check_act(mq, x, w, b, name, False)
    assert torch.equal(check_act(mq, x, w, b, name, False, want_pre=False), y)
    z, _ = check_act(mq, x, w, b, name, False, r)
    o = r.clone()
    assert mq.mx_linear(x, mq.mx_quantize_weights(w), b, residual=o, out=o, act=name) is o and torch.equal(o, z)
    check_act(mq, x, w, None, name, False, r, packed=True, want_pre=False)
    check_act(mq, x, w, b, name, False, packed=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("M,K,N", ((1, 32, 64), (1, 320, 2560), (3, 6944, 64), (32, 2080, 64), (7, 96, 192), (33, 1280, 128), (64, 288, 320), (100, 480, 576), (130, 128, 64), (260, 544, 704), (513, 320, 1088)))
def test_gate(mq, M, K, N, name, dtype):
    x, w, b = rand((M, K), dtype, M + K), rand((N, K), dtype, N, 0.05), rand((N,), dtype, 9, 0.5)
    y, pre = check_act(mq, x, w, b, name, True)
    assert torch.equal(check_act(mq, x, w, b, name, True, want_pre=False), y)
    check_act(mq, x, w, None, name, True, packed=True)


def exact_sums(mq, x, w, b):
    """Sums and magnitudes in float64 on the GPU, of large cases."""
    xv, wv = mq.mx_dequantize(mq.mx_quantize(x), BF16).double(), mq.mx_dequantize(mq.mx_quantize(w), BF16).double()  # (exact: two significant bits)
    return xv @ wv.T + b.double(), (x.shape[1] + 4) * 2 * U * (xv.abs() @ wv.abs().T + b.double().abs())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,N", ((8200, 704, 4160), (33000, 320, 1088), (2400, 640, 1984), (6000, 1280, 1600), (4096, 1280, 10240)))
def test_act_tiles(mq, M, K, N, dtype):
    """Large tiles and several for a workgroup, cut off on both sides: every element, with and without the sums, whole and gated."""
    x, w, b, r = rand((M, K), dtype, 11), rand((N, K), dtype, 12, 0.03), rand((N,), dtype, 13, 0.1), rand((M, N), dtype, 14)
    wq = mq.mx_quantize_weights(w)
    a, e = exact_sums(mq, x, w, b)
    step = lambda v: torch.finfo(dtype).eps / 2 * v.abs() + 2.0 ** -25
    # silu: slope below 1.1, curvature below 0.51; 40 U of its own covers 6 |z| (1 - s) + 14 (|z| e^-|z| is at most 0.37)
    f, e_f = a * torch.sigmoid(a), 1.1 * e + 0.51 * e * e + 40 * U * a.abs()
    y, pre = mq.mx_linear(x, wq, b, act="silu", want_pre=True)
    assert int(((pre.double() - a).abs() > e + step(a.abs() + e)).sum()) == 0
    assert int(((y.double() - f).abs() > e_f + step(f.abs() + e_f)).sum()) == 0
    assert torch.equal(mq.mx_linear(x, wq, b, act="silu"), y)
    z, again = mq.mx_linear(x, wq, b, act="silu", residual=r, want_pre=True)
    want = f + r.double()
    assert torch.equal(again, pre) and int(((z.double() - want).abs() > e_f + U * want.abs() + step(want.abs() + e_f)).sum()) == 0
    v, g, e_v, e_g = a[:, :N // 2], f[:, N // 2:], e[:, :N // 2], e_f[:, N // 2:]
    want, err = v * g, v.abs() * e_g + e_v * (g.abs() + e_g) + U * (v * g).abs()
    y, again = mq.mx_linear(x, wq, b, act="silu", gated=True, want_pre=True)
    assert torch.equal(again, pre) and int(((y.double() - want).abs() > err + step(want.abs() + err)).sum()) == 0
    assert torch.equal(mq.mx_linear(x, wq, b, act="silu", gated=True), y)


@pytest.mark.parametrize("M", (1, 5, 40, 200))
@pytest.mark.parametrize("gated", (False, True))
def test_act_views(mq, M, gated):
    K, N = 160, 192
    outs = N // 2 if gated else N
    x, w, b, r = rand((M, K), F16, 1), rand((N, K), F16, 2, 0.05), rand((N,), F16, 3), None if gated else rand((M, N), F16, 4)
    want, _ = check_act(mq, x, w, b, "gelu", gated, r)
    wq = mq.mx_quantize_weights(w)
    for pad, offset in ((8, 8), (1, 0), (5, 3), (16, 4)):
        o = spread(torch.zeros(M, outs, dtype=F16, device="cuda"), pad, offset)
        base = o._base if o._base is not None else o
        _, pre = mq.mx_linear(spread(x, pad, offset), wq, spread(b.view(1, -1), pad, offset)[0], out=o, residual=None if gated else spread(r, pad, offset), act="gelu",
                              gated=gated, want_pre=True)
        assert torch.equal(o, want) and int(torch.isnan(base).sum()) == base.numel() - M * outs
    both = x.clone()
    if outs <= K:
        mq.mx_linear(both, wq, b, act="gelu", gated=gated, out=both[:, 8:8 + outs])
        assert torch.equal(both[:, 8:8 + outs], want)


def test_act_special_values(mq):
    """Blocks with NaN make rows of NaN; saturated arguments give 0 and themselves."""
    for M in (4, 40, 200):
        x, w = torch.zeros(M, 64, dtype=BF16, device="cuda"), torch.zeros(64, 64, dtype=BF16, device="cuda")
        w[:, 0] = 1.0
        x[0, 0], x[1, 0], x[2, 0], x[3, 5] = 2.0 ** 100, -(2.0 ** 100), -16.0, float("nan")
        wq = mq.mx_quantize_weights(w)
        for name in ACTS:
            y = mq.mx_linear(x, wq, act=name).double()
            assert (y[0] == 2.0 ** 100).all() and (y[1] == 0).all() and torch.isnan(y[3]).all() and (y[4:] == 0).all()
            assert (y[2] <= 0).all() and (y[2] > -2e-6).all()
            g = mq.mx_linear(x, wq, act=name, gated=True).double()
            assert (g[1] == 0).all() and torch.isnan(g[3]).all()


def test_act_empty(mq):
    w = mq.mx_quantize_weights(rand((64, 64), F16, 1))
    x = torch.empty(0, 64, dtype=F16, device="cuda")
    assert mq.mx_linear(x, w, act="gelu").shape == (0, 64)
    y, pre = mq.mx_linear(x, w, act="silu", gated=True, want_pre=True)
    assert y.shape == (0, 32) and pre.shape == (0, 64)


def test_act_deterministic_and_independent_of_neighbours(mq):
    """The same bits twice and on streams at once; a row's result does not depend on the rows beside it."""
    w, ex = mq.mx_quantize_weights(rand((128, 320), BF16, 9, 0.05)), mq.mx_quantize_experts(rand((2, 128, 320), BF16, 10, 0.05))
    for M in (20, 60, 300):
        x = rand((M, 320), BF16, 8)
        off = torch.tensor([0, M // 2, M], dtype=torch.int32, device="cuda")
        calls = (lambda x: mq.mx_linear(x, w, act="gelu"), lambda x: mq.mx_linear(x, w, act="gelu", gated=True), lambda x: mq.mx_linear_grouped(x, ex, off, act="silu", gated=True))
        want = [c(x) for c in calls]
        torch.cuda.synchronize()
        streams, got = [torch.cuda.Stream() for _ in range(2)], []
        for s in streams:
            with torch.cuda.stream(s):
                got.append([c(x) for c in calls])
        torch.cuda.synchronize()
        for r in got:
            assert all(torch.equal(a, b) for a, b in zip(r, want))
        x2 = x.clone()
        x2[1:] = float("nan")
        assert all(torch.equal(c(x2)[0], v[0]) for c, v in zip(calls, want))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("gated", (False, True))
@pytest.mark.parametrize("M,N", ((1, 2), (1, 640), (2, 66), (16, 512), (17, 1000), (130, 130), (33, 2050), (1000, 320), (300, 4096)))
def test_act_grad(mq, M, N, name, gated, dtype):
    a, dy = rand((M, N), dtype, M + N, 2.0), rand((M, N // 2 if gated else N), dtype, 5)
    da, dbias = mq.act_grad(dy, a, name, gated)
    v, d = f64(a), f64(dy)
    want = ob.act_grad(d, v, name, gated)
    if gated:
        p, g = ob.halves(v)
        f, s, e_f, e_s = act_error(g, name, 0.0)
        err = np.concatenate((np.abs(d) * e_f, np.abs(d * p) * (e_s + U * np.abs(s))), 1) + U * np.abs(want)
    else:
        _, s, _, e_s = act_error(v, name, 0.0)
        err = np.abs(d) * e_s + U * np.abs(want)
    within(f64(da), want, err + half_step(np.abs(want) + err, dtype), "da", dtype)
    within(f64(dbias), want.sum(0), err.sum(0) + M * U * np.abs(want).sum(0) + 1e-37, "dbias")
    only, none = mq.act_grad(dy, a, name, gated, want_dbias=False)
    assert none is None and torch.equal(only, da)


def test_act_grad_values_everywhere(mq):
    """All finite 16-bit arguments."""
    for dtype in TYPES:
        p = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dtype)
        a = p[torch.isfinite(p.float())].view(-1, 64).cuda()
        for name in ACTS:
            da, _ = mq.act_grad(torch.ones_like(a), a, name)
            _, s, _, e_s = act_error(f64(a), name, 0.0)
            within(f64(da), s, e_s + half_step(np.abs(s) + e_s, dtype), name, dtype)
            both, _ = mq.act_grad(torch.ones_like(a), torch.cat((torch.ones_like(a), a), 1), name, True)
            f, _, e_f, _ = act_error(f64(a), name, 0.0)
            within(f64(both[:, :64]), f, e_f + half_step(np.abs(f) + e_f, dtype), name, dtype)
            assert torch.equal(both[:, 64:], da)


def test_act_grad_views_and_aliases(mq):
    M, N = 45, 202
    a, dy, half = rand((M, N), F16, 1), rand((M, N), F16, 2), rand((M, N // 2), F16, 3)
    for gated, d in ((False, dy), (True, half)):
        da, db = mq.act_grad(d, a, "gelu", gated)
        for pad, offset in ((8, 8), (1, 0), (5, 3)):
            o = spread(torch.zeros_like(a), pad, offset)
            base = o._base if o._base is not None else o
            g, b = mq.act_grad(spread(d, pad, offset), spread(a, pad, offset), "gelu", gated, out=o)
            assert g is o and torch.equal(o, da) and torch.equal(b, db) and int(torch.isnan(base).sum()) == base.numel() - M * N
        o = a.clone()
        assert torch.equal(mq.act_grad(d, o, "gelu", gated, out=o)[0], da)
    o = dy.clone()
    assert torch.equal(mq.act_grad(o, a, "gelu", out=o)[0], mq.act_grad(dy, a, "gelu")[0])
    e = torch.empty(0, 64, dtype=F16, device="cuda")
    da, db = mq.act_grad(e, e, "silu")
    assert da.shape == (0, 64) and not db.any()


def test_act_grad_against_differences(mq):
    """Through the forward call: sums moved by a bias of h, of which 16-bit biases hold every value used.  The second difference bounds what is left of the first."""
    M, K, N, h = 6, 64, 128, 2.0 ** -6
    x, w, dy = rand((M, K), BF16, 1, outliers=False), rand((N, K), BF16, 2, 0.1), rand((M, N), BF16, 3)
    wq = mq.mx_quantize_weights(w)
    a = omx.linear(omx.values(f64(x)), omx.values(f64(w)))[0]
    for name in ACTS:
        up, down = (ob.act(a + s, name) for s in (h, -h))
        got = (f64(mq.mx_linear(x, wq, torch.full((N,), s, dtype=BF16, device="cuda"), act=name)) for s in (h, -h))
        diff = np.subtract(*got) / (2 * h)
        # each result is off by half a step; the third derivatives are below 3: h^2 / 6 of that
        err = (half_step(up, BF16) + half_step(down, BF16) + 1e-4) / (2 * h) + 3 * h * h / 6
        _, pre = mq.mx_linear(x, wq, act=name, want_pre=True)
        da, _ = mq.act_grad(dy, pre, name)
        # the kept sums are off by half a step (slopes change by at most 1.2 per unit), and so are the results
        d = f64(dy)
        within(f64(da), diff * d, np.abs(d) * (err + 1.2 * half_step(a, BF16)) + half_step(np.abs(d) * 1.3, BF16), name)


# -------------------------------------------------------------------------------------------------------------- experts

def expert_case(M, E, K, N, dtype, sizes, seed=0):
    """sizes: rows of each expert; what is left over lies in front and behind."""
    x, w, b = rand((M, K), dtype, seed + 1), rand((E, N, K), dtype, seed + 2, 0.05), rand((E, N), dtype, seed + 3, 0.3)
    left = M - sum(sizes)
    assert left >= 0 and len(sizes) == E
    off = np.concatenate(([0], np.cumsum(sizes))) + left // 2
    return x, w, b, off, torch.tensor(off, dtype=torch.int32, device="cuda")


SPLITS = ((1, 1, 32, 32, (1,)), (1, 3, 64, 64, (0, 1, 0)), (5, 2, 96, 32, (0, 0)), (7, 4, 320, 96, (3, 0, 1, 2)), (40, 4, 160, 128, (33, 0, 7, 0)), (70, 2, 64, 64, (1, 66)),
          (300, 5, 288, 160, (31, 32, 33, 1, 200)), (260, 3, 128, 320, (130, 0, 129)), (1000, 2, 544, 192, (515, 470)), (500, 40, 64, 64, tuple((i * 7) % 25 for i in range(40))),
          (900, 300, 32, 32, tuple(3 if i % 3 else 0 for i in range(300))), (300, 40, 64, 64, (200,) + (0,) * 38 + (70,)), (50, 8, 4192, 64, (33, 0, 5, 0, 1, 0, 0, 9)),
          (1000, 100, 96, 64, tuple(i % 21 for i in range(100))), (1400, 130, 64, 32, (700,) + (0,) * 100 + (20,) * 29), (640, 6, 352, 256, (5, 300, 64, 128, 0, 140)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,E,K,N,sizes", SPLITS)
def test_experts(mq, M, E, K, N, sizes, dtype):
    """Rows by expert in all forms: each with its own weights and bias, and the rows of none left as they were."""
    x, w, b, off, offsets = expert_case(M, E, K, N, dtype, sizes)
    wq = mq.mx_quantize_experts(w)
    xv, wv = omx.values(f64(x)), omx.values(f64(w).reshape(E * N, K)).reshape(E, N, K)
    have = np.zeros(M, bool)
    have[off[0]:off[-1]] = True
    for bias in (b, None):
        a, mag = ob.grouped(xv, wv, off, None if bias is None else f64(bias))
        e = (K + 4) * 2 * U * mag
        for name, gated in ((None, False), ("gelu", False), ("silu", True)):
            if gated and N % 64:
                continue
            outs = N // 2 if gated else N
            out = torch.full((M, outs), 7.0, dtype=dtype, device="cuda")
            r = mq.mx_linear_grouped(x, wq, offsets, bias, out=out, act=name, gated=gated, want_pre=name is not None)
            y, pre = r if name else (r, None)
            assert y is out and (out[torch.from_numpy(~have).cuda()] == 7.0).all()
            check_activated(y[have], None if pre is None else pre[have], a[have], e[have], name, gated, dtype)
            again = mq.mx_linear_grouped(x, wq, offsets, bias, act=name, gated=gated)
            assert torch.equal(again[have], y[have])
    dy = rand((M, N), dtype, 4)
    out = torch.full((M, K), 7.0, dtype=dtype, device="cuda")
    dx = mq.mx_linear_grouped_grad(dy, wq, offsets, out=out)
    want, mag = ob.grouped_grad(f64(dy), wv, off)
    top = np.abs(wv).reshape(E, N, -1, 32).max((1, 3))
    per_row = np.zeros((M, K // 32))
    for i in range(E):
        per_row[off[i]:off[i + 1]] = top[i]
    acc = (N + 8) * 2 * U * mag + np.abs(f64(dy)).sum(1, keepdims=True) * np.repeat(per_row, 32, 1) * 2.0 ** -36
    within(f64(dx)[have], want[have], (acc + half_step(np.abs(want) + acc, dtype))[have], "dx", dtype)
    assert (out[torch.from_numpy(~have).cuda()] == 7.0).all()
    assert torch.equal(mq.mx_linear_grouped_grad(dy, wq, offsets)[have], dx[have])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,E,K,N", ((9000, 4, 704, 2112), (5000, 8, 1280, 2048), (12000, 3, 320, 1088)))
def test_experts_tiles(mq, M, E, K, N, dtype):
    """Many rows: every element against the linear of each expert's rows, which takes its sums in the same order."""
    g = torch.Generator().manual_seed(M)
    sizes = torch.multinomial(torch.rand(E, generator=g), M - 37, replacement=True, generator=g).bincount(minlength=E).tolist()
    sizes[1], sizes[0] = 0, sizes[0] + sizes[1]
    x, w, b, off, offsets = expert_case(M, E, K, N, dtype, sizes)
    wq = mq.mx_quantize_experts(w)
    dy = rand((M, N), dtype, 5)
    y = mq.mx_linear_grouped(x, wq, offsets, b)
    z, pre = mq.mx_linear_grouped(x, wq, offsets, b, act="gelu", gated=True, want_pre=True)
    dx = mq.mx_linear_grouped_grad(dy, wq, offsets)
    step = torch.finfo(dtype).eps
    for e in range(E):
        r = slice(int(off[e]), int(off[e + 1]))
        if r.start == r.stop:
            continue
        a, err = exact_sums(mq, x[r], w[e], b[e])
        bound = err + step / 2 * (a.abs() + err) + 2.0 ** -25
        assert int(((y[r].double() - a).abs() > bound).sum()) == 0 and torch.equal(pre[r], y[r])
        v, t, e_v, e_t = a[:, :N // 2], a[:, N // 2:], err[:, :N // 2], err[:, N // 2:]
        f = t * 0.5 * torch.special.erfc(-t / 2 ** 0.5)
        e_f = 1.13 * e_t + 1.2 * e_t * e_t + t.abs() * 1e-6
        bound = v.abs() * e_f + e_v * (f.abs() + e_f) + U * (v * f).abs()
        assert int(((z[r].double() - v * f).abs() > bound + step / 2 * ((v * f).abs() + bound) + 2.0 ** -25).sum()) == 0
        wv = mq.mx_dequantize(mq.mx_quantize(w[e]), BF16).double()
        want, mag = dy[r].double() @ wv, dy[r].double().abs() @ wv.abs()
        acc = (N + 8) * 2 * U * mag + dy[r].double().abs().sum(1, keepdim=True) * wv.abs().max() * 2.0 ** -36
        assert int(((dx[r].double() - want).abs() > acc + step / 2 * (want.abs() + acc) + 2.0 ** -25).sum()) == 0


@pytest.mark.parametrize("M,sizes", ((6, (2, 0, 4)), (200, (90, 10, 100))))
def test_experts_views(mq, M, sizes):
    x, w, b, off, offsets = expert_case(M, 3, 96, 64, F16, sizes)
    wq, dy = mq.mx_quantize_experts(w), rand((M, 64), F16, 6)
    want, gate, grad = mq.mx_linear_grouped(x, wq, offsets, b), mq.mx_linear_grouped(x, wq, offsets, b, act="silu", gated=True), mq.mx_linear_grouped_grad(dy, wq, offsets)
    for pad, offset in ((8, 8), (1, 0), (5, 3), (16, 4)):
        for ref, call, cols in ((want, lambda o: mq.mx_linear_grouped(spread(x, pad, offset), wq, offsets, b, out=o), 64),
                                (gate, lambda o: mq.mx_linear_grouped(spread(x, pad, offset), wq, offsets, b, out=o, act="silu", gated=True), 32),
                                (grad, lambda o: mq.mx_linear_grouped_grad(spread(dy, pad, offset), wq, offsets, out=o), 96)):
            o = spread(torch.zeros(M, cols, dtype=F16, device="cuda"), pad, offset)
            base = o._base if o._base is not None else o
            call(o)
            assert torch.equal(o, ref) and int(torch.isnan(base).sum()) == base.numel() - M * cols


def test_experts_of_one_are_the_linear(mq):
    """One expert with all the rows: the same bits as the linear's."""
    for M in (5, 33, 400):
        x, w, b = rand((M, 160), BF16, 1), rand((128, 160), BF16, 2, 0.05), rand((128,), BF16, 3)
        one, all_rows = mq.mx_quantize_experts(w[None]), torch.tensor([0, M], dtype=torch.int32, device="cuda")
        y = mq.mx_linear_grouped(x, one, all_rows, b[None], act="gelu", gated=True)
        z = mq.mx_linear(x, mq.mx_quantize_weights(w), b, act="gelu", gated=True)
        within(f64(y), f64(z), 2 * half_step(f64(z), BF16) + 1e-4, "one expert")
        if M == 400:  # (few rows are joined by another number of waves)
            assert torch.equal(y, z)


def test_experts_offsets_that_are_none(mq):
    """Offsets that leave the matrix or fall: nothing outside it is read or written, and experts in front of them keep their results."""
    for M in (6, 200):
        x, w, b, off, _ = expert_case(M, 4, 64, 64, F16, (M // 2, 0, M // 2, 0))
        wq, dy = mq.mx_quantize_experts(w), rand((M, 64), F16, 7)
        good = torch.tensor(off, dtype=torch.int32, device="cuda")
        y, dx = mq.mx_linear_grouped(x, wq, good, b), mq.mx_linear_grouped_grad(dy, wq, good)
        for bad in ((0, M // 2, M // 2, M + 1000, 2 ** 31 - 1), (-(2 ** 31), M // 2, M // 2, M, M), (0, M // 2, M // 2, M, -5), (0, M // 2, M // 4, M, 3)):
            o = torch.tensor(bad, dtype=torch.int32, device="cuda")
            pad = torch.full((M + 64, 64), 7.0, dtype=F16, device="cuda")
            z = mq.mx_linear_grouped(x, wq, o, b, out=pad[32:32 + M])
            g = mq.mx_linear_grouped_grad(dy, wq, o)
            assert torch.equal(z[:M // 4], y[:M // 4]) and torch.equal(g[:M // 4], dx[:M // 4])
            assert (pad[:32] == 7.0).all() and (pad[32 + M:] == 7.0).all()


def test_experts_empty_and_many(mq):
    w = rand((3, 64, 64), F16, 1, 0.05)
    wq, off = mq.mx_quantize_experts(w), torch.zeros(4, dtype=torch.int32, device="cuda")
    e = torch.empty(0, 64, dtype=F16, device="cuda")
    assert mq.mx_linear_grouped(e, wq, off).shape == (0, 64) and mq.mx_linear_grouped_grad(e, wq, off).shape == (0, 64)
    for M in (4, 300):  # no expert has a row
        out = torch.full((M, 64), 7.0, dtype=F16, device="cuda")
        mq.mx_linear_grouped(rand((M, 64), F16, 2), wq, off, out=out)
        assert (out == 7.0).all()
        mq.mx_linear_grouped_grad(rand((M, 64), F16, 2), wq, off, out=out)
        assert (out == 7.0).all()
    x = rand((4096, 32), F16, 3)  # the most experts, a row each
    many = rand((4096, 32, 32), F16, 4, 0.1)
    wq, off = mq.mx_quantize_experts(many), torch.arange(4097, dtype=torch.int32, device="cuda")
    y, dx = mq.mx_linear_grouped(x, wq, off), mq.mx_linear_grouped_grad(x, wq, off)
    xv, wv = mq.mx_dequantize(mq.mx_quantize(x), BF16).double(), mq.mx_dequantize(mq.mx_quantize(many.view(-1, 32)), BF16).double().view(4096, 32, 32)
    want, mag = (wv * xv[:, None]).sum(-1), (wv * xv[:, None]).abs().sum(-1)
    assert int(((y.double() - want).abs() > 72 * U * mag + 2.0 ** -11 * want.abs() * 1.001 + 2.0 ** -24).sum()) == 0
    want, mag = (wv * x.double()[:, :, None]).sum(1), (wv * x.double()[:, :, None]).abs().sum(1)
    assert int(((dx.double() - want).abs() > 80 * U * mag + 2.0 ** -11 * want.abs() * 1.001 + 2.0 ** -24).sum()) == 0


def test_experts_weights_past_32_bits(mq):
    """Experts whose codes lie past 2^32 bytes of the first's."""
    E, N, K = 34, 8192, 32768
    data = torch.zeros(mq.mx_bytes(E * N, K), dtype=torch.uint8, device="cuda")
    assert data.numel() > 2 ** 32
    last = mq.mx_quantize_weights(rand((N, K), F16, 1, 0.02))
    groups, codes = N // 32, N // 32 * (K // 64) * 1024
    data[(E - 1) * codes:E * codes] = last.data[:codes]
    data[E * codes + (E - 1) * (last.data.numel() - codes):] = last.data[codes:]
    w = mq.mx_experts(mq.MxTensor(data, E * N, K), E)
    for M in (3, 300):
        x, dy = rand((M, K), F16, 2), rand((M, N), F16, 3)
        off = torch.tensor([0] * (E - 1) + [1, M], dtype=torch.int32, device="cuda")
        y, dx = mq.mx_linear_grouped(x, w, off), mq.mx_linear_grouped_grad(dy, w, off)
        assert not y[:1].any() and not dx[:1].any()
        z, g = mq.mx_linear(x[1:], last).double(), mq.mx_linear_grad(dy[1:], last).double()
        # (sums of random signs in another order: 0.02 is far below one wrong block)
        assert ((y[1:].double() - z).abs() <= 2.0 ** -10 * z.abs() + 2e-2).all() and ((dx[1:].double() - g).abs() <= 2.0 ** -10 * g.abs() + 2e-2).all()


# ------------------------------------------------------------------------------------------------------------- together

def block_step(mq, s):
    """A block of a transformer forward and backward: norm, stacked q, k, v, head norms with rotation, attention by plain products, output projection with the
    skip, norm, gated feed-forward by expert, and back to the first gradient."""
    M, H, D = s["x"].shape[0], 4, 32
    n, mean, rstd = mq.layer_norm_mx(s["x"], s["gain"], s["shift"], want_stats=True)
    qkv = mq.mx_linear(n, s["qkv"], s["qkv_b"], dtype=s["x"].dtype)
    args = dict(q_heads=H, k_heads=H, q_weight=s["qw"], k_weight=s["kw"], rotary=s["rot"], positions=s["pos"])
    qk = mq.qk_norm_rope(qkv[:, :2 * H * D], **args)
    q, k, v = (t.view(M, H, D).transpose(0, 1).float() for t in (qk[:, :H * D].contiguous(), qk[:, H * D:].contiguous(), qkv[:, 2 * H * D:].contiguous()))
    p = torch.softmax(torch.matmul(q, k.transpose(1, 2).contiguous()) / D ** 0.5, -1)
    o = torch.matmul(p, v).transpose(0, 1).reshape(M, H * D).to(s["x"].dtype)
    h = mq.mx_linear(o, s["out"], s["out_b"], residual=s["x"])
    y, pre = mq.mx_linear(h, s["up"], s["up_b"], act="silu", gated=True, want_pre=True)
    z, kept = mq.mx_linear_grouped(y, s["experts"], s["offsets"], s["experts_b"], act="gelu", gated=True, want_pre=True)
    dz, _ = mq.act_grad(s["dz"], kept, "gelu", True, want_dbias=False)
    dy = mq.mx_linear_grouped_grad(dz, s["experts"], s["offsets"])
    da, dbias = mq.act_grad(dy, pre, "silu", True)
    dh = mq.mx_linear_grad(da, s["up"])
    do = mq.mx_linear_grad(dh, s["out"])
    dqk, dqw, dkw = mq.qk_norm_rope_grad(torch.cat((do, do), 1), qkv[:, :2 * H * D], **args)
    return dict(z=z, dbias=dbias, dh=dh, dqk=dqk, dqw=dqw, dkw=dkw, qk=qk)


def block_state(mq, dtype=BF16, M=70, C=128):
    u = lambda *shape, std=0.08: rand(shape, dtype, sum(shape), std, outliers=False)
    return dict(x=rand((M, C), dtype, 1), gain=rand((C,), F32, 2, 0.1, 1.0), shift=rand((C,), F32, 3, 0.1), qkv=mq.mx_quantize_weights(u(3 * C, C)), qkv_b=u(3 * C),
                qw=rand((32,), F32, 4, 0.1, 1.0), kw=rand((32,), F32, 5, 0.1, 1.0), rot=mq.rotary((4, 6, 6), interleaved=True),
                pos=torch.stack((torch.arange(M) // 35, torch.arange(M) // 7 % 5, torch.arange(M) % 7), 1).int().cuda(), out=mq.mx_quantize_weights(u(C, C)), out_b=u(C),
                up=mq.mx_quantize_weights(u(2 * C, C)), up_b=u(2 * C), experts=mq.mx_quantize_experts(u(3, 2 * C, C)), experts_b=u(3, 2 * C),
                offsets=torch.tensor([0, 20, 20, M], dtype=torch.int32, device="cuda"), dz=rand((M, C), dtype, 6))


def test_block_runs_together(mq):
    s = block_state(mq)
    r = block_step(mq, s)
    assert all(torch.isfinite(t.float()).all() for t in r.values())
    again = block_step(mq, s)
    assert all(torch.equal(r[k], again[k]) for k in r)


def test_block_graph_replays_and_side_stream(mq):
    """Captured and replayed with new inputs and offsets, with eager work between; on another stream; two graphs with workspaces of their own."""
    s = block_state(mq)
    s["x16"] = s["x"]
    ops = lambda: ops_of(mq, s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = ops()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(first, ops()):
        assert torch.equal(a, b)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            captured = ops()
        graphs.append((g, captured))
    for seed, cut in ((1, 20), (7, 0), (9, 70), (11, 33)):
        s["x"].copy_(rand(tuple(s["x"].shape), BF16, seed))
        s["dz"].copy_(rand(tuple(s["dz"].shape), BF16, seed + 1))
        s["offsets"].copy_(torch.tensor([0, cut, cut, 70], dtype=torch.int32))
        s["pos"].add_(seed)
        for g, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        want = ops()
        for _, captured in graphs:
            for a, b in zip(captured, want):
                assert torch.equal(a, b)


def ops_of(mq, s):
    """The operators of this file alone, few and many rows (the captured block without torch's products)."""
    args = dict(q_heads=2, k_heads=2, q_weight=s["qw"], k_weight=s["kw"], rotary=s["rot"], positions=s["pos"])
    y, pre = mq.mx_linear(s["x"], s["up"], s["up_b"], act="silu", gated=True, want_pre=True)
    few = mq.mx_linear(s["x"][:5], s["up"], s["up_b"], act="gelu")
    z = mq.mx_linear_grouped(s["x"], s["experts"], s["offsets"], s["experts_b"], act="gelu", gated=True)
    da, dbias = mq.act_grad(s["dz"], pre, "silu", True)
    dx = mq.mx_linear_grouped_grad(da, s["experts"], s["offsets"])
    return (y, pre, few, z, da, dbias, dx, mq.qk_norm_rope(s["x"], **args), *mq.qk_norm_rope_grad(s["dz"], s["x"], **args))


def test_graphs_are_refused(mq):
    """Operands that require a gradient: refused where autograd is on, the same bits as without where it is off."""
    s = block_state(mq)
    g = lambda t: t.clone().requires_grad_()
    x, dz = s["x"], s["dz"]
    up, pre = mq.mx_linear(x, s["up"], s["up_b"], act="silu", want_pre=True)
    args = dict(rotary=s["rot"], positions=s["pos"])
    calls = ((lambda t: mq.qk_norm_rope(t, 2, 2, **args), x), (lambda t: mq.qk_norm_rope(x, 2, 2, t, s["kw"], **args), s["qw"]), (lambda t: mq.qk_norm_rope(x, 2, 2, s["qw"], t, **args), s["kw"]),
             (lambda t: mq.qk_norm_rope_grad(t, x, 2, 2, **args)[0], dz), (lambda t: mq.mx_linear(t, s["up"], act="gelu"), x), (lambda t: mq.mx_linear(x, s["up"], t, act="gelu"), s["up_b"]),
             (lambda t: mq.act_grad(t, pre, "silu")[0], up), (lambda t: mq.act_grad(up, t, "silu")[0], pre), (lambda t: mq.mx_linear_grouped(t, s["experts"], s["offsets"]), x),
             (lambda t: mq.mx_linear_grouped(x, s["experts"], s["offsets"], t), s["experts_b"]), (lambda t: mq.mx_linear_grouped_grad(t, s["experts"], s["offsets"]), pre))
    for call, t in calls:
        with pytest.raises(RuntimeError, match="graph"):
            call(g(t))
        want = call(t)
        with torch.no_grad():
            assert torch.equal(torch.nan_to_num(call(g(t)).float()), torch.nan_to_num(want.float()))


def test_refusals(mq):
    """What the calls do not take is refused before anything runs."""
    s = block_state(mq)
    x, up, ex, off = s["x"], s["up"], s["experts"], s["offsets"]
    args = dict(rotary=s["rot"], positions=s["pos"])
    wide = x.repeat(1, 2)
    bad = (lambda: mq.qk_norm_rope(x, 3, 2, **args), lambda: mq.qk_norm_rope(x, 0, 0, **args), lambda: mq.qk_norm_rope(x, 2, 2, rotary=s["rot"]),
           lambda: mq.qk_norm_rope(x, 2, 2, positions=s["pos"]), lambda: mq.qk_norm_rope(x, 2, 2, rotary=s["rot"], positions=s["pos"][:, :2]),
           lambda: mq.qk_norm_rope(x, 2, 2, rotary=s["rot"], positions=s["pos"].float()), lambda: mq.qk_norm_rope(x, 2, 2, rotary=s["rot"], positions=s["pos"].cpu()),
           lambda: mq.qk_norm_rope(x, 2, 2, s["qw"], s["kw"], norm=False), lambda: mq.qk_norm_rope(x, 2, 2, s["qw"].half(), s["kw"], **args), lambda: mq.qk_norm_rope(x, 2, 2, s["qw"][:16]),
           lambda: mq.qk_norm_rope(x, 8, 8, **args), lambda: mq.qk_norm_rope(x, 2, 2, eps=-1.0), lambda: mq.qk_norm_rope(x, 2, 2, out=x[:, :64]), lambda: mq.qk_norm_rope(x.float(), 2, 2),
           lambda: mq.qk_norm_rope(wide[:, :128], 2, 2, out=wide[:, 1:129]), lambda: mq.qk_norm_rope_grad(x, None, 2, 2), lambda: mq.qk_norm_rope_grad(x, wide, 2, 2),
           lambda: mq.rotary((3,)), lambda: mq.rotary((4,) * 5), lambda: mq.rotary((4,), freqs=[1.0]), lambda: mq.rotary((4,), freqs=[float("nan")] * 4),
           lambda: mq.mx_linear(x, up, act="relu"), lambda: mq.mx_linear(x, up, gated=True), lambda: mq.mx_linear(x, up, want_pre=True), lambda: mq.mx_linear(x, up, act="gelu", gated=True, residual=x),
           lambda: mq.mx_linear(x, mq.mx_quantize_weights(rand((96, 128), BF16, 1)), act="gelu", gated=True), lambda: mq.mx_linear(x, up, act="gelu", out=x),
           lambda: mq.act_grad(x, x, None), lambda: mq.act_grad(x, x, "tanh"), lambda: mq.act_grad(x, x, "gelu", True), lambda: mq.act_grad(x, x.half(), "gelu"),
           lambda: mq.act_grad(wide[:, :64], wide[:, 64:192], "gelu", True, out=wide[:, 32:160]), lambda: mq.act_grad(x[:, :64], wide[:, :128], "gelu", True, out=wide[:, 1:129]),
           lambda: mq.mx_linear_grouped(x, ex, off.long()), lambda: mq.mx_linear_grouped(x, ex, off[:3]), lambda: mq.mx_linear_grouped(x, ex, off.cpu()),
           lambda: mq.mx_linear_grouped(x, ex, off, s["experts_b"].view(-1)), lambda: mq.mx_linear_grouped(wide[:, :128], ex, off, act="gelu", gated=True, out=wide[:, 64:192]),
           lambda: mq.mx_linear_grouped(x, mq.mx_experts(up, 16), off), lambda: mq.mx_experts(up, 3), lambda: mq.mx_quantize_experts(x), lambda: mq.mx_linear_grouped(x[:, :64], ex, off),
           lambda: mq.mx_linear_grouped_grad(x, ex, off), lambda: mq.mx_linear_grouped_grad(x.repeat(1, 2), mq.MxTensor(ex.data, ex.rows, ex.K, None, 3), off),
           lambda: mq.mx_linear_grad(x.repeat(1, 6), ex))
    for call in bad:
        with pytest.raises((ValueError, TypeError, mq.MixdqError)):
            call()


def gelu_bounds(a):
    """gelu and its slope, and what the kernels' are off by before they are rounded.  The tail's polynomial is fitted to 6.1e-7 max(1, 0.144 a^2) of it (1.5 a^2 U
    past 2.6); its argument, its terms and the product count 16 U at most; the exponential's argument, two products, carries 2.5 U of 0.73 a^2 log 2.  Below
    2^-126 exponentials are zero: 0.4 of that with |a| up to 14, and so 1e-37."""
    t, g, f, s = ob.tail(a), ob.gauss(a), ob.act(a, "gelu"), ob.slope(a, "gelu")
    e_t = t * (6.2e-7 + (3 * a * a + 16) * U)
    return f, s, np.abs(a) * e_t + U * np.abs(f) + 1e-37, e_t + np.abs(a) * g * (1.5 * a * a + 5) * U + U * np.abs(s) + 2e-37


def finite_values(dtype):
    p = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dtype)
    return p[torch.isfinite(p.float())]


@pytest.mark.parametrize("dtype", TYPES)
def test_gelu_of_every_value(mq, dtype):
    """All finite 16-bit arguments, from a bias behind weights of zero, in the kernels for few rows, for some, for tiles and for large tiles, whole and gated: the
    definition's value, rounded, far down the negative side too."""
    p = finite_values(dtype).cuda()
    with np.errstate(over="ignore", under="ignore"):
        f, _, e, _ = gelu_bounds(f64(p))
    bound = e + half_step(np.abs(f) + e, dtype)
    ones = torch.ones_like(p)
    for bias, gated in ((p, False), (torch.cat((ones, p)), True)):
        w = mq.mx_quantize_weights(torch.zeros(len(bias), 32, dtype=dtype, device="cuda"))
        for M in (1, 40, 200, 600):
            y = mq.mx_linear(torch.zeros(M, 32, dtype=dtype, device="cuda"), w, bias, act="gelu", gated=gated)
            assert torch.equal(y, y[:1].expand_as(y))
            within(f64(y[0]), f, bound, f"{M} rows", dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_gelu_grad_of_every_value(mq, dtype):
    a = finite_values(dtype).view(-1, 64).cuda()
    ones = torch.ones_like(a)
    with np.errstate(over="ignore", under="ignore"):
        f, s, e_f, e_s = gelu_bounds(f64(a))
    da, _ = mq.act_grad(ones, a, "gelu")
    within(f64(da), s, e_s + half_step(np.abs(s) + e_s, dtype), "slope", dtype)
    both, _ = mq.act_grad(ones, torch.cat((ones, a), 1), "gelu", True)
    within(f64(both[:, :64]), f, e_f + half_step(np.abs(f) + e_f, dtype), "gate", dtype)
    assert torch.equal(both[:, 64:], da)


@pytest.mark.parametrize("interleaved", (False, True))
def test_heads_squares_past_float32(mq, interleaved):
    """Finite heads whose squares pass float32 become zeros, forward and backward, add nothing to the weights' sums, and leave the others alone."""
    c = Heads(mq, 24, 2, 2, 64, (16,), interleaved, BF16, "f32")
    x, dy = rand((24, 256), BF16, 24), rand((24, 256), BF16, 25)
    calm, calm_dy = x.clone(), dy.clone()
    big = {(1, 0): 2.0 ** 66, (2, 1): 2.0 ** 100, (5, 3): 2.0 ** 127, (6, 2): -(2.0 ** 126)}
    for (m, h), v in big.items():
        x[m, 64 * h:64 * h + 64] = v
        calm[m, 64 * h:64 * h + 64] = 0.0
        calm_dy[m, 64 * h:64 * h + 64] = 0.0
    y, z = mq.qk_norm_rope(x, **c.args), mq.qk_norm_rope(calm, **c.args)
    assert torch.equal(y, z)
    (dx, dq, dk), (cx, cq, ck) = mq.qk_norm_rope_grad(dy, x, **c.args), mq.qk_norm_rope_grad(calm_dy, calm, **c.args)
    for m, h in big:
        assert not dx[m, 64 * h:64 * h + 64].any()
    assert torch.equal(dx, cx) and torch.equal(dq, cq) and torch.equal(dk, ck)
    c.check_gradient(calm_dy, calm, dx, dq, dk)


@pytest.mark.parametrize("interleaved", (False, True))
@pytest.mark.parametrize("near", (2 ** 32, -(2 ** 32), 2 ** 44, -(2 ** 44), 2 ** 62, -(2 ** 62)))
def test_heads_positions_of_two_words(mq, near, interleaved):
    """Positions past 32 bits: the oracle's angle is the table's fraction of a turn times the position, modulo a turn, in whole numbers."""
    M = 30
    c = Heads(mq, M, 2, 1, 64, (12, 16), interleaved, F16, pos_type=torch.int64)
    g = torch.Generator().manual_seed(abs(near) % 1000003)
    c.pos.copy_(near + torch.randint(-10 ** 6, 10 ** 6, (M, 2), generator=g))
    table, pos = c.rot.table.cpu().numpy().view(np.uint32), c.pos.tolist()
    turn = [[((int(lo) | int(hi) << 32) * pos[m][int(axis)]) % 2 ** 64 for lo, hi, axis, _ in table] for m in range(M)]
    c.angle = np.array(turn, np.float64) * (2 * np.pi / 2 ** 64)
    c.far_angle = lambda: 2.0 ** -50  # (of the oracle's conversion and product)
    x, dy = rand((M, 192), F16, 26), rand((M, 192), F16, 27)
    c.check_forward(x, mq.qk_norm_rope(x, **c.args))
    c.check_gradient(dy, x, *mq.qk_norm_rope_grad(dy, x, **c.args))


def test_experts_weights_past_32_bits_are_the_first_ones(mq):
    """The same weights as the first expert's and as those of the last, past 2^32 bytes: the same bits, of small blocks too."""
    E, N, K = 34, 8192, 32768
    one = mq.mx_quantize_weights(rand((N, K), F16, 1, 0.02) * torch.logspace(-2, 0, K // 32, 2.0, device="cuda").repeat_interleave(32).half())
    codes = N // 32 * (K // 64) * 1024
    scales = one.data.numel() - codes
    results = []
    for e in (0, E - 1):
        data = torch.zeros(mq.mx_bytes(E * N, K), dtype=torch.uint8, device="cuda")
        data[e * codes:(e + 1) * codes] = one.data[:codes]
        data[E * codes + e * scales:E * codes + (e + 1) * scales] = one.data[codes:]
        w = mq.mx_experts(mq.MxTensor(data, E * N, K), E)
        for M in (3, 300):
            x, dy = rand((M, K), F16, 2), rand((M, N), F16, 3)
            off = torch.tensor([0] * (e + 1) + [M] * (E - e), dtype=torch.int32, device="cuda")
            results += [mq.mx_linear_grouped(x, w, off), mq.mx_linear_grouped_grad(dy, w, off)]
        del w, data
    for a, b in zip(results[:4], results[4:]):
        assert a.any() and torch.equal(a, b)
