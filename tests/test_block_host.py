"""What stands around the microscaled linears of a transformer block, without a GPU: pins of the oracle, and the entry points' refusals (which come before
anything is launched)."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import block as ob
from test_mx_host import lib, overlapping  # noqa: F401


# ------------------------------------------------------------------------------------------------------- oracle pins

def test_turn_by_hand():
    """A quarter turn takes (1, 0) to (0, 1); neighbours or halves; what is past the pairs stays."""
    u = np.array([[[1.0, 2.0, 3.0, 4.0, 5.0, 6.0]]])
    quarter = np.full((1, 2), math.pi / 2)
    assert np.allclose(ob.turn(u, quarter, False), [[[-3, -4, 1, 2, 5, 6]]]) and np.allclose(ob.turn(u, quarter, True), [[[-2, 1, -4, 3, 5, 6]]])
    f, axis = ob.frequencies((2, 1), 100.0)
    assert np.allclose(f, [1.0, 0.1, 1.0]) and axis.tolist() == [0, 0, 1]
    assert np.allclose(ob.frequencies((2, 2), 16.0, restart=False)[0], [1.0, 0.5, 0.25, 0.125])
    assert np.allclose(ob.angles(np.array([[3, -1]]), f, axis), [[3.0, 0.3, -1.0]])


def test_heads_by_hand():
    x = np.array([[[3.0, 4.0]]])
    y = ob.heads(x, np.array([[2.0, 1.0]]), np.zeros((1, 0)), False, 0.0)
    assert np.allclose(y, [[[6 / math.sqrt(12.5), 4 / math.sqrt(12.5)]]])


def test_activations_by_hand():
    """Known values, symmetries (a f(-a) differs from -a + f(a) by nothing), and slopes against differences."""
    assert abs(ob.act(np.array([1.0]), "gelu")[0] - 0.8413447460685429) < 1e-15
    assert abs(ob.act(np.array([1.0]), "silu")[0] - 0.7310585786300049) < 1e-15
    assert abs(ob.act(np.array([1.0]), "gelu_tanh")[0] - 0.5 * (1 + math.tanh(math.sqrt(2 / math.pi) * 1.044715))) < 1e-15
    a = np.linspace(-9, 9, 181)
    for name in ("gelu", "gelu_tanh", "silu"):
        assert np.abs(ob.act(a, name) - ob.act(-a, name) - a).max() < 1e-14
        d = (ob.act(a + 1e-5, name) - ob.act(a - 1e-5, name)) / 2e-5
        assert np.abs(d - ob.slope(a, name)).max() < 1e-9
    v = np.array([[2.0, 3.0, 1.0, -1.0]])
    assert np.allclose(ob.activated(v, "silu", True), [[2 * 0.7310585786300049, -3 * 0.2689414213699951]])


def test_gradients_against_differences():
    """Central differences in 64 bits, h = 1e-5: good to some 1e-9 of values of order 1 to 100."""
    rng = np.random.default_rng(1)
    M, H, D, P, h = 2, 3, 8, 3, 1e-5
    x, w, dy, angle = rng.normal(size=(M, H, D)), rng.normal(1, 0.2, (H, D)), rng.normal(size=(M, H, D)), rng.normal(size=(M, P))
    for inter in (False, True):
        for norm in (True, False):
            f = lambda x, w: float((ob.heads(x, w, angle, inter, 1e-3, norm) * dy).sum())
            ones = w if norm else np.ones((H, D))
            dx, dw = ob.heads_grad(dy, x, ones, angle, inter, 1e-3, norm)
            for at in np.ndindex(M, H, D):
                d = np.zeros_like(x)
                d[at] = h
                assert abs((f(x + d, ones) - f(x - d, ones)) / (2 * h) - dx[at]) < 1e-7
            for at in np.ndindex(H, D) if norm else ():
                d = np.zeros_like(w)
                d[at] = h
                assert abs((f(x, w + d) - f(x, w - d)) / (2 * h) - dw[at]) < 1e-7
    a, g = rng.normal(size=(M, 8)) * 2, rng.normal(size=(M, 8))
    for name in ("gelu", "gelu_tanh", "silu"):
        for gated in (False, True):
            up = g[:, :4] if gated else g
            f = lambda a: float((ob.activated(a, name, gated) * up).sum())
            da = ob.act_grad(up, a, name, gated)
            for at in np.ndindex(*a.shape):
                d = np.zeros_like(a)
                d[at] = h
                assert abs((f(a + d) - f(a - d)) / (2 * h) - da[at]) < 1e-7
    wv, off, rows, dz = rng.normal(size=(2, 4, 32)), [0, 1, 3], rng.normal(size=(3, 32)), rng.normal(size=(3, 4))
    dxg = ob.grouped_grad(dz, wv, off)[0]
    f = lambda a: float((ob.grouped(a, wv, off)[0] * dz).sum())
    for at in ((0, 0), (1, 5), (2, 31)):
        d = np.zeros_like(rows)
        d[at] = h
        assert abs((f(rows + d) - f(rows - d)) / (2 * h) - dxg[at]) < 1e-7


# ------------------------------------------------------------------------------------------------------ rotation's table

def test_rotary_table(lib):
    """Fractions of a turn in 64 bits, against whole numbers; negative and whole turns; the axes."""
    freq = np.array([2 * math.pi / 8, 1.0, -1.0, 2 * math.pi, 0.0, 1e-9, 100.0])
    axis = np.array([0, 1, 2, 3, 0, 1, 2], np.int32)
    table = np.zeros((7, 4), np.uint32)
    p = lambda a: C.c_void_p(a.ctypes.data)
    assert lib.mq_rotary_table(p(freq), p(axis), 7, p(table)) == 0
    turns = [int(lo) | int(hi) << 32 for lo, hi in table[:, :2]]
    from fractions import Fraction
    pi2 = Fraction(6283185307179586476925286766559, 10 ** 30)  # 2 pi to 31 digits
    for t, f in zip(turns, freq):
        want = Fraction(f) / pi2 % 1 * 2 ** 64
        off = abs(want - t)
        # the frequency itself is exact; the quotient is taken in the host's extended type, 64 bits of it
        assert min(off, 2 ** 64 - off) <= 1 + abs(Fraction(f) / pi2) * 2
    assert turns[0] == 1 << 61 or abs(turns[0] - (1 << 61)) < 1 << 11  # (a double's 2 pi / 8)
    assert turns[1] + turns[2] == 1 << 64 and turns[4] == 0 and table[:, 2].tolist() == axis.tolist() and not table[:, 3].any()
    assert lib.mq_rotary_table(p(freq), p(axis), 0, C.c_void_p(0)) == 0
    assert lib.mq_rotary_table(C.c_void_p(0), p(axis), 1, p(table)) == -1 and lib.mq_rotary_table(p(freq), p(axis), -1, p(table)) == -2
    for bad, at in ((np.array([np.nan]), 0), (np.array([np.inf]), 0), (np.array([1.0]), 4), (np.array([1.0]), -1)):
        assert lib.mq_rotary_table(p(bad), p(np.array([at], np.int32)), 1, p(table)) == -1


def test_rotary_handle(lib):
    import paper_2405_17873_amd as mq
    r = mq.rotary((4, 0, 8), interleaved=True, device="cpu")
    assert (r.pairs, r.axes, r.interleaved, tuple(r.table.shape)) == (12, 3, True, (12, 4)) and r.table[:, 2].tolist() == [0] * 4 + [2] * 8
    assert (mq.rotary((4, 4), restart=False, device="cpu").table[:, :2] == mq.rotary((8,), device="cpu").table[:, :2]).all()
    for bad in ((3,), (4,) * 5, (), (-4, 8), (0,)):
        with pytest.raises(ValueError):
            mq.rotary(bad, device="cpu")
    with pytest.raises(ValueError):
        mq.rotary((4,), freqs=[1.0] * 5, device="cpu")


# ---------------------------------------------------------------------------------------------------------- refusals

def pointer():
    buf = (C.c_uint8 * (1 << 17))()
    return buf, C.c_void_p((C.addressof(buf) + 255) // 256 * 256)  # aligned fake pointer; every call below fails before it is used


def test_error_codes_of_heads(lib):
    buf, p = pointer()
    null, odd, st, L, f = C.c_void_p(0), C.c_void_p(p.value + 1), C.c_void_p(0), C.c_long, C.c_float
    far = C.c_void_p(p.value + (1 << 30))

    def call(x=p, M=4, q=2, k=2, D=64, ld=256, qw=null, kw=null, pt=2, eps=1e-6, norm=1, table=p, pairs=32, pos=p, bytes_=4, axes=1, ldpos=1, y=far, ldy=256, dt=0):
        return lib.mq_qk_norm_rope(x, M, q, k, D, L(ld), qw, kw, pt, f(eps), norm, table, pairs, 0, pos, bytes_, axes, L(ldpos), y, L(ldy), dt, st)

    for kw in (dict(x=null), dict(x=odd), dict(y=null), dict(y=odd), dict(dt=2), dict(dt=-1), dict(qw=p, pt=3), dict(qw=C.c_void_p(p.value + 2), pt=2), dict(kw=odd, pt=0), dict(eps=-1.0),
               dict(eps=math.nan), dict(norm=0, qw=p), dict(norm=0, kw=p), dict(table=null), dict(table=C.c_void_p(p.value + 8)), dict(pos=null), dict(pos=C.c_void_p(p.value + 2)),
               dict(pos=C.c_void_p(p.value + 4), bytes_=8), dict(bytes_=2), dict(y=C.c_void_p(p.value + 2)), dict(y=p, ldy=512)):
        assert call(**kw) == -1, kw
    for kw in (dict(M=-1), dict(q=-1), dict(q=0, k=0), dict(q=4097), dict(D=0), dict(D=60), dict(D=520, ld=4096, ldy=4096), dict(ld=255), dict(ldy=255), dict(pairs=30), dict(pairs=36),
               dict(pairs=-4), dict(axes=0), dict(axes=5, ldpos=5), dict(axes=2, ldpos=1), dict(M=1 << 28, q=4096, ld=1 << 20, ldy=1 << 20)):
        assert call(**kw) == -2, kw
    assert call(M=0, x=null, y=null, pos=null) == 0
    need = lib.mq_qk_norm_rope_grad_workspace_bytes(4, 2, 2, 64)
    assert need >= 2 * 64 * 4 and lib.mq_qk_norm_rope_grad_workspace_bytes(0, 2, 2, 64) == 0

    def grad(dy=p, x=p, dx=far, lddx=256, dq=p, dk=p, ws=p, n=need, norm=1, lddy=256):
        return lib.mq_qk_norm_rope_grad(dy, L(lddy), x, 4, 2, 2, 64, L(256), null, null, 2, f(1e-6), norm, p, 32, 0, p, 4, 1, L(1), dx, L(lddx), 0, dq, dk, ws, C.c_size_t(n), st)

    assert grad(dy=null) == -1 and grad(x=null) == -1 and grad(dx=null) == -1 and grad(dq=C.c_void_p(p.value + 2)) == -1 and grad(ws=null) == -1
    assert grad(ws=C.c_void_p(p.value + 64)) == -1 and grad(n=need - 1) == -4 and grad(norm=0) == -1 and grad(lddy=200) == -2 and grad(lddx=200) == -2
    assert grad(dx=C.c_void_p(p.value + 2)) == -1 and grad(dx=C.c_void_p(p.value + 2), norm=0, dq=null, dk=null) == -1


def test_error_codes_of_activations(lib):
    buf, p = pointer()
    null, odd, st, L = C.c_void_p(0), C.c_void_p(p.value + 1), C.c_void_p(0), C.c_long
    far, further = C.c_void_p(p.value + (1 << 30)), C.c_void_p(p.value + (1 << 31))

    def call(codes, M=4, K=64, N=64, x=p, w=p, bias=null, act=1, gated=0, y=far, ldy=64, dt=0, res=null, ldr=64, pre=further, ldpre=64, ws=p, n=1 << 20):
        tail = (w, N, bias, act, gated, y, L(ldy), dt, res, L(ldr), pre, L(ldpre))
        if codes:
            return lib.mq_mx_linear_act_codes(x, M, K, *tail, st)
        return lib.mq_mx_linear_act(x, M, K, L(K), *tail, ws, C.c_size_t(n), st)

    for codes in (0, 1):
        for kw in (dict(x=null), dict(w=null), dict(y=null), dict(y=odd), dict(bias=odd), dict(act=-1), dict(act=4), dict(gated=1, act=0), dict(gated=1, res=p), dict(dt=2), dict(res=odd), dict(pre=odd),
                   dict(pre=far), dict(pre=C.c_void_p(far.value + 2)), dict(res=C.c_void_p(far.value + 2)), dict(res=further), dict(pre=further, res=C.c_void_p(further.value + 100))):
            assert call(codes, **kw) == -1, (codes, kw)
        for kw in (dict(M=-1), dict(N=0), dict(K=48), dict(gated=1, N=96), dict(ldy=63), dict(ldpre=63), dict(res=p, ldr=63), dict(gated=1, ldy=31), dict(N=(1 << 22) + 64, ldy=1 << 23, ldpre=1 << 23),
                   dict(gated=1, N=1 << 22, K=2048, ldy=1 << 23, ldpre=1 << 23)):
            assert call(codes, **kw) == -2, (codes, kw)
        assert call(codes, M=0, x=null, y=null, pre=null) == 0
    assert call(0, M=100, ws=null) == -1 and call(0, M=100, n=100) == -4
    assert call(0, ws=null, y=p, pre=null) == -1 and call(0, ws=null, pre=p) == -1  # results over the activations go by the workspace

    def grad(dy=p, pre=p, M=4, N=64, act=1, gated=0, da=far, lddy=64, ldpre=64, ldda=64, dt=0, dbias=p, ws=p, n=1 << 20):
        return lib.mq_act_grad(dy, M, N, L(lddy), pre, L(ldpre), act, gated, da, L(ldda), dt, dbias, ws, C.c_size_t(n), st)

    for kw in (dict(dy=null), dict(dy=odd), dict(pre=null), dict(da=null), dict(act=0), dict(act=4), dict(dt=2), dict(dbias=C.c_void_p(p.value + 2)), dict(ws=null), dict(ws=odd),
               dict(da=C.c_void_p(p.value + 2)), dict(da=p, ldda=128), dict(gated=1, dy=far, da=far), dict(gated=1, dy=far, pre=p, da=C.c_void_p(far.value - 64))):
        assert grad(**kw) == -1, kw
    for kw in (dict(M=-1), dict(N=0), dict(gated=1, N=63), dict(lddy=63), dict(ldpre=63), dict(ldda=63), dict(M=(1 << 28) + 1), dict(N=(1 << 22) + 2, lddy=1 << 23, ldpre=1 << 23, ldda=1 << 23)):
        assert grad(**kw) == -2, kw
    assert grad(n=lib.mq_act_grad_workspace_bytes(4, 64, 0) - 1) == -4


def test_error_codes_of_experts(lib):
    buf, p = pointer()
    null, odd, st, L = C.c_void_p(0), C.c_void_p(p.value + 1), C.c_void_p(0), C.c_long
    far, further = C.c_void_p(p.value + (1 << 30)), C.c_void_p(p.value + (1 << 31))

    def call(x=p, M=100, K=64, ldx=64, w=p, N=64, E=2, off=p, bias=null, act=1, gated=0, y=far, ldy=64, dt=0, pre=further, ldpre=64, ws=p, n=1 << 24):
        return lib.mq_mx_linear_grouped(x, M, K, L(ldx), w, N, E, off, bias, act, gated, y, L(ldy), dt, pre, L(ldpre), ws, C.c_size_t(n), st)

    for kw in (dict(x=null), dict(x=odd), dict(w=null), dict(w=C.c_void_p(p.value + 64)), dict(off=null), dict(off=C.c_void_p(p.value + 2)), dict(bias=odd), dict(act=4), dict(gated=1, act=0), dict(y=null),
               dict(y=odd), dict(dt=2), dict(pre=odd), dict(pre=far), dict(y=p), dict(pre=p), dict(y=C.c_void_p(p.value + 2)), dict(ws=null), dict(ws=C.c_void_p(p.value + 64))):
        assert call(**kw) == -1, kw
    for kw in (dict(M=-1), dict(K=48), dict(N=0), dict(N=48), dict(E=0), dict(E=4097), dict(E=4096, N=1 << 17), dict(gated=1, N=32), dict(ldx=63), dict(ldy=63), dict(ldpre=63), dict(M=(1 << 28) + 1),
               dict(gated=1, N=1 << 22, K=2048, ldx=4096, E=1, ldy=1 << 23, ldpre=1 << 23)):
        assert call(**kw) == -2, kw
    need = lib.mq_mx_linear_grouped_workspace_bytes(100, 64, 64, 2)
    assert need >= lib.mq_mx_bytes(100, 64) and call(n=need - 1) == -4 and lib.mq_mx_linear_grouped_workspace_bytes(0, 64, 64, 2) == 0
    assert lib.mq_mx_linear_grouped_workspace_bytes(20, 64, 64, 2) == 0 and call(M=0, x=null, y=null, pre=null) == 0

    def grad(dy=p, M=100, N=64, lddy=64, w=p, top=p, K=64, E=2, off=p, dx=far, lddx=64, dt=0):
        return lib.mq_mx_linear_grouped_grad(dy, M, N, L(lddy), w, top, K, E, off, dx, L(lddx), dt, st)

    for kw in (dict(dy=null), dict(w=null), dict(top=null), dict(off=null), dict(dx=null), dict(dx=odd), dict(dt=3), dict(dx=p), dict(dx=C.c_void_p(p.value + 2))):
        assert grad(**kw) == -1, kw
    for kw in (dict(M=-1), dict(K=40), dict(N=40), dict(E=0), dict(lddy=63), dict(lddx=63)):
        assert grad(**kw) == -2, kw
    assert grad(M=0, dy=null, dx=null) == 0
    top = lambda mx=p, E=2, N=64, K=64, t=p: lib.mq_mx_experts_column_top(mx, E, N, K, t, st)
    assert top(mx=null) == -1 and top(t=null) == -1 and top(E=0) == -2 and top(N=40) == -2 and top(K=40) == -2


def test_python_refusals(lib):
    """Operands on the host, rows that overlap, and what autograd would have to go through."""
    import torch

    import paper_2405_17873_amd as mq
    x, v = torch.zeros(4, 64, dtype=torch.float16), torch.zeros(32)
    w = mq.MxTensor(torch.zeros(mq.mx_bytes(64, 64), dtype=torch.uint8), 64, 64, torch.zeros(2, dtype=torch.uint8))
    off = torch.zeros(2, dtype=torch.int32)
    calls = lambda t: (lambda: mq.qk_norm_rope(t, 1, 1), lambda: mq.qk_norm_rope_grad(t, t, 1, 1), lambda: mq.mx_linear(t, w, act="gelu"), lambda: mq.act_grad(t, t, "silu"),
                       lambda: mq.mx_linear_grouped(t, w, off), lambda: mq.mx_linear_grouped_grad(t, w, off))
    for call in calls(x):
        with pytest.raises(ValueError):
            call()
    for t in overlapping():
        for call in calls(t):
            with pytest.raises(ValueError, match="overlap"):
                call()
    for call in calls(x.clone().requires_grad_()):
        with pytest.raises(RuntimeError, match="graph"):
            call()
    with pytest.raises(RuntimeError, match="graph"):
        mq.qk_norm_rope(x, 1, 1, v.requires_grad_())
    with pytest.raises(ValueError):
        mq.mx_linear(w, w, act="gelu")
    for bad in ("relu", "GELU", 1):
        with pytest.raises(ValueError):
            mq.mx_linear(x, w, act=bad)


def test_experts_on_another_device(lib, monkeypatch):
    """Weights on another device than the current one are refused before anything is allocated or launched there."""
    import torch
    from types import SimpleNamespace as Object

    import paper_2405_17873_amd as mq
    device = torch.device("cuda:1")
    buffer = Object(device=device, dtype=torch.uint8, is_cuda=True, is_contiguous=lambda: True, numel=lambda: 1 << 20, stride=lambda: (1,), data_ptr=lambda: 0)
    weights = Object(device=device, shape=(2, 32, 32), dim=lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for call in (lambda: mq.mx_experts(mq.MxTensor(buffer, 64, 64), 2), lambda: mq.mx_quantize_experts(weights)):
        with pytest.raises(ValueError, match="current device"):
            call()


def test_sizes_past_32_bits(lib):
    """2^32 + 4 rows are refused, not taken for 4: matrices without memory behind them, and a microscaled one made by hand."""
    import torch

    import paper_2405_17873_amd as mq
    rows = 2 ** 32 + 4
    t = torch.empty(rows, 64, dtype=torch.float16, device="meta")
    w = mq.MxTensor(torch.zeros(mq.mx_bytes(64, 64), dtype=torch.uint8), 64, 64, torch.zeros(2, dtype=torch.uint8))
    off = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: mq.qk_norm_rope(t, 1, 1), lambda: mq.qk_norm_rope_grad(t, t, 1, 1), lambda: mq.mx_linear(t, w, act="gelu"), lambda: mq.act_grad(t, t, "silu"),
                 lambda: mq.mx_linear_grouped(t, w, off), lambda: mq.mx_linear_grouped_grad(t, w, off), lambda: mq.mx_linear(t, w), lambda: mq.mx_linear_grad(t, w),
                 lambda: mq.layer_norm(t), lambda: mq.mx_quantize(t), lambda: mq.mx_dequantize(mq.MxTensor(w.data, rows, 64)),
                 lambda: mq.mx_pack(torch.empty(rows, 32, dtype=torch.uint8, device="meta"), torch.empty(rows, 2, dtype=torch.uint8, device="meta"))):
        with pytest.raises(ValueError, match="below 2.31"):
            call()
