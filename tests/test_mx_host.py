"""Microscaled 4-bit floats, layer norm and gradients, without a GPU: pins of the oracle, and the entry points' refusals (which come
before anything is launched)."""
import ctypes as C
import os

import numpy as np
import pytest

from oracle import mx as omx


@pytest.fixture(scope="module")
def lib():
    import paper_2405_17873_amd as mq
    if not os.path.exists(mq.lib_path()):
        from paper_2405_17873_amd import build
        build.build()
    return mq.load()


# ------------------------------------------------------------------------------------------------------- oracle pins

def test_block_by_hand():
    """Largest magnitude 5: 2^2, unit 1.  Every border of the codes, ties to the even code."""
    x = np.zeros((1, 32))
    x[0, :16] = [5.0, 0.25, 0.2500001, 0.75, 1.25, 1.75, 2.5, 3.5, -5.0, -0.25, -0.74, -1.26, -1.76, -2.51, -3.49, 4.999]
    c, s = omx.quantize(x)
    assert s.tolist() == [[127]]
    want = [4.0, 0.0, 0.5, 1.0, 1.0, 2.0, 2.0, 4.0, -4.0, -0.0, -0.5, -1.5, -2.0, -3.0, -3.0, 4.0]
    assert omx.decode(c, s)[0, :16].tolist() == want
    assert np.signbit(omx.decode(c, s)[0, 9])


def test_scales_by_hand():
    for top, byte in ((1.0, 125), (1.999, 125), (2.0, 126), (7.99, 127), (65504.0, 140), (2.0 ** -24, 101), (0.0, 0), (2.0 ** -133, 0),
                      (2.0 ** -125, 0), (2.0 ** -124, 1), (2.0 ** 127, 252), (np.inf, 255), (np.nan, 255)):
        x = np.zeros((1, 64))
        x[0, 5], x[0, 40] = top, -1.0
        assert omx.scale_bytes(x).tolist() == [[byte, 125]], top


def test_values_saturate_and_round_trip():
    x = np.zeros((1, 32))
    x[0, :3] = [7.99, -7.0, 6.9]
    assert omx.values(x)[0, :3].tolist() == [6.0, -6.0, 6.0]
    rng = np.random.default_rng(0)
    v = omx.values(rng.normal(size=(5, 96)))
    assert np.array_equal(omx.values(v), v) or np.abs(v).max() > 0  # values of a saturated block may take a smaller scale
    c, s = omx.quantize(rng.normal(size=(3, 64)))
    assert np.array_equal(omx.unflat(omx.flat(c)), c)


def test_gradients_against_differences():
    """The gradient formulas against central differences of the forward formulas in 64 bits: h = 1e-5, so that the differences are good to about
    h^2 and 1e-16 / h, some 1e-9 of values of order 1 to 100."""
    rng = np.random.default_rng(1)
    M, K, eps, h = 3, 17, 1e-5, 1e-5
    x, w, b, dy, res = rng.normal(size=(M, K)), rng.normal(1, 0.1, K), rng.normal(size=K), rng.normal(size=(M, K)), rng.normal(size=(M, K))
    f = lambda x, w, b: float((omx.norm(x, w, b, eps) * dy).sum() + (x * res).sum())
    dx, dw, db = omx.norm_grad(dy, x, w, *omx.norm_stats(x, eps), residual=res)
    for m in range(M):
        for k in range(K):
            d = np.zeros_like(x)
            d[m, k] = h
            assert abs((f(x + d, w, b) - f(x - d, w, b)) / (2 * h) - dx[m, k]) < 1e-7
    for k in range(K):
        d = np.zeros(K)
        d[k] = h
        assert abs((f(x, w + d, b) - f(x, w - d, b)) / (2 * h) - dw[k]) < 1e-7
        assert abs((f(x, w, b + d) - f(x, w, b - d)) / (2 * h) - db[k]) < 1e-7
    wq, g = omx.values(rng.normal(size=(5, 32))), rng.normal(size=(M, 5))
    a = rng.normal(size=(M, 32))
    fl = lambda a: float((omx.linear(a, wq)[0] * g).sum())
    dxl = omx.linear_grad(g, wq)[0]
    for m, k in ((0, 0), (1, 31), (2, 7)):
        d = np.zeros_like(a)
        d[m, k] = h
        assert abs((fl(a + d) - fl(a - d)) / (2 * h) - dxl[m, k]) < 1e-7


def test_norm_by_hand():
    x = np.array([[1.0, 3.0]])
    assert np.allclose(omx.norm(x, np.array([2.0, 4.0]), np.array([0.5, 0.0]), 0.0), [[-1.5, 4.0]])
    mean, rstd = omx.norm_stats(np.full((1, 5), 7.0), 1e-4)
    assert mean[0, 0] == 7.0 and abs(rstd[0, 0] - 100.0) < 1e-10


# ---------------------------------------------------------------------------------------------------------- refusals

def test_sizes(lib):
    import paper_2405_17873_amd as mq
    assert mq.mx_bytes(32, 64) == 1024 + 256
    assert mq.mx_bytes(33, 96) == 2 * 2 * 1024 + 2 * 256
    assert mq.mx_bytes(1, 320) == 5 * 1024 + 2 * 256
    assert mq.mx_bytes(4, 48) == 0 and mq.mx_bytes(-1, 64) == 0 and mq.mx_bytes(0, 64) == 0
    assert mq.mx_linear_workspace_bytes(4, 8, 64) == 0  # a few rows are quantised in the product
    assert mq.mx_linear_workspace_bytes(64, 8, 64) >= mq.mx_bytes(64, 64)
    assert mq.mx_linear_workspace_bytes(0, 8, 64) == 0
    assert mq.layer_norm_grad_workspace_bytes(1, 8) >= 64 and mq.layer_norm_grad_workspace_bytes(0, 8) == 0


def test_error_codes_without_a_gpu(lib):
    buf = (C.c_uint8 * 4096)()
    p = C.c_void_p((C.addressof(buf) + 255) // 256 * 256)  # aligned fake pointer; every call below fails before it is used
    odd, off = C.c_void_p(p.value + 1), C.c_void_p(p.value + 64)
    null, st = C.c_void_p(0), C.c_void_p(0)
    L = C.c_long
    q = lambda x=p, M=4, K=64, ld=64, dt=0, mx=p: lib.mq_mx_quantize(x, M, K, L(ld), dt, mx, st)
    assert q(x=null) == -1 and q(x=odd) == -1 and q(mx=null) == -1 and q(mx=off) == -1 and q(dt=2) == -1
    assert q(M=-1) == -2 and q(K=48) == -2 and q(K=0) == -2 and q(ld=63) == -2 and q(K=(1 << 21) + 32, ld=1 << 22) == -2
    d = lambda mx=p, M=4, K=64, dt=0, y=p, ld=64: lib.mq_mx_dequantize(mx, M, K, dt, y, L(ld), st)
    assert d(mx=null) == -1 and d(y=null) == -1 and d(dt=7) == -1 and d(ld=32) == -2 and d(K=40) == -2
    assert lib.mq_mx_pack(null, p, 4, 64, p, st) == -1 and lib.mq_mx_pack(p, null, 4, 64, p, st) == -1 and lib.mq_mx_pack(p, p, 4, 65, p, st) == -2
    assert lib.mq_mx_unpack(p, 4, 64, p, null, st) == -1 and lib.mq_mx_unpack(null, 4, 64, p, p, st) == -1
    assert lib.mq_mx_column_top(p, 4, 64, null, st) == -1 and lib.mq_mx_column_top(p, 4, 72, p, st) == -2
    lin = lambda x=p, M=4, K=64, ldx=64, w=p, N=8, b=null, y=p, ldy=8, dt=0, r=null, ldr=0, ws=p, wsb=4096: lib.mq_mx_linear(
        x, M, K, L(ldx), w, N, b, y, L(ldy), dt, r, L(ldr), ws, C.c_size_t(wsb), st)
    far = C.c_void_p(p.value + (1 << 30))
    assert lin(x=null) == -1 and lin(w=null) == -1 and lin(w=off) == -1 and lin(y=null) == -1
    assert lin(ws=null) == -1 and lin(ws=off) == -1                     # (Y overlaps X)
    assert lin(M=64, y=far, ws=null) == -1 and lin(M=64, y=far, ws=off) == -1
    assert lin(dt=2) == -1 and lin(b=odd) == -1 and lin(r=odd, ldr=8) == -1
    assert lin(M=-1) == -2 and lin(N=0) == -2 and lin(K=33) == -2 and lin(ldx=32) == -2 and lin(ldy=7) == -2 and lin(r=p, ldr=7) == -2
    assert lin(N=(1 << 22) + 1, ldy=1 << 23) == -2
    assert lin(wsb=100) == -4
    code = lambda a=p, M=4, K=64, y=p, ldy=8: lib.mq_mx_linear_codes(a, M, K, p, 8, null, y, L(ldy), 0, null, L(0), st)
    assert code(a=null) == -1 and code(a=off) == -1 and code(y=null) == -1 and code(ldy=4) == -2 and code(K=63) == -2
    gr = lambda dy=p, M=4, N=8, ld=8, w=p, top=p, K=64, dx=p, lddx=64, dt=0, ws=null, wsb=0: lib.mq_mx_linear_grad(
        dy, M, N, L(ld), w, top, K, dx, L(lddx), dt, ws, C.c_size_t(wsb), st)
    assert gr(dy=null) == -1 and gr(w=null) == -1 and gr(top=null) == -1 and gr(dx=null) == -1 and gr(dt=3) == -1
    assert gr(M=-1) == -2 and gr(N=0) == -2 and gr(K=31) == -2 and gr(ld=7) == -2 and gr(lddx=63) == -2
    need = lib.mq_mx_linear_grad_workspace_bytes(4, 16384, 64)  # a long reduction of few results is cut into parts
    assert need > 0 and gr(N=16384, ld=16384) == -1 and gr(N=16384, ld=16384, ws=p, wsb=need - 1) == -4 and gr(N=16384, ld=16384, ws=off, wsb=need) == -1
    f = C.c_float
    ln = lambda x=p, M=4, N=64, ld=64, w=null, b=null, pt=2, eps=1e-5, y=p, ldy=64, dt=0: lib.mq_layer_norm(
        x, M, N, L(ld), w, b, pt, f(eps), y, L(ldy), dt, null, null, st)
    assert ln(x=null) == -1 and ln(y=null) == -1 and ln(dt=2) == -1 and ln(w=p, pt=5) == -1 and ln(w=C.c_void_p(p.value + 2)) == -1
    assert ln(eps=-1.0) == -1 and ln(eps=float("nan")) == -1
    assert ln(M=-1) == -2 and ln(N=0) == -2 and ln(N=16385, ld=20000, ldy=20000) == -2 and ln(ld=63) == -2 and ln(ldy=63) == -2
    lm = lambda N=64, mx=p: lib.mq_layer_norm_mx(p, 4, N, L(128), null, null, 2, f(1e-5), mx, 0, null, null, st)
    assert lm(N=48) == -2 and lm(mx=null) == -1 and lm(mx=off) == -1
    lg = lambda dy=p, M=4, N=64, mean=p, rstd=p, r=null, ldr=0, dx=p, lddx=64, ws=p, wsb=1 << 20: lib.mq_layer_norm_grad(
        dy, L(64), p, L(64), M, N, null, 2, mean, rstd, r, L(ldr), dx, L(lddx), 0, p, p, ws, C.c_size_t(wsb), st)
    assert lg(dy=null) == -1 and lg(mean=null) == -1 and lg(rstd=null) == -1 and lg(dx=null) == -1 and lg(ws=null) == -1 and lg(ws=off) == -1
    assert lg(M=-1) == -2 and lg(lddx=63) == -2 and lg(r=p, ldr=63) == -2 and lg(wsb=255) == -4
    # no rows: nothing to point to, nothing launched
    assert q(M=0, x=null, mx=null) == 0 and d(M=0, mx=null, y=null) == 0 and lin(M=0, x=null, y=null, ws=null, wsb=0) == 0
    assert code(M=0, a=null, y=null) == 0 and gr(M=0, dy=null, dx=null) == 0 and ln(M=0, x=null, y=null) == 0


def test_python_refusals_without_a_gpu(lib):
    import torch

    import paper_2405_17873_amd as mq
    x = torch.zeros(4, 64, dtype=torch.float16)
    for call in (lambda: mq.mx_quantize(x), lambda: mq.layer_norm(x), lambda: mq.mx_linear(x, None)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        mq.mx_pack(x, x)


def test_grad_workspace_of_copied_rows(lib):
    """Reductions that are no multiple of eight need room for their rows."""
    need = lambda N: lib.mq_mx_linear_grad_workspace_bytes(300, N, 352)
    assert need(1003) >= need(1008) + 300 * 1008 * 2 and need(1000) == need(1008)


def overlapping():
    """Matrices [4, 64] whose rows lie on or over one another: a broadcast row, and rows 16 values apart."""
    import torch
    v = torch.zeros(256, dtype=torch.float16)
    return v[:64].expand(4, 64), v.as_strided((4, 64), (16, 1))


def test_row_strides_are_the_tensors_own(lib):
    """A stride below the row reaches the entry points as it is, which refuse it: a larger one would have them read past the allocation."""
    import torch

    from paper_2405_17873_amd import binding
    assert [binding._ld(t).value for t in overlapping()] == [0, 16]
    assert binding._ld(torch.zeros(4, 80)[:, :64]).value == 80
    assert binding._ld(torch.zeros(1, 64).as_strided((1, 64), (7, 1))).value == 64  # a single row's stride says nothing
    assert binding._ld(torch.zeros(0, 64)).value == 64


def test_overlapping_rows_are_refused(lib):
    import torch

    import paper_2405_17873_amd as mq
    w = mq.MxTensor(torch.zeros(mq.mx_bytes(64, 64), dtype=torch.uint8), 64, 64, torch.zeros(2, dtype=torch.uint8))
    stats = torch.zeros(4)
    for t in overlapping():
        for call in (lambda: mq.mx_quantize(t), lambda: mq.mx_linear(t, w), lambda: mq.mx_linear_grad(t, w), lambda: mq.layer_norm(t), lambda: mq.layer_norm_mx(t),
                     lambda: mq.mx_dequantize(w, torch.float16, out=t), lambda: mq.layer_norm_grad(t, t, None, stats, stats)):
            with pytest.raises(ValueError, match="overlap"):
                call()


def test_buffers_are_looked_at(lib):
    """What a microscaled matrix carries, its column scales and workspaces: on the host, too short, of another type or not contiguous."""
    import dataclasses

    import torch

    import paper_2405_17873_amd as mq
    from paper_2405_17873_amd import binding
    n = mq.mx_bytes(64, 64)
    on_host = mq.MxTensor(torch.zeros(n, dtype=torch.uint8), 64, 64, torch.zeros(2, dtype=torch.uint8))
    bad = [on_host] + [dataclasses.replace(on_host, data=d) for d in (torch.zeros(n - 1, dtype=torch.uint8), torch.zeros(n, dtype=torch.int8),
                                                                     torch.zeros(1, dtype=torch.uint8).expand(n), torch.zeros(2 * n, dtype=torch.uint8)[::2])]
    for t in bad:
        for call in (lambda: mq.mx_dequantize(t), lambda: mq.mx_unpack(t), lambda: mq.mx_linear(t, on_host), lambda: binding._with_top(t)):
            with pytest.raises(ValueError):
                call()
    for t, what in zip(bad, ("on", "bytes", "bytes", "bytes", "bytes")):
        with pytest.raises(ValueError, match=what):
            binding._mx_data(t)
    cpu = torch.device("cpu")
    for ws in (torch.zeros(512, dtype=torch.uint8)[::2], torch.zeros(1, dtype=torch.uint8).expand(512), torch.zeros(512, dtype=torch.uint8, device="meta")):
        with pytest.raises(ValueError):
            binding._mx_workspace(256, cpu, ws)
    assert binding._mx_workspace(256, cpu, None).numel() == 256


def test_once_per_device(tmp_path):
    """What kernels with much LDS are prepared with: done on every device, once, and again after a failure."""
    import re
    import subprocess
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2405_17873_amd", "csrc")
    (tmp_path / "t.cpp").write_text("""
#include <stdio.h>
#include "per_device.h"
int main() {
    static mq::PerDevice prepared;
    int calls = 0, fail = 0;
    auto f = [&] { ++calls; return fail; };
    for (int d : {0, 0, 1, 0, 1, 15}) prepared(d, f);
    printf("%d ", calls);
    fail = 7;
    const int a = prepared(2, f), b = prepared(2, f), c = prepared(0, f);
    fail = 0;
    const int d = prepared(2, f), e = prepared(2, f);
    printf("%d %d %d %d %d %d ", calls, a, b, c, d, e);
    prepared(99, f), prepared(99, f), prepared(-1, f);
    printf("%d", calls);
}""")
    subprocess.run(["g++", "-std=c++17", "-I", csrc, str(tmp_path / "t.cpp"), "-o", str(tmp_path / "t"), "-pthread"], check=True)
    assert subprocess.run([str(tmp_path / "t")], check=True, capture_output=True, text=True).stdout.split() == "3 6 7 7 0 0 0 9".split()
    for name in sorted(os.listdir(csrc)):
        if name.startswith("mx_"):
            for line in open(os.path.join(csrc, name)):
                assert not re.search(r"static\s+const\s+hipError_t", line), f"{name} keeps one device's answer for all: {line}"


def test_graphs_are_refused(lib):
    """A result that autograd would have to know of is refused, with the operands as they come; without autograd the same operands pass that check."""
    import torch

    import paper_2405_17873_amd as mq
    x, p = torch.zeros(4, 64, dtype=torch.float16), torch.zeros(64)
    w = mq.MxTensor(torch.zeros(mq.mx_bytes(64, 64), dtype=torch.uint8), 64, 64, torch.zeros(2, dtype=torch.uint8))
    gx, gp, gb = (t.clone().requires_grad_() for t in (x, p, p.half()))
    calls = (lambda: mq.mx_linear(gx, w), lambda: mq.mx_linear(x, w, gb), lambda: mq.mx_linear(x, w, residual=gx), lambda: mq.mx_linear(w, w, gb),
             lambda: mq.layer_norm(gx), lambda: mq.layer_norm(x, gp, p), lambda: mq.layer_norm(x, p, gp), lambda: mq.layer_norm_mx(gx), lambda: mq.layer_norm_mx(x, gp),
             lambda: mq.mx_linear_grad(gx, w), lambda: mq.layer_norm_grad(gx, x, p, p, p))
    for call in calls:
        with pytest.raises(RuntimeError, match="graph"):
            call()
        with torch.no_grad(), pytest.raises(ValueError):  # (on the host)
            call()


def test_float_pointers_are_looked_at(lib):
    """Statistics and sums are float32: addresses off four bytes are refused, and so are 16-bit operands off two."""
    buf = (C.c_uint8 * 4096)()
    p = C.c_void_p((C.addressof(buf) + 255) // 256 * 256)  # every call below fails before it is used
    half, null, st, L, f = C.c_void_p(p.value + 2), C.c_void_p(0), C.c_void_p(0), C.c_long, C.c_float
    ln = lambda mean=null, rstd=null: lib.mq_layer_norm(p, 4, 64, L(64), null, null, 2, f(1e-5), p, L(64), 0, mean, rstd, st)
    lm = lambda mean=null, rstd=null: lib.mq_layer_norm_mx(p, 4, 64, L(64), null, null, 2, f(1e-5), p, 0, mean, rstd, st)
    assert ln(mean=half) == -1 and ln(rstd=half) == -1 and lm(mean=half) == -1 and lm(rstd=half) == -1
    lg = lambda mean=p, rstd=p, dw=p, db=p: lib.mq_layer_norm_grad(p, L(64), p, L(64), 4, 64, null, 2, mean, rstd, null, L(0), p, L(64), 0, dw, db, p,
                                                                   C.c_size_t(1 << 20), st)
    assert lg(mean=half) == -1 and lg(rstd=half) == -1 and lg(dw=half) == -1 and lg(db=half) == -1


def test_sizes_past_the_limits(lib):
    """A size that no call takes has no bytes."""
    import paper_2405_17873_amd as mq
    assert mq.mx_bytes(4, 1 << 21) > 0 and mq.mx_bytes(4, (1 << 21) + 32) == 0
    assert mq.mx_bytes(1 << 28, 32) > 0 and mq.mx_bytes((1 << 28) + 1, 32) == 0


def test_outputs_over_operands_are_refused(lib):
    """An output that lies over an operand without being that operand, row for row."""
    buf = (C.c_uint8 * 65536)()
    p = C.c_void_p((C.addressof(buf) + 255) // 256 * 256)  # every call below fails before it is used
    null, st, L, f = C.c_void_p(0), C.c_void_p(0), C.c_long, C.c_float
    at = lambda values: C.c_void_p(p.value + 2 * values)
    far = C.c_void_p(p.value + (1 << 30))
    gr = lambda dx=p, lddx=64, K=64, N=64, ld=64: lib.mq_mx_linear_grad(p, 4, N, L(ld), far, far, K, dx, L(lddx), 0, null, C.c_size_t(0), st)
    assert gr() == -1 and gr(dx=at(255)) == -1 and gr(dx=at(64)) == -1 and gr(dx=at(63), lddx=128, ld=128) == -1 and gr(dx=at(-255)) == -1
    assert gr(dx=at(64), lddx=128, ld=127) == -1  # rows of another distance: taken as one over the other
    lin = lambda r, ldr, y=p, ldy=64, M=40, codes=0: (lib.mq_mx_linear_codes(far, M, 64, far, 64, null, y, L(ldy), 0, r, L(ldr), st) if codes else lib.mq_mx_linear(
        far, M, 64, L(64), far, 64, null, y, L(ldy), 0, r, L(ldr), far, C.c_size_t(1 << 20), st))
    for codes in (0, 1):
        for M in (4, 40, 200):
            assert lin(at(64), 64, M=M, codes=codes) == -1 and lin(at(1), 64, M=M, codes=codes) == -1 and lin(p, 128, M=M, codes=codes) == -1
            assert lin(at(63), 128, ldy=128, M=M, codes=codes) == -1
    ln = lambda y, ldy: lib.mq_layer_norm(p, 4, 64, L(64), null, null, 2, f(1e-5), y, L(ldy), 0, null, null, st)
    assert ln(at(64), 64) == -1 and ln(at(1), 64) == -1 and ln(p, 128) == -1 and ln(at(-64), 64) == -1
    lg = lambda dx=far, lddx=64, dy=at(4096), x=at(8192), r=null: lib.mq_layer_norm_grad(
        dy, L(64), x, L(64), 4, 64, null, 2, p, p, r, L(64), dx, L(lddx), 0, p, p, p, C.c_size_t(1 << 20), st)
    assert lg(dx=at(4096 + 64)) == -1 and lg(dx=at(8192 - 64)) == -1 and lg(dx=at(100), r=at(99)) == -1 and lg(dx=at(4096), lddx=65) == -1


def test_values_are_their_own():
    """Quantised values quantise to themselves: a block's largest, 4 to 8 units before, is 4 or 6 units after, and so has the same scale."""
    rng = np.random.default_rng(7)
    for std in (1.0, 1e-3, 1e30, 2.0 ** -126, 2.0 ** -130):
        x = rng.normal(size=(40, 96)) * std
        x[rng.random(x.shape) < 0.05] *= 9.0
        x[3], x[4, 32:64], x[5, :32] = 0.0, std * 7.9, std * 6.0
        v = omx.values(x)
        assert np.abs(v).max() > 0 and np.array_equal(omx.values(v), v)
        assert np.array_equal(omx.scale_bytes(v), omx.scale_bytes(x))
