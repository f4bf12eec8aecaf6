"""The layer operations (affine layer with its epilogue, dropout, group norm) against their definitions in 64 bits.

Tolerances are bounds worked out from the operations' arithmetic, element by element: u = half a step of the storage type
relative to the value (bf16 2^-8, fp32 2^-24), sums of K
terms in fp32 that may truncate (2^-23 of the sum of magnitudes per addition), activations whose exponential is good to
2^-20 at the arguments used, slopes |act'| <= 1.13 and |act''| <= 0.8.
"""
import math
import time

import numpy as np
import pytest

import helpers
from oracle import philox
from paper_2301_08895_b200 import abs as gpu

pytestmark = pytest.mark.gpu

ACTS = [gpu.ACT_NONE, gpu.ACT_RELU, gpu.ACT_GELU, gpu.ACT_SILU]
E20, E23 = 2.0 ** -20, 2.0 ** -23


def _torch():
    import torch
    return torch


def dt(bf16):
    torch = _torch()
    return torch.bfloat16 if bf16 else torch.float32


def half_step(bf16):
    return _torch().finfo(dt(bf16)).eps / 2


def act64(z, act):
    torch = _torch()
    if act == gpu.ACT_RELU:
        return z.clamp(min=0)
    if act == gpu.ACT_GELU:
        return z * 0.5 * torch.special.erfc(-z / math.sqrt(2))
    if act == gpu.ACT_SILU:
        return z * torch.special.expit(z)
    return z


def slope64(z, act):
    torch = _torch()
    if act == gpu.ACT_RELU:
        return (z > 0).double()
    if act == gpu.ACT_GELU:
        return 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == gpu.ACT_SILU:
        s = torch.special.expit(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def smooth(act):
    return act in (gpu.ACT_GELU, gpu.ACT_SILU)


class Held:
    """A matrix (or maps) inside a larger buffer: row pitch, offset from an aligned start; what surrounds it is NaN and has to stay."""

    def __init__(self, rows, cols, dtype, pad=0, offset=0, values=None):
        torch = _torch()
        self.buf = torch.full((offset + max(rows, 1) * (cols + pad) + 16,), float("nan"), dtype=dtype, device="cuda")
        self.t = self.buf[offset:offset + max(rows, 1) * (cols + pad)].view(max(rows, 1), cols + pad)[:rows, :cols]
        if values is not None:
            self.t.copy_(values)
        self.rows, self.cols, self.pad, self.offset = rows, cols, pad, offset

    def surroundings_untouched(self):
        torch = _torch()
        mask = torch.ones_like(self.buf, dtype=torch.bool)
        mask[self.offset:self.offset + max(self.rows, 1) * (self.cols + self.pad)].view(max(self.rows, 1), -1)[:self.rows, :self.cols] = False
        return bool(torch.isnan(self.buf[mask]).all())


def randn(g, *shape, scale=1.0, dtype=None):
    torch = _torch()
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype or torch.float32)


def gen(seed):
    return _torch().Generator(device="cuda").manual_seed(seed)


def within(got, want, tol):
    torch = _torch()
    got, bad = got.double(), None
    err = (got - want).abs()
    ok = bool((err <= tol).all())
    if not ok:
        i = int((err - tol).argmax())
        bad = (i, float(got.flatten()[i]), float(want.flatten()[i]), float(tol.flatten()[i] if torch.is_tensor(tol) else tol))
    assert ok, "at %d: got %.9g, want %.9g, tolerance %.3g" % bad


# ------------------------------------------------------------------------------------------------ affine layer

def linear_case(M, K, N, bf16, act, residual, pre, bias=True, pad=0, offset=0, seed=0, in_place=False):
    torch = _torch()
    g = gen(seed)
    d, u = dt(bf16), half_step(bf16)
    x = Held(M, K, d, pad, offset, randn(g, M, K, dtype=d))
    w = Held(K, N, d, pad, offset, randn(g, K, N, scale=math.sqrt(2.0 / K), dtype=d))
    b = randn(g, N, scale=0.3, dtype=d) if bias else None
    r = Held(M, N, d, pad, offset, randn(g, M, N, dtype=d)) if residual else None
    r64 = r.t.double().clone() if residual else 0.0
    y = r if in_place else Held(M, N, d, pad, offset)
    z = Held(M, N, d, pad, offset) if pre else None
    gpu.linear(x.t, w.t, b, r.t if residual else None, y.t, act, pre=z.t if pre else None)
    torch.cuda.synchronize()
    x64, w64 = x.t.double(), w.t.double()
    b64 = b.double() if bias else torch.zeros(N, dtype=torch.float64, device="cuda")
    z64 = x64 @ w64 + b64
    tz = (K + 4) * E23 * (x64.abs() @ w64.abs() + b64.abs())
    a64 = act64(z64, act)
    y64 = a64 + r64
    ty = u * y64.abs() + 1.2 * tz + (E20 * (1 + z64.abs()) if smooth(act) else 0.0) + E23 * (a64.abs() + (r64.abs() if residual else 0.0))
    within(y.t, y64, ty)
    assert y.surroundings_untouched()
    if pre:
        within(z.t, z64, u * z64.abs() + 1.2 * tz)
        assert z.surroundings_untouched()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("M,K,N", [
    (1, 1, 1), (1, 784, 256), (1, 785, 10), (2, 7, 3), (5, 64, 1000), (8, 256, 64), (9, 256, 64), (16, 1000, 40), (17, 33, 129),
    (127, 64, 64), (128, 128, 256), (129, 65, 257), (200, 8, 8), (300, 300, 123), (384, 512, 512), (513, 96, 10), (1000, 784, 256),
    (33, 4096, 96), (40, 4099, 72)])
def test_linear_sizes(M, K, N, bf16):
    linear_case(M, K, N, bf16, gpu.ACT_RELU, False, False, seed=M + K + N)
    linear_case(M, K, N, bf16, gpu.ACT_SILU, True, True, seed=M + K + N + 1)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("M,K,N", [
    (2, 1030, 88), (3, 1030, 88), (4, 1030, 88), (5, 1024, 88), (8, 2500, 24), (9, 2500, 24), (1, 4096, 4096), (2, 100, 6000),    # a few rows
    (255, 256, 10), (256, 256, 10), (257, 8, 16), (400, 40, 1), (1000, 256, 16), (1000, 264, 16), (300, 512, 9), (300, 520, 9), (4000, 64, 17)])
def test_linear_around_the_borders_of_its_kernels(M, K, N, bf16):
    linear_case(M, K, N, bf16, gpu.ACT_GELU, True, True, seed=M + K)
    linear_case(M, K, N, bf16, gpu.ACT_NONE, False, False, bias=False, pad=8, offset=8, seed=M + K)
    linear_case(M, K, N, bf16, gpu.ACT_RELU, True, False, pad=1, offset=0, seed=M + K)


@pytest.mark.parametrize("M,K,N", [(130, 5000, 136), (1, 3000, 200), (520, 100, 1032), (1100, 700, 520), (40, 33, 4100)])
def test_linear_fp32_shared_sums(M, K, N):
    """Sums shared by two to eight CTAs of a cluster, both tile sizes, ragged ends."""
    linear_case(M, K, N, False, gpu.ACT_SILU, True, True, seed=K)
    grad_case(M, K, N, False, gpu.ACT_SILU, seed=K)
    grad_case(M, K, N, False, gpu.ACT_NONE, seed=K, want=(False, True, False))
    grad_case(M, K, N, False, gpu.ACT_NONE, seed=K, want=(True, False, True))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("act", ACTS)
def test_activations_far_from_zero(act, bf16):
    """z of both signs up to 1e30 through the forward and the backward pass, in the layer and in group norm: values and slopes of the definitions
    (SiLU below z = -41 is zero to 4e-17, its slope too)."""
    torch = _torch()
    d, u = dt(bf16), half_step(bf16)
    z = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 0.5, -0.5, 3.0, -3.0, 9.0, -9.0, 20.0, -20.0, 41.0, -41.0, 60.0, -60.0, 88.0, -88.0, 200.0, -200.0,
                      1e4, -1e4, 1e15, -1e15, 1e30, -1e30], device="cuda").to(d)
    n = z.numel()
    want = act64(z.double(), act)
    slope = torch.nan_to_num(slope64(z.double(), act), nan=0.0)
    tol = u * want.abs() + 1e-6 * torch.clamp(z.double().abs(), max=10.0) + 1e-37
    for rows in (1, 40, 300):
        y = torch.empty(rows, n, device="cuda", dtype=d)
        gpu.linear(torch.zeros(rows, 16, device="cuda", dtype=d), torch.zeros(16, n, device="cuda", dtype=d), z, None, y, act)
        within(y, want.expand(rows, n), tol)
        dy, x = torch.ones(rows, n, device="cuda", dtype=d), torch.zeros(rows, 16, device="cuda", dtype=d)
        x[0, 0] = 1.0
        db, dw = torch.empty(n, device="cuda", dtype=d), torch.empty(16, n, device="cuda", dtype=d)
        gpu.linear_grad(dy, x, torch.zeros(16, n, device="cuda", dtype=d), z.expand(rows, n).contiguous(), None, dw, db, act)
        within(dw[0], slope, u * slope.abs() + 2e-6)
        within(db, rows * slope, 2 * u * rows * slope.abs() + 2e-6 * rows)
    # group norm of constant maps: u = b
    for P in (4, 300000):
        b = torch.nn.functional.pad(z, (0, 32 - n))
        y = torch.empty(1, P, 32, device="cuda", dtype=d)
        x = torch.full((1, P, 32), 2.0, device="cuda", dtype=d)
        mean, rstd = torch.empty(1, 2, device="cuda"), torch.empty(1, 2, device="cuda")
        gpu.group_norm(x, 2, None, b, y, mean, rstd, 1.0, act)
        within(y[0, 0, :n], want, tol)
        assert bool((y[0] == y[0, 0]).all())
        dy = torch.full((1, P, 32), 1.0 / P, device="cuda", dtype=d)
        db = torch.empty(32, device="cuda", dtype=d)
        gpu.group_norm_grad(dy, x, 2, None, b, mean, rstd, None, None, db, act)
        total = float(dy.double()[0, :, 0].sum()) * slope
        within(db[:n], total, 2 * u * total.abs() + 4e-6)


@pytest.mark.parametrize("M,K,N", [(2300, 1000, 4096), (4224, 328, 2568), (9000, 512, 1025)])
def test_linear_of_many_tiles(M, K, N):
    linear_case(M, K, N, True, gpu.ACT_GELU, True, True, seed=M)
    grad_case(M, K, N, True, gpu.ACT_GELU, seed=M)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("residual,pre,bias", [(False, False, False), (True, False, True), (False, True, False), (True, True, True)])
def test_linear_epilogues(act, residual, pre, bias, bf16):
    for M in (3, 150):
        linear_case(M, 96, 136, bf16, act, residual, pre, bias, seed=act)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("pad,offset", [(8, 0), (8, 8), (1, 0), (0, 1), (3, 5), (2, 2), (4, 4)])
def test_linear_pitches_and_alignment(pad, offset, bf16):
    for M, K, N in ((1, 128, 64), (6, 120, 72), (150, 128, 256), (140, 72, 40)):
        linear_case(M, K, N, bf16, gpu.ACT_GELU, True, True, pad=pad, offset=offset, seed=pad + 10 * offset)


@pytest.mark.parametrize("bf16", [False, True])
def test_linear_adds_to_the_residual_in_place(bf16):
    for M, N in ((1, 64), (130, 128), (130, 65)):
        linear_case(M, 64, N, bf16, gpu.ACT_SILU, True, True, seed=5, in_place=True)


@pytest.mark.parametrize("bf16", [False, True])
def test_linear_infinities_stay_in_their_rows_and_columns(bf16):
    """An infinite activation reaches its row only, an infinite weight its column only, a NaN bias its column only."""
    torch = _torch()
    d = dt(bf16)
    for M in (4, 140):
        x = torch.ones(M, 72, device="cuda", dtype=d)
        w = torch.ones(72, 130, device="cuda", dtype=d)
        b = torch.zeros(130, device="cuda", dtype=d)
        x[2, 71], w[0, 129], b[5] = float("inf"), float("inf"), float("nan")
        y = torch.zeros(M, 130, device="cuda", dtype=d)
        gpu.linear(x, w, b, None, y)
        want = torch.full((M, 130), 72.0, device="cuda")
        want[2, :], want[:, 129] = float("inf"), float("inf")
        want[:, 5] = float("nan")
        assert torch.equal(torch.nan_to_num(y.float(), nan=-1.0), torch.nan_to_num(want, nan=-1.0))


def grad_case(M, K, N, bf16, act, pad=0, offset=0, seed=0, want=(True, True, True), differences=False):
    torch = _torch()
    g = gen(seed)
    d, u = dt(bf16), half_step(bf16)
    x = Held(M, K, d, pad, offset, randn(g, M, K, dtype=d))
    w = Held(K, N, d, pad, offset, randn(g, K, N, scale=math.sqrt(2.0 / K), dtype=d))
    dy = Held(M, N, d, pad, offset, randn(g, M, N, dtype=d))
    b = randn(g, N, scale=0.3, dtype=d)
    z = None
    if act != gpu.ACT_NONE:
        z = Held(M, N, d, pad, offset, (x.t.double() @ w.t.double() + b.double()).to(d))
    dx = Held(M, K, d, pad, offset) if want[0] else None
    dw = Held(K, N, d, pad, offset) if want[1] else None
    db = torch.full((N,), float("nan"), device="cuda", dtype=d) if want[2] else None
    gpu.linear_grad(dy.t, x.t, w.t, z.t if z else None, dx.t if dx else None, dw.t if dw else None, db, act)
    torch.cuda.synchronize()
    x64, w64, dy64 = x.t.double(), w.t.double(), dy.t.double()
    dz = dy64 * slope64(z.t.double(), act) if z else dy64
    tdz = (E20 * (1 + z.t.double().abs()) * dy64.abs() if smooth(act) else 0.0 * dz) + E23 * dz.abs()
    tb = tdz + (M + 4) * E23 * dz.abs()
    if bf16 and z:
        tdz = tdz + u * dz.abs()                        # dz enters the products rounded to storage
    if dx:
        want_dx = dz @ w64.T
        within(dx.t, want_dx, u * want_dx.abs() + 1.01 * ((tdz + (N + 4) * E23 * dz.abs()) @ w64.abs().T))
        assert dx.surroundings_untouched()
    if dw:
        want_dw = x64.T @ dz
        within(dw.t, want_dw, u * want_dw.abs() + 1.01 * (x64.abs().T @ (tdz + (M + 4) * E23 * dz.abs())))
        assert dw.surroundings_untouched()
    if db is not None:
        want_db = dz.sum(0)
        within(db, want_db, u * want_db.abs() + 1.01 * tb.sum(0))
    if differences:
        # directional derivative of L = sum dy act(x w + b) by central differences of the definition in 64 bits
        # (step 1e-6: truncation 1e-12, rounding 1e-10 of L's terms); the gradients' own errors as above, summed.  Where the
        # saved pre-activation is rounded (bf16) the gradient is the one at the rounded value: fp32 only.
        assert not bf16
        b64, h = b.double(), 1e-6
        loss = lambda xx, ww, bb: float((dy64 * act64(xx @ ww + bb, act)).sum())           # noqa: E731
        for got, at, tol in ((dx.t, 0, (tdz + (N + 4) * E23 * dz.abs()) @ w64.abs().T), (dw.t, 1, x64.abs().T @ (tdz + (M + 4) * E23 * dz.abs())),
                             (db, 2, tb.sum(0))):
            v = randn(g, *got.shape).double()
            args = [x64, w64, b64]
            lo, hi = list(args), list(args)
            lo[at], hi[at] = args[at] - h * v, args[at] + h * v
            num = (loss(*hi) - loss(*lo)) / (2 * h)
            # pre is stored in fp32: the slope is taken up to 2^-24 |z| away, |act''| <= 0.8
            shift = 0.8 * 2.0 ** -24 * (dy64 * z.t.double()).abs()
            extra = {0: lambda: shift @ w64.abs().T, 1: lambda: x64.abs().T @ shift, 2: lambda: shift.sum(0)}[at]()
            slack = float(((2 * tol + u * got.double().abs() + extra) * v.abs()).sum()) + 1e-8 * float((dy64 * z.t.double()).abs().sum())
            assert abs(float((got.double() * v).sum()) - num) <= slack


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("M,K,N", [
    (1, 1, 1), (1, 784, 256), (2, 7, 3), (7, 64, 10), (8, 256, 64), (31, 300, 123), (64, 64, 64), (129, 65, 257), (256, 128, 256),
    (300, 400, 120), (513, 96, 10), (1000, 784, 256), (2000, 40, 24), (4100, 264, 8)])
def test_linear_grad_sizes(M, K, N, bf16):
    grad_case(M, K, N, bf16, gpu.ACT_NONE, seed=M)
    grad_case(M, K, N, bf16, gpu.ACT_SILU, seed=M + 1)


@pytest.mark.parametrize("pad,offset", [(0, 0), (1, 0), (8, 8)])
@pytest.mark.parametrize("M,K,N", [(3001, 20, 17), (9001, 37, 29), (20011, 130, 70), (70, 65, 12001)])
def test_linear_fp32_long_sums(M, K, N, pad, offset):
    """Long sums of few tiles: parts through scratch, with and without clusters in each."""
    linear_case(70, M, N % 500, False, gpu.ACT_GELU, True, True, pad=pad, offset=offset, seed=M)
    linear_case(70, M, K, False, gpu.ACT_NONE, False, False, pad=pad, offset=offset, seed=M, bias=False)
    grad_case(M, K, N, False, gpu.ACT_SILU, pad=pad, offset=offset, seed=M)
    grad_case(M, K, N, False, gpu.ACT_NONE, pad=pad, offset=offset, seed=M, want=(False, True, True))
    grad_case(M, K, N, False, gpu.ACT_RELU, pad=pad, offset=offset, seed=M, want=(True, False, False))


def takes_pieces(M, K, N, grad=False):
    """Whether the call's scratch has room for three bf16 pieces of each of its matrices."""
    pieces = 6 * (M * K + K * N + (M * N if grad else 0))
    return gpu.linear_scratch_bytes(M, K, N, gpu.ACT_NONE, gpu.FP32, grad) > pieces


@pytest.mark.parametrize("pad,offset", [(0, 0), (1, 0), (3, 5), (8, 8)])
@pytest.mark.parametrize("M,K,N", [(1037, 785, 501), (512, 1024, 1024), (8192, 784, 256), (1100, 701, 520), (2500, 2500, 641), (300, 10000, 300)])
def test_linear_fp32_in_pieces(M, K, N, pad, offset):
    """Six products of bf16 pieces: what they leave out is below 2^-23 of |x| |w|, one more term in the bound's K + 4; the tensor cores add 16
    products at a time, K / 16 such additions of the results' size and 5 K / 16 of at most 2^-7 of it."""
    assert takes_pieces(M, K, N)
    linear_case(M, K, N, False, gpu.ACT_SILU, True, True, pad=pad, offset=offset, seed=K)
    linear_case(M, K, N, False, gpu.ACT_NONE, False, False, bias=False, pad=pad, offset=offset, seed=K)
    linear_case(M, K, N, False, gpu.ACT_RELU, True, False, pad=pad, offset=offset, seed=K, in_place=True)


@pytest.mark.parametrize("pad,offset", [(0, 0), (1, 0), (8, 8)])
@pytest.mark.parametrize("M,K,N", [(2048, 1024, 1024), (1037, 785, 501), (20000, 400, 120), (777, 2049, 1300)])
def test_linear_grad_fp32_in_pieces(M, K, N, pad, offset):
    assert takes_pieces(M, K, N, True)
    grad_case(M, K, N, False, gpu.ACT_GELU, pad=pad, offset=offset, seed=M)
    for want in ((True, False, False), (False, True, False), (False, False, True), (True, False, True), (False, True, True)):
        grad_case(M, K, N, False, gpu.ACT_NONE, pad=pad, offset=offset, seed=M, want=want)


def test_linear_fp32_in_pieces_of_single_products():
    """Sums of one product each, in the three layouts: what the three pairs left out make up (2^-23 of it) and a rounding."""
    torch = _torch()
    M, K, N = 520, 1024, 1030
    assert takes_pieces(M, K, N) and takes_pieces(M, K, N, True)
    dev = lambda a: torch.from_numpy(a).cuda()                          # noqa: E731
    x, w = map(dev, helpers.one_product_operands(M, K, N, 1))
    y = torch.empty(M, N, device="cuda")
    gpu.linear(x, w, None, None, y)
    want = x.double() @ w.double()
    within(y, want, 2.0 ** -22 * want.abs())
    dy, wt = map(dev, helpers.one_product_operands(M, N, K, 2))         # dx = dy w^T
    dx = torch.empty(M, K, device="cuda")
    gpu.linear_grad(dy, x, wt.t().contiguous(), None, dx, None, None)
    want = dy.double() @ wt.double()
    within(dx, want, 2.0 ** -22 * want.abs())
    xt, dy = map(dev, helpers.one_product_operands(K, M, N, 3))         # dw = x^T dy
    dw = torch.empty(K, N, device="cuda")
    gpu.linear_grad(dy, xt.t().contiguous(), w, None, None, dw, None)
    want = xt.double() @ dy.double()
    within(dw, want, 2.0 ** -22 * want.abs())


@pytest.mark.parametrize("one_sign", [False, True])
@pytest.mark.parametrize("layout", ["y", "dx", "dw"])
@pytest.mark.parametrize("K", [785, 4096, 20000])
def test_linear_fp32_in_pieces_does_not_drift(K, layout, one_sign):
    """The tensor cores' accumulator truncates: a sum of 16 products and itself loses up to 2^-23 of itself, half of it on average.  It takes 256
    terms, 16 such additions, before the parts are added to nearest: of a part whose terms have one sign, that is at most 8 2^-23, on average half of it;
    the K / 256 additions behind add at most K / 512 2^-24.  Terms of both signs: an addition loses up to 2^-23, on average half, of a partial sum of
    up to 16 terms' size, two thirds of that on average: 16 * 10.7 * 2^-24 for each of K / 256 independent parts, 10.7 sqrt(K) 2^-24 of a term."""
    torch = _torch()
    M, N = 512, 640
    g = gen(K)
    draw = (lambda *s: torch.rand(*s, generator=g, device="cuda") + 0.5) if one_sign else (lambda *s: torch.randn(*s, generator=g, device="cuda"))
    a, b = draw(M, K), draw(K, N)
    got, want = torch.empty(M, N, device="cuda"), a.double() @ b.double()
    if layout == "y":
        assert takes_pieces(M, K, N)
        gpu.linear(a, b, None, None, got)
    elif layout == "dx":
        assert takes_pieces(M, N, K, True)
        gpu.linear_grad(a, torch.empty(M, N, device="cuda"), b.t().contiguous(), None, got, None, None)
    else:
        assert takes_pieces(K, M, N, True)
        gpu.linear_grad(b, a.t().contiguous(), torch.empty(M, N, device="cuda"), None, None, got, None)
    err = got.double() - want
    if one_sign:
        assert abs(float((err / want).mean())) <= 2.0 ** -21
        within(got, want, (2.0 ** -20 + K / 512 * 2.0 ** -24 + 2.0 ** -22) * want)
    else:
        assert float(err.square().mean().sqrt()) <= 12 * math.sqrt(K) * 2.0 ** -24


def test_linear_grad_bf16_over_many_rows():
    """134 million rows of one sign: the sum in bf16 is that of the terms, rounded (2^-8), not that of a truncating accumulator (off by 1.4e-2).  64
    stretches of 4096 terms each lose at most 2^-13 of themselves on average, the sums behind are to nearest."""
    torch = _torch()
    rows, n = 1 << 27, 8
    g = gen(3)
    x, dy = ((torch.rand(rows, n, generator=g, device="cuda") * 0.5 + 0.5).bfloat16() for _ in range(2))
    dw, db = torch.empty(n, n, device="cuda", dtype=torch.bfloat16), torch.empty(n, device="cuda", dtype=torch.bfloat16)
    gpu.linear_grad(dy, x, torch.zeros(n, n, device="cuda", dtype=torch.bfloat16), None, None, dw, db)
    want, total = torch.zeros(n, n, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
    for i in range(0, rows, 1 << 22):
        part = dy[i:i + (1 << 22)].double()
        want += x[i:i + (1 << 22)].double().T @ part
        total += part.sum(0)
    within(dw, want, (2.0 ** -8 + 2.0 ** -12) * want)
    within(db, total, (2.0 ** -8 + 2.0 ** -12) * total)


@pytest.mark.parametrize("K", [65536, 65600, 131072])
def test_linear_bf16_long_sums_do_not_drift(K):
    """Terms of one sign, tiles enough that no sum is split: the mean error, in which the roundings to bf16 cancel, stays below an eighth of one."""
    torch = _torch()
    M, N = 2500, 2560
    g = gen(K)
    x = torch.empty(M, K, device="cuda", dtype=torch.bfloat16).uniform_(0.5, 1.5, generator=g)
    w = torch.empty(K, N, device="cuda", dtype=torch.bfloat16).uniform_(0.5, 1.5, generator=g)
    b, r = randn(g, N, scale=1e4, dtype=torch.bfloat16), randn(g, M, N, scale=1e4, dtype=torch.bfloat16)
    y, z = torch.empty(M, N, device="cuda", dtype=torch.bfloat16), torch.empty(M, N, device="cuda", dtype=torch.bfloat16)
    gpu.linear(x, w, b, r, y, pre=z)
    want = torch.zeros(M, N, dtype=torch.float64, device="cuda")
    for k in range(0, K, 16384):
        want += x[:, k:k + 16384].double() @ w[k:k + 16384].double()
    total = want.clone()                                 # (of K positive terms; bias and residual can turn the results' sign)
    for got, more in ((z, b.double()), (y, r.double())):
        want += more
        assert abs(float((got.double() - want).mean())) <= 2.0 ** -11 * float(total.mean())
        within(got, want, 2.0 ** -8 * want.abs() + 2.0 ** -10 * total)


def test_linear_fp32_of_what_pieces_cannot_hold():
    """Infinities, NaN, the largest and the smallest numbers: the results of fp32 all the same, in the forward and the backward products."""
    torch = _torch()
    M, K, N = 520, 1024, 1030
    assert takes_pieces(M, K, N) and takes_pieces(M, K, N, True)
    top = torch.finfo(torch.float32).max
    for bad in (float("inf"), -float("inf"), float("nan"), top, -top, 2.0 ** -112, 1e-42, 0.0):
        for scale in (1.0, 2.0 ** -100):
            g = gen(7)
            x, w, r = randn(g, M, K), randn(g, K, N, scale=2.0 ** -20), randn(g, M, N)
            x = x * scale
            x[17, 33] = bad
            w[40, 21] = 0.0
            y = r.clone()
            gpu.linear(x, w, None, y, y)
            x64, w64, r64 = x.double(), w.double(), r.double()
            want = x64 @ w64 + r64
            tol = 1.2 * (K + 4) * E23 * (x64.abs() @ w64.abs()) + 2 * E23 * (r64.abs() + want.abs()) + 2.0 ** -126
            inf = torch.isinf(want)
            assert torch.equal(torch.isnan(y), torch.isnan(want)) and torch.equal(y[inf].double(), want[inf])
            ok = torch.isfinite(want)
            within(y[ok], want[ok], tol[ok])
    for value in (2.0 ** -112, 2.0 ** -120):             # all of a matrix below what pieces hold
        g = gen(8)
        x, w, dy = randn(g, M, K) * value, randn(g, K, N) * 2.0 ** 90, randn(g, M, N) * value
        y, dx, dw = torch.empty(M, N, device="cuda"), torch.empty_like(x), torch.empty_like(w)
        gpu.linear(x, w, None, None, y)
        within(y, x.double() @ w.double(), 1.2 * (K + 4) * E23 * (x.double().abs() @ w.double().abs()))
        gpu.linear_grad(dy, randn(g, M, K), w, None, dx, None, None)
        within(dx, dy.double() @ w.double().T, 1.2 * (N + 4) * E23 * (dy.double().abs() @ w.double().abs().T))
        xx = randn(g, M, K) * 2.0 ** 90
        gpu.linear_grad(dy, xx, w, None, None, dw, None)
        within(dw, xx.double().T @ dy.double(), 1.2 * (M + 4) * E23 * (xx.double().abs().T @ dy.double().abs()))


def test_linear_fp32_in_pieces_of_tiny_elements():
    """One element of a saturated unit's size, down to the smallest float, sends nothing to the slow kernel: results that it cannot reach keep their bits.
    Whole matrices of that size have fp32's results."""
    torch = _torch()
    M, K, N = 520, 1024, 1030
    assert takes_pieces(M, K, N) and takes_pieces(M, K, N, True)
    g = gen(12)
    x, w, dy = randn(g, M, K), randn(g, K, N), randn(g, M, N)

    def results():
        y, dx, dw = torch.empty(M, N, device="cuda"), torch.empty_like(x), torch.empty_like(w)
        gpu.linear(x, w, None, None, y)
        gpu.linear_grad(dy, x, w, None, dx, dw, None)
        return y, dx, dw
    x[17, 33] = dy[5, 99] = w[40, 21] = 0.0
    y0, dx0, dw0 = results()
    for tiny in (2.0 ** -111, 2.0 ** -126, 1e-42, 2.0 ** -149):
        x[17, 33], dy[5, 99], w[40, 21] = tiny, -tiny, tiny
        y, dx, dw = results()
        assert torch.equal(y, y0) and torch.equal(dx, dx0) and torch.equal(dw, dw0)
    lowest = 2.0 ** -149
    for down, up in ((2.0 ** -112, 2.0 ** 30), (2.0 ** -128, 2.0 ** 12), (2.0 ** -140, 1.0), (2.0 ** -60, 2.0 ** -75)):
        a, b, c = randn(g, M, K) * down, randn(g, K, N) * up, randn(g, M, N) * down
        y, dx, dw = torch.empty(M, N, device="cuda"), torch.empty_like(a), torch.empty_like(b)
        gpu.linear(a, b, None, None, y)
        gpu.linear_grad(c, b[:M, :K].contiguous(), b, None, dx, dw, None)
        xx = b[:M, :K].double()
        tol = lambda p, q, n: 1.2 * (n + 4) * E23 * (p.abs() @ q.abs()) + lowest           # noqa: E731
        within(y, a.double() @ b.double(), tol(a.double(), b.double(), K))
        within(dx, c.double() @ b.double().T, tol(c.double(), b.double().T, N))
        within(dw, xx.T @ c.double(), tol(xx.T, c.double(), M))


@pytest.mark.parametrize("size", [41.9, 42.5, 58.0])
def test_linear_fp32_in_pieces_of_large_elements(size):
    """Terms of one sign up to where scaled sums would overflow, and beyond: fp32's sums, which do not."""
    torch = _torch()
    M, K, N = 520, 1024, 1030
    assert takes_pieces(M, K, N) and takes_pieces(M, K, N, True)
    x, w, dy = (torch.full(s, 2.0 ** size, device="cuda") for s in ((M, K), (K, N), (M, N)))
    y, dx, dw = torch.empty(M, N, device="cuda"), torch.empty(M, K, device="cuda"), torch.empty(K, N, device="cuda")
    gpu.linear(x, w, None, None, y)
    gpu.linear_grad(dy, x, w, None, dx, dw, None)
    square = float(x[0, 0]) ** 2
    for got, n in ((y, K), (dx, N), (dw, M)):
        want = torch.full_like(got, n * square, dtype=torch.float64)
        within(got, want, (n + 4) * 2.0 ** -24 * want)


def test_linear_fp32_in_pieces_captured_and_on_another_stream():
    """The flags of a step are its own: a replay with an infinity in x, and one without it again."""
    torch = _torch()
    g = gen(11)
    M, K, N = 600, 1024, 1024
    x, w, dy = randn(g, M, K), randn(g, K, N), randn(g, M, N)
    y, dx, dw, db = torch.empty(M, N, device="cuda"), torch.empty_like(x), torch.empty_like(w), torch.empty(N, device="cuda")
    size = max(gpu.linear_scratch_bytes(M, K, N, dtype=gpu.FP32), gpu.linear_scratch_bytes(M, K, N, dtype=gpu.FP32, grad=True))
    scratch = torch.empty(size, dtype=torch.uint8, device="cuda")
    outs = (y, dx, dw, db)

    def step():
        gpu.linear(x, w, None, None, y, scratch=scratch)
        gpu.linear_grad(dy, x, w, None, dx, dw, db, scratch=scratch)
    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for t in outs:
            t.fill_(float("nan"))
        step()
    side.synchronize()
    assert all(torch.equal(t, v) for t, v in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    keep = float(x[5, 6])
    for value in (keep, float("inf"), keep):
        x[5, 6] = value
        graph.replay()
        torch.cuda.synchronize()
        if value == keep:
            assert all(torch.equal(t, v) for t, v in zip(outs, want))
        else:
            assert not torch.isfinite(y[5]).any() and bool(torch.isfinite(y[6:]).all()) and bool(torch.isfinite(y[:5]).all())
            assert not torch.isfinite(dw[6]).any() and bool(torch.isfinite(dw[7:]).all()) and bool(torch.isfinite(dx).all())


def test_linear_fp32_parts_in_a_captured_step():
    """The scratch of a call serves the next one on its stream: forward, gradients and forward again in one graph, replayed, give the same bits."""
    torch = _torch()
    g = gen(5)
    x, w, dy = randn(g, 3001, 20), randn(g, 20, 17), randn(g, 3001, 17)
    a, b = randn(g, 70, 3001), randn(g, 3001, 17)
    y, dw, db, dx, again = torch.empty(70, 17, device="cuda"), torch.empty_like(w), torch.empty(17, device="cuda"), torch.empty_like(x), torch.empty(70, 17, device="cuda")
    size = max(gpu.linear_scratch_bytes(70, 3001, 17, dtype=gpu.FP32), gpu.linear_scratch_bytes(3001, 20, 17, dtype=gpu.FP32, grad=True))
    assert size > 0
    scratch = torch.empty(size, dtype=torch.uint8, device="cuda")

    def step():
        gpu.linear(a, b, None, None, y, scratch=scratch)
        gpu.linear_grad(dy, x, w, None, dx, dw, db, scratch=scratch)
        gpu.linear(a, b, None, None, again, scratch=scratch)
    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in (y, dw, db, dx, again)]
    assert torch.equal(y, again)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t in (y, dw, db, dx, again):
        t.fill_(float("nan"))
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for t, v in zip((y, dw, db, dx, again), want):
        assert torch.equal(t, v)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("want", [(True, False, False), (False, True, False), (False, False, True), (True, True, False)])
def test_linear_grad_of_chosen_operands(act, want, bf16):
    grad_case(150, 72, 136, bf16, act, want=want, seed=act)
    grad_case(150, 72, 136, bf16, act, want=want, pad=1, offset=3, seed=act)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("pad,offset", [(8, 0), (8, 8), (1, 0), (0, 1), (2, 2), (4, 4)])
def test_linear_grad_pitches_and_alignment(pad, offset, bf16):
    grad_case(140, 128, 72, bf16, gpu.ACT_GELU, pad=pad, offset=offset, seed=3)
    grad_case(6, 72, 128, bf16, gpu.ACT_NONE, pad=pad, offset=offset, seed=4)


@pytest.mark.parametrize("act", [gpu.ACT_GELU, gpu.ACT_SILU])
def test_linear_grad_against_differences(act):
    grad_case(37, 29, 23, False, act, seed=11, differences=True)


def test_linear_without_rows():
    torch = _torch()
    for bf16 in (False, True):
        d = dt(bf16)
        w = torch.ones(16, 8, device="cuda", dtype=d)
        gpu.linear(torch.empty(0, 16, device="cuda", dtype=d), w, None, None, torch.empty(0, 8, device="cuda", dtype=d))
        dw, db = Held(16, 8, d, 3, 1), torch.ones(8, device="cuda", dtype=d)
        gpu.linear_grad(torch.empty(0, 8, device="cuda", dtype=d), torch.empty(0, 16, device="cuda", dtype=d), w, None,
                        torch.empty(0, 16, device="cuda", dtype=d), dw.t, db)
        assert float(dw.t.abs().sum()) == 0.0 and float(db.abs().sum()) == 0.0 and dw.surroundings_untouched()


def test_linear_of_matrices_behind_32_bit_offsets():
    """Rows 2^30 elements apart: offsets of 2^31 elements and 2^32 bytes."""
    torch = _torch()
    pitch = 1 << 30
    for K, N in ((64, 64), (63, 10)):
        big = torch.empty(2 * pitch + 256, dtype=torch.bfloat16, device="cuda")
        x = big.as_strided((3, K), (pitch, 1))
        y = big.as_strided((3, N), (pitch, 1), 128)
        x.copy_(randn(gen(1), 3, K, dtype=torch.bfloat16))
        w = randn(gen(2), K, N, scale=0.1, dtype=torch.bfloat16)
        gpu.linear(x, w, None, None, y)
        want = x.double() @ w.double()
        within(y, want, 2.0 ** -8 * want.abs() + (K + 4) * E23 * (x.double().abs() @ w.double().abs()))
        del big, x, y
        torch.cuda.empty_cache()


# ------------------------------------------------------------------------------------------------ dropout

def keep_mask(rows, cols, p, seed, call):
    """The mask by the oracle's generator."""
    nblk = (cols + 7) // 8
    blk, row = np.meshgrid(np.arange(nblk), np.arange(rows))
    w = philox.philox4x32_10_blocks(blk.ravel(), row.ravel(), np.full(blk.size, 2), np.full(blk.size, call), philox.seed_key(seed))
    half = np.stack([w & 0xFFFF, w >> 16], axis=-1).reshape(rows, nblk * 8)[:, :cols]
    return half >= int(math.floor(p * 65536 + 0.5))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows,cols,p,pad,offset", [
    (1, 1, 0.5, 0, 0), (1, 7, 0.3, 0, 0), (3, 8, 0.5, 0, 0), (5, 9, 0.5, 7, 0), (128, 256, 0.1, 0, 0), (33, 1000, 0.9, 0, 0), (200, 10, 0.5, 0, 1),
    (64, 257, 0.25, 3, 5), (1, 100003, 0.5, 0, 0), (1000, 1, 0.5, 0, 0), (7, 512, 0.999999, 0, 0), (4, 64, 0.0, 8, 8), (4, 64, 1.0, 8, 0),
    (300, 2056, 1.0 / 65536, 0, 0), (2500, 1024, 0.2, 0, 0), (2600, 1003, 0.2, 0, 0), (2600, 1000, 0.2, 1, 1)])
def test_dropout(rows, cols, p, pad, offset, residual, bf16):
    torch = _torch()
    d, u = dt(bf16), half_step(bf16)
    g = gen(rows + cols)
    x = Held(rows, cols, d, pad, offset, randn(g, rows, cols, dtype=d) + 3.0)
    r = Held(rows, cols, d, pad, offset, randn(g, rows, cols, dtype=d)) if residual else None
    y = Held(rows, cols, d, pad, offset)
    seed, call = (0x123456789ABCDEF0 + rows) % 2 ** 64, 4000000000 + cols
    gpu.dropout(x.t, r.t if r else None, y.t, p, seed, call % 2 ** 32)
    keep = torch.from_numpy(keep_mask(rows, cols, p, seed, call % 2 ** 32)).cuda()
    T = int(math.floor(p * 65536 + 0.5))
    kept = torch.where(keep, x.t.double() * (65536.0 / (65536 - T) if T < 65536 else 0.0), torch.zeros((), dtype=torch.float64, device="cuda"))
    want = kept + (r.t.double() if r else 0.0)
    within(y.t, want, u * want.abs() + 2.0 ** -23 * kept.abs() + 2.0 ** -24 * want.abs())   # scale, product, sum; storage
    if not r:
        assert torch.equal(y.t != 0, keep & (x.t != 0))
    assert y.surroundings_untouched()


@pytest.mark.parametrize("bf16", [False, True])
def test_dropout_in_place_and_dropped_infinities(bf16):
    torch = _torch()
    d = dt(bf16)
    for cols in (64, 61):
        x = torch.ones(40, cols, device="cuda", dtype=d)
        keep = torch.from_numpy(keep_mask(40, cols, 0.5, 7, 1)).cuda()
        x[~keep] = float("nan")
        x[0][~keep[0]] = float("inf")
        gpu.dropout(x, None, x, 0.5, 7, 1)
        assert torch.equal(x, torch.where(keep, 2.0, 0.0).to(d))
        r = torch.full((40, cols), 3.0, device="cuda", dtype=d)
        gpu.dropout(x, r, r, 0.5, 7, 1)
        assert torch.equal(r, torch.where(keep, 7.0, 3.0).to(d))


def test_dropout_gradient_is_the_same_call():
    """L = sum c dropout(x): the derivative along v is sum dropout(c) v, exactly linear in x."""
    torch = _torch()
    g = gen(3)
    x, c, v = (randn(g, 50, 77).double() for _ in range(3))
    keep = torch.from_numpy(keep_mask(50, 77, 0.3, 9, 2)).cuda()
    s = 65536.0 / (65536 - 19661)
    dx = torch.empty(50, 77, device="cuda")
    gpu.dropout(c.float(), None, dx, 0.3, 9, 2)
    h = 1e-3
    loss = lambda t: float((c.float().double() * torch.where(keep, t * s, 0.0)).sum())     # noqa: E731
    num = (loss(x + h * v) - loss(x - h * v)) / (2 * h)
    assert abs(float((dx.double() * v).sum()) - num) <= 1e-6 * float((dx.double() * v).abs().sum())


def test_dropout_rate_and_calls():
    """Half of 4 M elements: the count lies within six standard deviations; calls and seeds give other masks."""
    torch = _torch()
    x = torch.ones(2048, 2048, device="cuda", dtype=torch.bfloat16)
    outs = []
    for seed, call in ((1, 0), (1, 1), (2, 0)):
        y = torch.empty_like(x)
        gpu.dropout(x, None, y, 0.5, seed, call)
        n = int((y != 0).sum())
        assert abs(n - 2 ** 21) <= 6 * 1024
        outs.append(y != 0)
    for a, b in ((0, 1), (0, 2), (1, 2)):
        assert abs(int((outs[a] == outs[b]).sum()) - 2 ** 21) <= 6 * 1024


def test_dropout_of_more_than_2_32_elements():
    torch = _torch()
    rows, cols, p, seed, call = 70000, 65528, 0.5, 11, 3
    x = torch.ones(rows, cols, device="cuda", dtype=torch.bfloat16)
    gpu.dropout(x, None, x, p, seed, call)
    blk = np.arange(cols // 8)
    for r in (0, 1, 65535, 65536, rows - 1):
        w = philox.philox4x32_10_blocks(blk, np.full(blk.size, r), np.full(blk.size, 2), np.full(blk.size, call), philox.seed_key(seed))
        half = np.stack([w & 0xFFFF, w >> 16], axis=-1).reshape(cols)
        assert np.array_equal((x[r] != 0).cpu().numpy(), half >= 32768)
    del x
    torch.cuda.empty_cache()


# ------------------------------------------------------------------------------------------------ group norm

def maps(N, P, C, dtype, pad_p=0, pad_s=0, offset=0, values=None):
    """Maps [N, P, C] with pitches C + pad_p and P (C + pad_p) + pad_s inside a buffer of NaN; (buffer, view, mask of what is not ours)."""
    torch = _torch()
    sp, ss = C + pad_p, P * (C + pad_p) + pad_s
    buf = torch.full((offset + N * ss + 16,), float("nan"), dtype=dtype, device="cuda")
    view = buf.as_strided((N, P, C), (ss, sp, 1), offset)
    if values is not None:
        view.copy_(values)
    outside = torch.ones_like(buf, dtype=torch.bool)
    outside.as_strided((N, P, C), (ss, sp, 1), offset).fill_(False)
    return buf, view, outside


def chain(n):
    """Longest run of additions in a sum of n terms: at most n / 64 per thread and 64 in the tree above them."""
    return 64 + n / 64


def norm_parts(x64, G, eps):
    N, P, C = x64.shape
    xg = x64.view(N, P, G, C // G)
    mean = xg.mean(dim=(1, 3))
    var = ((xg - mean[:, None, :, None]) ** 2).mean(dim=(1, 3))
    return xg, mean, var, 1 / (var + eps).sqrt()


def norm_case(N, P, C, G, bf16, act, affine=True, pad_p=0, pad_s=0, offset=0, seed=0, shift=0.5, eps=1e-5, stats=True, in_place=False):
    torch = _torch()
    g = gen(seed)
    d, u = dt(bf16), half_step(bf16)
    _, x, _ = maps(N, P, C, d, pad_p, pad_s, offset, (randn(g, N, P, C) + shift * randn(g, C)).to(d))
    x64 = x.double().clone()
    buf, y, outside = (None, x, None) if in_place else maps(N, P, C, d, pad_p, pad_s, offset)
    w = (1 + 0.2 * randn(g, C)).to(d) if affine else None
    b = randn(g, C, scale=0.3, dtype=d) if affine else None
    mean = torch.full((N, G), float("nan"), device="cuda") if stats else None
    rstd = torch.full((N, G), float("nan"), device="cuda") if stats else None
    gpu.group_norm(x, G, w, b, y, mean, rstd, eps, act)
    torch.cuda.synchronize()
    xg, m64, v64, r64 = norm_parts(x64, G, eps)
    n = P * (C // G)
    # mean: n additions in chains, a division; variance: deviations from the computed mean (its error enters squared)
    tm = (chain(n) + 4) * 2.0 ** -24 * xg.abs().mean(dim=(1, 3))
    tv = (chain(n) + 8) * 2.0 ** -23 * v64 + tm ** 2 + 2 * tm * 2.0 ** -23 * v64.sqrt()
    tr = r64 * (0.5 * tv / (v64 + eps) + 2.0 ** -22)
    if stats:
        within(mean, m64, tm)
        within(rstd, r64, tr)
    e = lambda t: t[:, None, :, None]                                     # noqa: E731
    xh = (xg - e(m64)) * e(r64)
    txh = e(tm) * e(r64) + (xg - e(m64)).abs() * e(tr) + 2.0 ** -22 * xh.abs()
    w64 = w.double().view(G, C // G) if affine else 1.0
    b64 = b.double().view(G, C // G) if affine else 0.0
    z = xh * w64 + b64
    tz = txh * (w64.abs() if affine else 1.0) + 2.0 ** -23 * (z.abs() + (b64.abs() if affine else 0.0))
    want = act64(z, act)
    tol = u * want.abs() + 1.2 * tz + (E20 * (1 + z.abs()) if smooth(act) else 0.0) + E23 * want.abs()
    within(y, want.view(N, P, C), tol.view(N, P, C))
    if not in_place:
        assert bool(torch.isnan(buf[outside]).all())


NORM_SIZES = [
    (1, 1, 1, 1), (2, 1, 6, 3), (3, 49, 7, 7), (5, 13, 64, 64), (4, 196, 6, 2), (20, 784, 6, 3), (3, 100, 16, 1), (2, 1024, 64, 8), (2, 255, 320, 32),
    (7, 81, 84, 7), (2, 4096, 32, 4), (1, 20000, 8, 2), (1, 9000, 96, 3), (3, 16, 1000, 10), (2, 5, 4099, 1), (2, 30, 8200, 2), (1, 70000, 20, 4),
    (64, 64, 128, 32), (2, 3000, 512, 4), (1, 300000, 16, 2), (3000, 2, 8, 2), (1, 500, 8208, 3), (50, 1000, 64, 4), (60, 1000, 120, 12), (40, 1100, 77, 7),
    (700, 300, 30, 3), (1300, 100, 40, 1), (5, 130, 4104, 2)]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("N,P,C,G", NORM_SIZES)
def test_group_norm_sizes(N, P, C, G, bf16):
    norm_case(N, P, C, G, bf16, gpu.ACT_SILU, seed=N + P + C)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("affine", [False, True])
def test_group_norm_epilogues(act, affine, bf16):
    norm_case(3, 144, 48, 6, bf16, act, affine, seed=act, stats=affine)
    norm_case(3, 50, 21, 3, bf16, act, affine, seed=act, in_place=True)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("pad_p,pad_s,offset", [(8, 0, 0), (0, 24, 8), (1, 0, 0), (0, 1, 0), (0, 0, 1), (3, 5, 7), (4, 4, 4)])
def test_group_norm_pitches_and_alignment(pad_p, pad_s, offset, bf16):
    for C, G in ((64, 8), (24, 8), (10, 5)):
        norm_case(3, 120, C, G, bf16, gpu.ACT_RELU, pad_p=pad_p, pad_s=pad_s, offset=offset, seed=offset)


@pytest.mark.parametrize("bf16", [False, True])
def test_group_norm_far_from_zero(bf16):
    """Means 300 standard deviations away: the variance is that of the deviations."""
    norm_case(2, 400, 32, 4, bf16, gpu.ACT_NONE, shift=300.0, seed=2)


@pytest.mark.parametrize("bf16", [False, True])
def test_group_norm_of_constant_groups(bf16):
    """No variance: y = act(b), rstd = 1 / sqrt(eps)."""
    torch = _torch()
    d = dt(bf16)
    x = torch.full((2, 9, 16), 3.0, device="cuda", dtype=d)
    b = torch.arange(16, device="cuda").to(d)
    y = torch.empty_like(x)
    mean, rstd = torch.empty(2, 4, device="cuda"), torch.empty(2, 4, device="cuda")
    gpu.group_norm(x, 4, None, b, y, mean, rstd, 1e-4)
    assert torch.equal(y, b.expand(2, 9, 16)) and torch.equal(mean, torch.full_like(mean, 3.0))
    within(rstd, torch.full_like(rstd, 100.0).double(), 100 * 2.0 ** -22)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("N,P,C,G", [(1, 300000, 16, 2), (700, 300, 30, 3), (2, 30, 8200, 2)])
def test_group_norm_in_place_of_large_maps(N, P, C, G, bf16):
    norm_case(N, P, C, G, bf16, gpu.ACT_SILU, seed=N, in_place=True)
    norm_grad_case(N, P, C, G, bf16, gpu.ACT_SILU, seed=N, in_place=True)


@pytest.mark.parametrize("P", [3, 40, 100000])
def test_group_norm_of_huge_and_tiny_values(P):
    """Constant maps of 1e30 have no variance (threads without rows must not bring 0 times infinity into it); values of 1e-30 vanish beside eps."""
    torch = _torch()
    for bf16 in (False, True):
        x = torch.full((2, P, 24), 1e30, device="cuda", dtype=dt(bf16))
        x[1] = 1e-30
        y = torch.empty_like(x)
        mean, rstd = torch.empty(2, 3, device="cuda"), torch.empty(2, 3, device="cuda")
        gpu.group_norm(x, 3, None, torch.full((24,), 0.5, device="cuda", dtype=dt(bf16)), y, mean, rstd, 1.0)
        # (the mean of 1e30 is off by roundings; what is left of x - mean over sqrt(eps) is of their size)
        assert bool(torch.isfinite(y).all()) and bool(torch.isfinite(mean).all()) and bool(torch.isfinite(rstd).all())
        assert float((mean[0] / float(x[0, 0, 0].float()) - 1).abs().max()) <= (chain(P * 8) + 4) * 2.0 ** -24
        within(y[1], torch.full_like(y[1], 0.5).double(), half_step(bf16))


@pytest.mark.parametrize("bf16", [False, True])
def test_group_norm_keeps_nan_in_its_group(bf16):
    torch = _torch()
    d = dt(bf16)
    for P in (10, 5000):
        x = randn(gen(1), 3, P, 32, dtype=d)
        x[1, 4, 9] = float("nan")
        y = torch.empty_like(x)
        gpu.group_norm(x, 4, None, None, y, None, None)
        bad = torch.isnan(y)
        assert bool(bad[1, :, 8:16].all()) and int(bad.sum()) == P * 8


def nan_at(t, *where):
    """t is NaN at `where`, an index or mask, and finite elsewhere."""
    torch = _torch()
    mask = torch.zeros_like(t, dtype=torch.bool)
    mask[where] = True
    return bool(torch.isnan(t[mask]).all()) and bool(torch.isfinite(t[~mask]).all())


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("act", [gpu.ACT_GELU, gpu.ACT_SILU])
@pytest.mark.parametrize("D", [1, 2, 3, 8])
@pytest.mark.parametrize("P", [10, 200000])
def test_group_norm_with_an_activation_keeps_nan_in_its_group(P, D, act, bf16):
    """A NaN in x stays in its group, one in w or b in its channel; backward, one in x or w or b in its group's dx and its channel's dw and db
    (in x also those of the group's other channels, through their xh)."""
    torch = _torch()
    d, C = dt(bf16), 48
    G, c = C // D, 25
    lo = c // D * D
    group = slice(lo, lo + D)
    for what in ("x", "w", "b"):
        g = gen(D)
        x, dy = randn(g, 2, P, C, dtype=d), randn(g, 2, P, C, dtype=d)
        w, b = torch.ones(C, device="cuda", dtype=d), torch.zeros(C, device="cuda", dtype=d)
        mean, rstd = torch.empty(2, G, device="cuda"), torch.empty(2, G, device="cuda")
        y = torch.empty_like(x)
        {"x": x[1, P // 2], "w": w, "b": b}[what][c] = float("nan")
        gpu.group_norm(x, G, w, b, y, mean, rstd, 1e-5, act)
        assert nan_at(y, 1, slice(None), group) if what == "x" else nan_at(y, slice(None), slice(None), c)
        dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
        gpu.group_norm_grad(dy, x, G, w, b, mean, rstd, dx, dw, db, act)
        assert nan_at(dx, 1, slice(None), group) if what == "x" else nan_at(dx, slice(None), slice(None), group)
        channels = group if what == "x" else c
        assert nan_at(dw, channels) and nan_at(db, channels)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("act", [gpu.ACT_GELU, gpu.ACT_SILU])
def test_linear_grad_keeps_nan_in_its_column(act, bf16):
    """A NaN in the saved pre-activation reaches its column of dw and db and its row of dx."""
    torch = _torch()
    d = dt(bf16)
    for M, K, N in ((300, 40, 64), (300, 40, 63), (5, 24, 32), (1500, 1024, 1024)):
        g = gen(M)
        dy, x, w, z = randn(g, M, N, dtype=d), randn(g, M, K, dtype=d), randn(g, K, N, dtype=d), randn(g, M, N, dtype=d)
        z[M // 2, N // 2 + 1] = float("nan")
        dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(N, device="cuda", dtype=d)
        gpu.linear_grad(dy, x, w, z, dx, dw, db, act)
        assert nan_at(dx, M // 2) and nan_at(dw, slice(None), N // 2 + 1) and nan_at(db, N // 2 + 1)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n", [96, 95])
def test_silu_slopes_far_above_zero_beside_smaller_ones(n, bf16):
    """s (1 + z (1 - s)) for z of every size next to z of every other: 1 - s is exp(-z) s, not the rounding of s.  A slope of 1.1 at most, its
    factors good to 2^-20."""
    torch = _torch()
    d, u = dt(bf16), half_step(bf16)
    large = [12.0, 20.0, 30.0, 80.0, 1e3, 1e5, 1e8, 1e15, 1e30]
    small = [-40.0, -3.0, 0.0, 0.3, 0.7, 1.5, 2.5, 5.0]
    for shift in range(4):                                               # (which of its neighbours shares something with an element is the kernel's choice)
        for big in large:
            z = torch.tensor([big if (j >> 1) % 2 == shift % 2 and (j % 2 == 0 or shift > 1) else small[(j * 5 + shift) % 8] for j in range(n)], device="cuda").to(d)
            slope = slope64(z.double(), gpu.ACT_SILU)
            db, dw = torch.empty(n, device="cuda", dtype=d), torch.empty(16, n, device="cuda", dtype=d)
            x = torch.zeros(4, 16, device="cuda", dtype=d)
            x[0, 0] = 1.0
            gpu.linear_grad(torch.ones(4, n, device="cuda", dtype=d), x, torch.zeros(16, n, device="cuda", dtype=d), z.expand(4, n).contiguous(), None, dw, db,
                            gpu.ACT_SILU)
            within(dw[0], slope, u * slope.abs() + 2 * E20)
            within(db, 4 * slope, 4 * u * slope.abs() + 8 * E20)
            x = torch.full((1, 64, n), 2.0, device="cuda", dtype=d)      # constant maps: u = b
            mean, rstd = torch.full((1, 1), 2.0, device="cuda"), torch.ones(1, 1, device="cuda")
            gpu.group_norm_grad(torch.ones_like(x), x, 1, None, z, mean, rstd, None, None, db, gpu.ACT_SILU)
            within(db, 64 * slope, 64 * (u * slope.abs() + 2 * E20))


def norm_grad_case(N, P, C, G, bf16, act, affine=True, pad_p=0, pad_s=0, offset=0, seed=0, want=(True, True, True), in_place=False, differences=False):
    torch = _torch()
    g = gen(seed)
    d, u = dt(bf16), half_step(bf16)
    eps = 1e-5
    _, x, _ = maps(N, P, C, d, pad_p, pad_s, offset, (randn(g, N, P, C) + 0.5 * randn(g, C)).to(d))
    _, dy, _ = maps(N, P, C, d, pad_p, pad_s, offset, randn(g, N, P, C, dtype=d))
    x64, dy64 = x.double(), dy.double().clone()
    w = (1 + 0.2 * randn(g, C)).to(d) if affine else None
    b = randn(g, C, scale=0.3, dtype=d) if affine else None
    _, m64, _, r64 = norm_parts(x64, G, eps)
    mean, rstd = m64.float().contiguous(), r64.float().contiguous()
    buf, dx, outside = maps(N, P, C, d, pad_p, pad_s, offset)
    if in_place:
        dx = dy
    dw = torch.full((C,), float("nan"), device="cuda", dtype=d) if want[1] else None
    db = torch.full((C,), float("nan"), device="cuda", dtype=d) if want[2] else None
    gpu.group_norm_grad(dy, x, G, w, b, mean, rstd, dx if want[0] else None, dw, db, act)
    torch.cuda.synchronize()
    e = lambda t: t.double()[:, None, :, None]                            # noqa: E731
    xg, gy = x64.view(N, P, G, C // G), dy64.view(N, P, G, C // G)
    xh = (xg - e(mean)) * e(rstd)
    w64 = w.double().view(G, C // G) if affine else torch.ones(G, C // G, dtype=torch.float64, device="cuda")
    b64 = b.double().view(G, C // G) if affine else torch.zeros(G, C // G, dtype=torch.float64, device="cuda")
    z = xh * w64 + b64
    txh = 2.0 ** -22 * xh.abs()
    tz = txh * w64.abs() + 2.0 ** -23 * (z.abs() + b64.abs())
    gz = gy * slope64(z, act)
    tg = 2.0 ** -23 * gz.abs() + (gy.abs() * (0.8 * tz + E20 * (1 + z.abs())) if smooth(act) else 0.0)
    n = P * (C // G)
    if want[1]:
        s = (gz * xh).sum(dim=(0, 1))
        tol = (tg * xh.abs() + gz.abs() * txh + (chain(N * P) + 8) * 2.0 ** -23 * (gz * xh).abs()).sum(dim=(0, 1))
        within(dw, s.reshape(C), (u * s.abs() + tol).reshape(C))
    if want[2]:
        s = gz.sum(dim=(0, 1))
        within(db, s.reshape(C), (u * s.abs() + (tg + (chain(N * P) + 8) * 2.0 ** -23 * gz.abs()).sum(dim=(0, 1))).reshape(C))
    if want[0]:
        gw, tgw = gz * w64, tg * w64.abs() + 2.0 ** -23 * (gz * w64).abs()
        mean_of = lambda t: t.mean(dim=(1, 3), keepdim=True)              # noqa: E731
        s1, s2 = mean_of(gw), mean_of(gw * xh)
        L = (chain(n) + 8) * 2.0 ** -23
        t1 = mean_of(tgw) + L * mean_of(gw.abs())
        t2 = mean_of(tgw * xh.abs() + gw.abs() * txh) + L * mean_of((gw * xh).abs())
        out = e(rstd) * (gw - s1 - xh * s2)
        tol = u * out.abs() + e(rstd) * (tgw + t1 + xh.abs() * t2 + txh * s2.abs() + 2.0 ** -22 * (gw.abs() + s1.abs() + (xh * s2).abs()))
        within(dx, out.view(N, P, C), tol.view(N, P, C))
        if not in_place:
            assert bool(torch.isnan(buf[outside]).all())
    if differences:
        # L = sum dy act(group_norm(x) w + b) in 64 bits, central differences of step 1e-6 (truncation 1e-10 or less); the gradients
        # are taken at mean and rstd rounded to fp32 (2^-24 each), which moves xh by 2^-23 (|xh| + |mean| rstd)
        h = 1e-6

        def loss(xx, ww, bb):
            q, m, _, r = norm_parts(xx, G, eps)
            return float((gy * act64((q - m[:, None, :, None]) * r[:, None, :, None] * ww + bb, act)).sum())

        for got, at in ((dx, 0), (dw, 1), (db, 2)):
            args = [x64.contiguous(), w64, b64]
            v = torch.randn(args[at].shape, generator=g, device="cuda", dtype=torch.float64)
            lo, hi = list(args), list(args)
            lo[at], hi[at] = args[at] - h * v, args[at] + h * v
            num = (loss(*hi) - loss(*lo)) / (2 * h)
            mag = float((got.double().reshape(v.shape).abs() * v.abs()).sum())
            assert abs(float((got.double().reshape(v.shape) * v).sum()) - num) <= 1e-5 * mag + 1e-6


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("N,P,C,G", NORM_SIZES)
def test_group_norm_grad_sizes(N, P, C, G, bf16):
    norm_grad_case(N, P, C, G, bf16, gpu.ACT_SILU, seed=N + P + C)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("affine", [False, True])
def test_group_norm_grad_epilogues(act, affine, bf16):
    norm_grad_case(3, 144, 48, 6, bf16, act, affine, seed=act)
    norm_grad_case(3, 50, 21, 3, bf16, act, affine, seed=act, in_place=True)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("want", [(True, False, False), (False, True, False), (False, False, True), (False, True, True)])
def test_group_norm_grad_of_chosen_operands(want, bf16):
    norm_grad_case(3, 144, 48, 6, bf16, gpu.ACT_GELU, seed=1, want=want)
    norm_grad_case(2, 3000, 48, 6, bf16, gpu.ACT_GELU, seed=1, want=want)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("pad_p,pad_s,offset", [(8, 0, 0), (0, 24, 8), (1, 0, 0), (0, 1, 0), (0, 0, 1), (3, 5, 7), (4, 4, 4)])
def test_group_norm_grad_pitches_and_alignment(pad_p, pad_s, offset, bf16):
    for C, G in ((64, 8), (24, 8), (10, 5)):
        norm_grad_case(3, 120, C, G, bf16, gpu.ACT_RELU, pad_p=pad_p, pad_s=pad_s, offset=offset, seed=offset)


@pytest.mark.parametrize("bf16,N,P,C,G", [(True, 1300, 784, 6, 3), (True, 1, 1000000, 3, 1), (True, 1100, 1024, 7, 7), (True, 3, 2500001, 1, 1),
                                          (False, 1, 262144, 3, 3), (False, 700, 784, 6, 3), (False, 1300, 784, 3, 1), (False, 3, 600001, 2, 2)])
def test_group_norm_of_few_channels_in_large_calls(bf16, N, P, C, G):
    """Datasets of 28 x 28 x 6 maps, single RGB images: a position has fewer channels than a 16-byte vector, and the call more than 12 MB."""
    norm_case(N, P, C, G, bf16, gpu.ACT_SILU, seed=C)
    norm_grad_case(N, P, C, G, bf16, gpu.ACT_SILU, seed=C)


@pytest.mark.parametrize("act", [gpu.ACT_NONE, gpu.ACT_GELU, gpu.ACT_SILU])
def test_group_norm_grad_against_differences(act):
    norm_grad_case(3, 40, 24, 4, False, act, seed=9, differences=True)


def test_group_norm_of_images_and_without_samples():
    """[N, H, W, C] maps, also as a crop of larger images whose rows are not at one pitch (refused) and at one pitch (taken)."""
    torch = _torch()
    x = randn(gen(4), 2, 8, 8, 16)
    y = torch.empty_like(x)
    gpu.group_norm(x, 4, None, None, y, None, None)
    flat = torch.empty(2, 64, 16, device="cuda")
    gpu.group_norm(x.view(2, 64, 16), 4, None, None, flat, None, None)
    assert torch.equal(y.view(2, 64, 16), flat)
    with pytest.raises(ValueError):
        gpu.group_norm(x[:, :, :5], 4, None, None, y[:, :, :5], None, None)
    crop = torch.empty(2, 5, 8, 16, device="cuda")
    gpu.group_norm(x[:, :5], 4, None, None, crop, None, None)
    want = torch.empty(2, 5, 8, 16, device="cuda")
    gpu.group_norm(x[:, :5].contiguous(), 4, None, None, want, None, None)
    assert torch.equal(crop, want)
    empty = torch.empty(0, 8, 8, 16, device="cuda")
    gpu.group_norm(empty, 4, None, None, empty.clone(), None, None)
    dw = torch.ones(16, device="cuda")
    st = torch.empty(0, 4, device="cuda")
    gpu.group_norm_grad(empty, empty.clone(), 4, None, None, st, st.clone(), empty.clone(), dw, None)
    assert float(dw.abs().sum()) == 0.0


# ------------------------------------------------------------------------------------------------ together, streams, graphs

class Block:
    """A residual block of channels-last maps x [N, P, C]: y = x + dropout(gelu(silu(group_norm(x)) W1 + b1)) W2 + b2, forward and
    backward through the operations, all buffers its own."""

    def __init__(self, N, P, C, H, bf16, seed):
        torch = _torch()
        g, d = gen(seed), dt(bf16)
        self.N, self.P, self.C, self.H, self.p, self.seed, self.call = N, P, C, H, 0.25, 77, 5
        self.x, self.dy = randn(g, N, P, C, dtype=d), randn(g, N, P, C, dtype=d)
        self.gw, self.gb = (1 + 0.1 * randn(g, C)).to(d), randn(g, C, scale=0.1, dtype=d)
        self.w1, self.b1 = randn(g, C, H, scale=math.sqrt(2 / C), dtype=d), randn(g, H, scale=0.1, dtype=d)
        self.w2, self.b2 = randn(g, H, C, scale=math.sqrt(2 / H), dtype=d), randn(g, C, scale=0.1, dtype=d)
        e = lambda *s: torch.zeros(*s, device="cuda", dtype=d)            # noqa: E731
        self.h, self.z, self.a, self.q, self.y = e(N, P, C), e(N * P, H), e(N * P, H), e(N * P, H), e(N, P, C)
        self.mean, self.rstd = torch.zeros(N, 4, device="cuda"), torch.zeros(N, 4, device="cuda")
        self.dq, self.da, self.dh, self.dx = e(N * P, H), e(N * P, H), e(N, P, C), e(N, P, C)
        self.dw1, self.db1, self.dw2, self.db2, self.dgw, self.dgb = e(C, H), e(H), e(H, C), e(C), e(C), e(C)
        code = gpu.BF16_FP32MASTER if bf16 else gpu.FP32
        need = [gpu.linear_scratch_bytes(N * P, C, H, gpu.ACT_GELU, code, grad) for grad in (False, True)]
        need += [gpu.linear_scratch_bytes(N * P, H, C, gpu.ACT_NONE, code, grad) for grad in (False, True)]
        need += [gpu.group_norm_scratch_bytes(N, P, C, 4, code, grad) for grad in (False, True)]
        self.scratch = torch.empty(max(need) + 1, dtype=torch.uint8, device="cuda")

    def step(self, stream=None):
        N, P, C = self.N, self.P, self.C
        rows = lambda t: t.view(N * P, C)                                 # noqa: E731
        kw = dict(scratch=self.scratch, stream=stream)
        gpu.group_norm(self.x, 4, self.gw, self.gb, self.h, self.mean, self.rstd, 1e-5, gpu.ACT_SILU, **kw)
        gpu.linear(rows(self.h), self.w1, self.b1, None, self.a, gpu.ACT_GELU, pre=self.z, **kw)
        gpu.dropout(self.a, None, self.q, self.p, self.seed, self.call, stream=stream)
        gpu.linear(self.q, self.w2, self.b2, rows(self.x), rows(self.y), **kw)
        gpu.linear_grad(rows(self.dy), self.q, self.w2, None, self.dq, self.dw2, self.db2, **kw)
        gpu.dropout(self.dq, None, self.da, self.p, self.seed, self.call, stream=stream)
        gpu.linear_grad(self.da, rows(self.h), self.w1, self.z, rows(self.dh), self.dw1, self.db1, gpu.ACT_GELU, **kw)
        gpu.group_norm_grad(self.dh, self.x, 4, self.gw, self.gb, self.mean, self.rstd, self.dx, self.dgw, self.dgb, gpu.ACT_SILU, **kw)

    def results(self):
        """(dx is the branch's part: the residual path adds dy)"""
        return [t.clone() for t in (self.y, self.dx, self.dgw, self.dgb, self.dw1, self.db1, self.dw2, self.db2)]

    def reference(self):
        torch = _torch()
        N, P, C, G = self.N, self.P, self.C, 4
        leaves = [t.double().requires_grad_() for t in (self.x, self.gw, self.gb, self.w1, self.b1, self.w2, self.b2)]
        x, gw, gb, w1, b1, w2, b2 = leaves
        keep = torch.from_numpy(keep_mask(N * P, self.H, self.p, self.seed, self.call)).cuda()
        xg, m, _, r = norm_parts(x, G, 1e-5)
        u = ((xg - m[:, None, :, None]) * r[:, None, :, None]).reshape(N * P, C) * gw + gb
        a = act64(act64(u, gpu.ACT_SILU) @ w1 + b1, gpu.ACT_GELU)
        branch = (keep * a * (65536 / (65536 - 16384))) @ w2 + b2
        grads = torch.autograd.grad((branch * self.dy.double().view(N * P, C)).sum(), leaves)
        return [(branch + x.view(N * P, C)).view(N, P, C).detach(), grads[0]] + list(grads[1:])


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("N,P,C,H", [(3, 49, 32, 64), (2, 100, 36, 75), (4, 256, 128, 256)])
def test_a_residual_block_forward_and_backward(N, P, C, H, bf16):
    """Relative to each result's norm: six stored quantities lie between the inputs and the last gradient, each rounded by at most half
    a step u; the products' sums in fp32 add (C + H) 2^-23.  Independent errors at most add up: 8 u."""
    block = Block(N, P, C, H, bf16, 1)
    block.step()
    tol = 8 * half_step(bf16) + 4 * (C + H) * E23
    for got, want in zip(block.results(), block.reference()):
        assert float((got.double().view(want.shape) - want).norm()) <= tol * float(want.norm())


@pytest.mark.parametrize("bf16", [False, True])
def test_captured_steps_and_other_streams_give_the_same_bits(bf16):
    torch = _torch()
    one = Block(4, 100, 64, 128, bf16, 2)
    one.step()
    torch.cuda.synchronize()
    want = one.results()
    one.step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(one.results(), want))
    # two steps at once on streams of their own
    two, three = Block(4, 100, 64, 128, bf16, 2), Block(4, 100, 64, 128, bf16, 2)
    s2, s3 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        two.step(stream=s2)
        three.step(stream=s3)
    torch.cuda.synchronize()
    for blk in (two, three):
        assert all(torch.equal(a, b) for a, b in zip(blk.results(), want))
    # captured, then replayed on new inputs
    four = Block(4, 100, 64, 128, bf16, 3)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        four.step()
    four.x.copy_(one.x)
    four.dy.copy_(one.dy)
    for name in ("gw", "gb", "w1", "b1", "w2", "b2"):
        getattr(four, name).copy_(getattr(one, name))
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(four.results(), want))


def test_scratch_allocated_by_the_call_on_another_stream():
    torch = _torch()
    g = gen(6)
    dy, x, w, z = randn(g, 500, 129), randn(g, 500, 65), randn(g, 65, 129), randn(g, 500, 129)
    outs = []
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (None, s):
        dx, dw, db = torch.empty(500, 65, device="cuda"), torch.empty(65, 129, device="cuda"), torch.empty(129, device="cuda")
        torch.cuda.synchronize()
        for _ in range(4):
            gpu.linear_grad(dy, x, w, z, dx, dw, db, gpu.ACT_GELU, stream=stream)
        torch.cuda.synchronize()
        outs.append((dx, dw, db))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("bf16", [False, True])
def test_a_trained_model_evaluated_on_its_data(bf16):
    """get_params of a run, layer by layer through `linear` over the whole dataset, against the same in 64 bits."""
    torch = _torch()
    from paper_2301_08895_b200 import inputs
    cfg = inputs.config(3).scaled(n_samples=4096, dtype=inputs.BF16 if bf16 else inputs.FP32)
    X, y, _ = inputs.make_data(cfg)
    Xd = torch.from_numpy(X.view(np.int16)).cuda().view(torch.bfloat16) if bf16 else torch.from_numpy(X).cuda()
    ctx = gpu.context_from_config(cfg, Xd, torch.from_numpy(y).cuda(), inputs.make_w0(cfg), max_rounds=4)
    ctx.run_rounds(4)
    params = ctx.get_params()
    ctx.close()
    d, off, h, h64 = dt(bf16), 0, Xd, Xd.double()
    for l in range(2):
        i, o = cfg.dims[l], cfg.dims[l + 1]
        w = torch.from_numpy(params[off:off + i * o].reshape(i, o)).cuda().to(d)
        b = torch.from_numpy(params[off + i * o:off + i * o + o]).cuda().to(d)
        off += i * o + o
        act = gpu.ACT_RELU if l == 0 else gpu.ACT_NONE
        out = torch.empty(h.shape[0], o, device="cuda", dtype=d)
        gpu.linear(h, w, b, None, out, act)
        h64 = act64(h64 @ w.double() + b.double(), act)
        h = out
    # two stored layers: each rounded by half a step, the first one's rounding goes through the second
    assert float((h.double() - h64).norm()) <= 3 * (half_step(bf16) + 800 * E23) * float(h64.norm())
    assert off == params.size


def test_a_wait_that_runs_out_is_reported_once():
    torch = _torch()
    gpu.op_status()
    assert gpu.lib().abs_op_selftest_wait_timeout(1000, torch.cuda.current_stream().cuda_stream) == gpu.OK
    with pytest.raises(gpu.AbsError) as e:
        gpu.op_status()
    assert e.value.code == gpu.ETIMEOUT
    gpu.op_status()
    test_linear_adds_to_the_residual_in_place(True)               # (the operations go on working)
    gpu.op_status()


def test_no_report_of_a_wait_is_lost_beside_other_readers():
    """Two threads ask for the status all the time while waits run out on a third stream, one at a time: one of them, or the last question, reports
    each."""
    import threading
    torch = _torch()
    gpu.op_status()
    reports, done, lock = [0], threading.Event(), threading.Lock()

    def ask(stream):
        try:
            gpu.op_status(stream)
        except gpu.AbsError as e:
            assert e.code == gpu.ETIMEOUT
            with lock:
                reports[0] += 1

    def reader():
        stream = torch.cuda.Stream()
        while not done.is_set():
            ask(stream)
    threads = [threading.Thread(target=reader) for _ in range(2)]
    for t in threads:
        t.start()
    raised = torch.cuda.Stream()
    lost = 0
    for k in range(300):
        before = reports[0]
        assert gpu.lib().abs_op_selftest_wait_timeout(1 + k % 7, raised.cuda_stream) == gpu.OK
        raised.synchronize()
        ask(raised)
        for _ in range(2000):
            if reports[0] > before:
                break
            time.sleep(1e-4)
        lost += reports[0] == before
    done.set()
    for t in threads:
        t.join()
    assert lost == 0 and reports[0] == 300
    gpu.op_status()


def test_column_ranges_of_one_buffer():
    """Operands and results that are column ranges of one matrix do not overlap."""
    torch = _torch()
    for bf16 in (False, True):
        d = dt(bf16)
        buf = randn(gen(8), 300, 64 + 32 + 32 + 8, dtype=d)
        before = buf.clone()
        w = randn(gen(9), 64, 32, dtype=d)
        gpu.linear(buf[:, :64], w, None, buf[:, 64:96], buf[:, 96:128])
        want = before[:, :64].double() @ w.double() + before[:, 64:96].double()
        tol = half_step(bf16) * want.abs() + 70 * E23 * (before[:, :64].double().abs() @ w.double().abs() + before[:, 64:96].double().abs())
        within(buf[:, 96:128], want, tol)
        assert torch.equal(buf[:, :96], before[:, :96]) and torch.equal(buf[:, 128:], before[:, 128:])
        with pytest.raises(gpu.AbsError):
            gpu.linear(buf[:, :64], w, None, None, buf[:, 60:92])


def test_layer_operations_refuse_wrong_tensors():
    torch = _torch()
    x, w, y = torch.zeros(4, 8, device="cuda"), torch.zeros(8, 16, device="cuda"), torch.zeros(4, 16, device="cuda")
    with pytest.raises(ValueError):
        gpu.linear(x.double(), w, None, None, y)
    with pytest.raises(ValueError):
        gpu.linear(x, w.bfloat16(), None, None, y)
    with pytest.raises(ValueError):
        gpu.linear(x, w, None, None, y[:3])
    with pytest.raises(ValueError):
        gpu.linear(x, w, None, None, torch.zeros(16, 4, device="cuda").t())
    with pytest.raises(ValueError):
        gpu.linear(x, w.cpu(), None, None, y)
    with pytest.raises(gpu.AbsError) as e:
        gpu.linear(x, w, None, None, y.as_strided((4, 16), (8, 1)))
    assert e.value.code == gpu.EINVAL
    with pytest.raises(gpu.AbsError) as e:
        gpu.linear_grad(y, x, w, None, torch.empty_like(x), None, torch.empty(16, device="cuda"),
                        scratch=torch.empty(8, dtype=torch.uint8, device="cuda"))
    assert e.value.code == gpu.ENOSPACE
    with pytest.raises(gpu.AbsError) as e:
        gpu.linear(x, w, None, None, y, 9)
    assert e.value.code == gpu.EUNSUPPORTED
    with pytest.raises(ValueError):
        gpu.dropout(x, None, x, 0.5, 1 << 64, 0)
    with pytest.raises(gpu.AbsError) as e:
        gpu.dropout(x, None, x, 1.5, 0, 0)
    assert e.value.code == gpu.EINVAL
    m = torch.zeros(2, 9, 16, device="cuda")
    with pytest.raises(gpu.AbsError) as e:
        gpu.group_norm(m, 5, None, None, m, None, None)
    assert e.value.code == gpu.EINVAL
    with pytest.raises(ValueError):
        gpu.group_norm(m, 4, torch.ones(8, device="cuda"), None, m, None, None)


@pytest.mark.parametrize("bf16", [False, True])
def test_silu_is_one_function(bf16):
    """Values and slopes far below zero, at -infinity and at NaN are the same wherever they are formed: element by element or in vectors, in
    the layer of a few or many rows, in its gradient and in group norm."""
    torch = _torch()
    d = dt(bf16)
    z = [-30.0, -41.0, -42.0, -60.0, -88.0, -90.0, -200.0, -1e4, -1e30, -float("inf"), float("nan"), -41.4]
    vals, slopes = [], []
    for n in (96, 95):                                       # whole vectors, or not
        zt = torch.tensor([z[j % len(z)] for j in range(n)], device="cuda").to(d)
        for rows in (1, 5, 300):
            y = torch.empty(rows, n, device="cuda", dtype=d)
            gpu.linear(torch.zeros(rows, 16, device="cuda", dtype=d), torch.zeros(16, n, device="cuda", dtype=d), zt, None, y, gpu.ACT_SILU)
            vals.append(y[rows - 1, :len(z)])
            db = torch.empty(n, device="cuda", dtype=d)
            dy = torch.zeros(rows, n, device="cuda", dtype=d)
            dy[rows - 1] = 1.0
            gpu.linear_grad(dy, torch.zeros(rows, 16, device="cuda", dtype=d), torch.zeros(16, n, device="cuda", dtype=d), zt.expand(rows, n).contiguous(),
                            None, None, db, gpu.ACT_SILU)
            slopes.append(db[:len(z)])
        for P in (1, 400000):
            x = torch.full((1, P, n), 2.0, device="cuda", dtype=d)        # constant maps: u = b
            y, st = torch.empty_like(x), [torch.empty(1, 1, device="cuda") for _ in range(2)]
            gpu.group_norm(x, 1, None, zt, y, *st, 1.0, gpu.ACT_SILU)
            vals.append(y[0, P - 1, :len(z)])
            dy = torch.zeros_like(x)
            dy[0, P // 2] = 1.0
            gpu.group_norm_grad(dy, x, 1, None, zt, *st, None, None, db, gpu.ACT_SILU)
            slopes.append(db[:len(z)])
    for got in (vals, slopes):
        first = got[0].double()
        assert bool(torch.isnan(first[10])) and bool(torch.isfinite(torch.cat([first[:10], first[11:]])).all())
        # (the reciprocal shared with another partner is another rounding: rcp 2^-22, two products 2^-24 each)
        assert 0 < -float(first[2]) < 4e-17 and bool(((first[2:10] / first[2] - 1).abs() <= 2.0 ** -19).all())
        for other in got[1:]:                                # (the two forms of the reciprocal differ by roundings; u for a step of bf16)
            assert bool(torch.isnan(other[10]))
            keep = [i for i in range(len(z)) if i != 10]
            within(other[keep], first[keep], (2.0 ** -19 + (2 * half_step(bf16) if bf16 else 0.0)) * first[keep].abs())


def test_gelu_on_a_dense_grid():
    """Phi good to 2^-21 everywhere, and for z in [-12, 0] to 2^-16 of itself: the fit 2^-24.9, its evaluation 2^-21, exp(-z^2 / 2) at arguments up
    to 104 rounded twice 2^-16.8.  The slope adds z exp(-z^2 / 2) / sqrt(2 pi), below 0.25, good to 2^-20 where it counts."""
    torch = _torch()
    z = torch.linspace(-14, 14, 1 << 20, device="cuda")
    n = z.numel()
    z64 = z.double()
    phi = 0.5 * torch.special.erfc(-z64 / math.sqrt(2))
    slope = phi + z64 * torch.exp(-z64 * z64 / 2) / math.sqrt(2 * math.pi)
    left = (z >= -12) & (z <= 0)
    got = []
    for rows in (1, 9):                                                  # a few rows; the tiled product
        y = torch.empty(rows, n, device="cuda")
        gpu.linear(torch.zeros(rows, 8, device="cuda"), torch.zeros(8, n, device="cuda"), z, None, y, gpu.ACT_GELU)
        got.append(y[rows - 1])
    x = torch.full((1, 16, n), 2.0, device="cuda")                       # constant maps: u = b
    mean, rstd = torch.empty(1, 1, device="cuda"), torch.empty(1, 1, device="cuda")
    y, db, db2 = torch.empty_like(x), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    gpu.group_norm(x, 1, None, z, y, mean, rstd, 1.0, gpu.ACT_GELU)
    got.append(y[0, 3])
    for y in got:
        within(y, z64 * phi, 2.0 ** -21 * z64.abs() + 2.0 ** -24 * (z64 * phi).abs())
        within(y[left], (z64 * phi)[left], 2.0 ** -16 * (z64 * phi)[left].abs())
    gpu.linear_grad(torch.ones(1, n, device="cuda"), torch.zeros(1, 8, device="cuda"), torch.zeros(8, n, device="cuda"), z.view(1, n), None, None, db,
                    gpu.ACT_GELU)
    dy = torch.zeros_like(x)
    dy[0, 5] = 1.0
    gpu.group_norm_grad(dy, x, 1, None, z, mean, rstd, None, None, db2, gpu.ACT_GELU)
    for d in (db, db2):
        within(d, slope, torch.full_like(slope, 2.0 ** -20))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("P,pad", [(1, 0), (1, 5), (9, 0), (9, 3)])
def test_group_norm_of_channel_ranges_of_one_buffer(P, pad, bf16):
    """Maps that are channel ranges of one buffer do not overlap: also with one position per sample, and where a sample's pitch is no multiple of a
    position's.  One channel less between them and they do."""
    torch = _torch()
    d, C, N = dt(bf16), 16, 6
    wide = 3 * C + 8
    buf = torch.full((N * (P * wide + pad) + 16,), 7.0, device="cuda", dtype=d)
    part = lambda c: buf.as_strided((N, P, C), (P * wide + pad, wide, 1), c)         # noqa: E731
    x, y, dx = part(0), part(C + 8), part(2 * C + 8)
    x.copy_(randn(gen(P), N, P, C, dtype=d))
    keep = x.clone()
    mean, rstd, want = torch.empty(N, 2, device="cuda"), torch.empty(N, 2, device="cuda"), torch.empty_like(keep)
    gpu.group_norm(keep, 2, None, None, want, mean, rstd, 1e-5, gpu.ACT_GELU)
    gpu.group_norm(x, 2, None, None, y, None, None, 1e-5, gpu.ACT_GELU)
    assert torch.equal(y, want) and torch.equal(x, keep)
    dy = randn(gen(P + 1), N, P, C, dtype=d)
    y.copy_(dy)
    gpu.group_norm_grad(dy, keep, 2, None, None, mean, rstd, want, None, None, gpu.ACT_GELU)
    gpu.group_norm_grad(y, x, 2, None, None, mean, rstd, dx, None, None, gpu.ACT_GELU)
    assert torch.equal(dx, want) and torch.equal(y, dy) and torch.equal(x, keep)
    assert bool((part(C)[:, :, :8] == 7.0).all())
    for other in (part(C - 1), part(2 * C + 9 + (pad if P == 1 else 0))):  # (the last one's end reaches the next position's first channel)
        with pytest.raises(gpu.AbsError) as e:
            gpu.group_norm(x[:N - 1], 2, None, None, other[:N - 1], None, None)
        assert e.value.code == gpu.EINVAL
