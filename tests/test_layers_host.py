"""Argument checks of the layer operations' C entry points, and their scratch sizes; none of it reaches a device."""
import ctypes as C
import os
import subprocess
import sys
import time

import numpy as np
import pytest

import helpers
from paper_2301_08895_b200 import abs as gpu
from paper_2301_08895_b200 import build


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


A = 1 << 20          # addresses that are never read


def linear(x=A, ldx=8, w=2 * A, ldw=16, bias=0, res=0, ldr=0, y=3 * A, ldy=16, pre=0, ldp=0, rows=4, n_in=8, n_out=16, act=0, dtype=0,
           scratch=0, sz=0):
    return gpu.lib().abs_linear(x, ldx, w, ldw, bias, res, ldr, y, ldy, pre, ldp, rows, n_in, n_out, act, dtype, scratch, sz, None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(dtype=2), gpu.EUNSUPPORTED, "dtype"), (dict(act=4), gpu.EUNSUPPORTED, "activation"), (dict(act=-1), gpu.EUNSUPPORTED, "activation"),
    (dict(rows=-1), gpu.EINVAL, "rows"), (dict(rows=1 << 31), gpu.EINVAL, "rows"), (dict(n_in=0), gpu.EINVAL, "n_in"),
    (dict(n_out=(1 << 20) + 1), gpu.EINVAL, "n_out"), (dict(x=0), gpu.EINVAL, "x is null"), (dict(w=0), gpu.EINVAL, "w is null"),
    (dict(y=0), gpu.EINVAL, "y is null"), (dict(ldx=7), gpu.EINVAL, "x: row pitch"), (dict(ldw=15), gpu.EINVAL, "w: row pitch"),
    (dict(ldy=0), gpu.EINVAL, "y: row pitch"), (dict(bias=4 * A + 1), gpu.EINVAL, "bias"), (dict(x=A + 2), gpu.EINVAL, "aligned"), (dict(y=A), gpu.EINVAL, "y overlaps"),
    (dict(y=2 * A + 4), gpu.EINVAL, "y overlaps"), (dict(bias=3 * A + 64), gpu.EINVAL, "y overlaps"),
    (dict(pre=3 * A, ldp=16), gpu.EINVAL, "pre overlaps"), (dict(res=3 * A + 64, ldr=16), gpu.EINVAL, "residual"),
    (dict(res=3 * A, ldr=32), gpu.EINVAL, "residual"),
    (dict(x=3 * A, ldx=30, y=3 * A + 32, ldy=32), gpu.EINVAL, "y overlaps"),        # column ranges, but not at one pitch
])
def test_linear_refuses(kw, code, text):
    assert linear(**kw) == code
    assert text in gpu.last_error()


def test_linear_fp32_long_sum_needs_scratch():
    need = gpu.linear_scratch_bytes(64, 4096, 64, dtype=gpu.FP32)
    assert need >= 2 * 64 * 64 * 4
    far = dict(rows=64, n_in=4096, ldx=4096, n_out=64, ldw=64, ldy=64, x=A, w=2 * A, y=3 * A)
    for kw, code, text in ((dict(sz=need - 1, scratch=8 * A), gpu.ENOSPACE, "scratch holds"), (dict(sz=need), gpu.EINVAL, "scratch"),
                           (dict(sz=need, scratch=2 * A + 256), gpu.EINVAL, "scratch overlaps")):
        assert linear(**far, **kw) == code
        assert text in gpu.last_error()


def test_linear_without_rows_needs_no_matrices():
    assert linear(x=0, w=0, y=0, rows=0) == gpu.OK


def linear_grad(dy=A, lddy=16, x=2 * A, ldx=8, w=3 * A, ldw=16, pre=4 * A, ldp=16, dx=5 * A, lddx=8, dw=6 * A, lddw=16, db=7 * A, rows=4, n_in=8,
                n_out=16, act=2, dtype=0, scratch=8 * A, sz=1 << 30):
    return gpu.lib().abs_linear_grad(dy, lddy, x, ldx, w, ldw, pre, ldp, dx, lddx, dw, lddw, db, rows, n_in, n_out, act, dtype, scratch, sz, None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(dy=0), gpu.EINVAL, "dy is null"), (dict(pre=0), gpu.EINVAL, "pre is null"), (dict(x=0), gpu.EINVAL, "x is null"),
    (dict(w=0), gpu.EINVAL, "w is null"), (dict(lddx=7), gpu.EINVAL, "dx: row pitch"), (dict(lddw=8), gpu.EINVAL, "dw: row pitch"),
    (dict(ldp=15), gpu.EINVAL, "pre: row pitch"), (dict(dx=A), gpu.EINVAL, "overlaps an operand"), (dict(dw=3 * A), gpu.EINVAL, "overlaps an operand"),
    (dict(db=6 * A), gpu.EINVAL, "two gradients"), (dict(sz=0), gpu.ENOSPACE, "scratch holds 0"), (dict(scratch=0), gpu.EINVAL, "scratch"),
    (dict(scratch=8 * A + 16), gpu.EINVAL, "scratch"), (dict(scratch=A), gpu.EINVAL, "scratch overlaps"), (dict(db=7 * A + 2), gpu.EINVAL, "db"),
    (dict(act=7), gpu.EUNSUPPORTED, "activation"),
])
def test_linear_grad_refuses(kw, code, text):
    assert linear_grad(**kw) == code
    assert text in gpu.last_error()


def test_linear_scratch_bytes():
    f = gpu.linear_scratch_bytes
    assert f(0, 8, 8) == 0 or f(0, 8, 8) > 0
    for dtype in (gpu.FP32, gpu.BF16_FP32MASTER):
        for grad in (False, True):
            for rows, n_in, n_out in ((1, 1, 1), (1000, 785, 10), (60000, 784, 256), (8192, 4096, 4096)):
                a, b = (f(rows, n_in, n_out, gpu.ACT_GELU, dtype, grad, al) for al in (True, False))
                assert 0 <= a <= b <= (1 << 34)
    with pytest.raises(gpu.AbsError) as e:
        f(1, 0, 1)
    assert e.value.code == gpu.EINVAL
    assert gpu.lib().abs_linear_scratch_bytes(1, 1, 1, 0, 0, 0, 0, None) == gpu.EINVAL


def dropout(x=A, ldx=16, res=0, ldr=0, y=2 * A, ldy=16, rows=4, cols=16, p=0.5, dtype=0):
    return gpu.lib().abs_dropout(x, ldx, res, ldr, y, ldy, rows, cols, p, 1, 0, dtype, None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(dtype=3), gpu.EUNSUPPORTED, "dtype"), (dict(rows=-1), gpu.EINVAL, "rows"), (dict(rows=1 << 32), gpu.EINVAL, "rows"),
    (dict(cols=0), gpu.EINVAL, "cols"), (dict(cols=1 << 31), gpu.EINVAL, "cols"), (dict(p=-0.1), gpu.EINVAL, "p "), (dict(p=1.01), gpu.EINVAL, "p "),
    (dict(p=float("nan")), gpu.EINVAL, "p "), (dict(x=0), gpu.EINVAL, "null"), (dict(y=0), gpu.EINVAL, "null"), (dict(ldx=15), gpu.EINVAL, "pitch"),
    (dict(res=3 * A, ldr=4), gpu.EINVAL, "pitch"), (dict(y=A + 4), gpu.EINVAL, "overlaps"), (dict(y=A, ldy=17), gpu.EINVAL, "overlaps"),
    (dict(res=2 * A + 64, ldr=16), gpu.EINVAL, "residual"),
])
def test_dropout_refuses(kw, code, text):
    assert dropout(**kw) == code
    assert text in gpu.last_error()


def test_dropout_without_rows():
    assert dropout(x=0, y=0, rows=0) == gpu.OK


def norm(x=A, xs=160, xp=16, y=2 * A, ys=160, yp=16, mean=0, rstd=0, n=4, pos=10, ch=16, groups=4, eps=1e-5, act=0, dtype=0):
    return gpu.lib().abs_group_norm(x, xs, xp, None, None, y, ys, yp, mean, rstd, n, pos, ch, groups, eps, act, dtype, None, 0, None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(dtype=5), gpu.EUNSUPPORTED, "dtype"), (dict(act=4), gpu.EUNSUPPORTED, "activation"), (dict(n=-1), gpu.EINVAL, "samples"),
    (dict(pos=1 << 31), gpu.EINVAL, "positions"), (dict(ch=0), gpu.EINVAL, "channels"), (dict(groups=0), gpu.EINVAL, "groups"),
    (dict(groups=3), gpu.EINVAL, "groups"), (dict(groups=32), gpu.EINVAL, "groups"), (dict(eps=0.0), gpu.EINVAL, "eps"),
    (dict(eps=float("nan")), gpu.EINVAL, "eps"), (dict(mean=3 * A), gpu.EINVAL, "mean and rstd"), (dict(x=0), gpu.EINVAL, "x is null"),
    (dict(y=0), gpu.EINVAL, "y is null"), (dict(xp=15), gpu.EINVAL, "position pitch"), (dict(xs=150), gpu.EINVAL, "samples overlap"),
    (dict(y=A + 4), gpu.EINVAL, "overlaps"), (dict(y=A, yp=20, ys=200), gpu.EINVAL, "overlaps"),
])
def test_group_norm_refuses(kw, code, text):
    assert norm(**kw) == code
    assert text in gpu.last_error()


def test_group_norm_refuses_overlapping_vectors():
    f = gpu.lib().abs_group_norm
    for w, b, mean, rstd, text in ((2 * A, None, None, None, "y overlaps w or b"), (3 * A + 2, None, None, None, "w is not aligned"),
                                   (None, None, 4 * A, 4 * A + 4, "mean overlaps rstd"), (None, None, A, 4 * A, "mean or rstd overlaps"),
                                   (None, None, 4 * A + 2, 5 * A, "mean is not aligned")):
        assert f(A, 160, 16, w, b, 2 * A, 160, 16, mean, rstd, 4, 10, 16, 4, 1e-5, 0, 0, None, 0, None) == gpu.EINVAL
        assert text in gpu.last_error()
    g = gpu.lib().abs_group_norm_grad
    for dw, db, text in ((A, None, "a gradient overlaps"), (6 * A, 6 * A + 4, "two gradients"), (3 * A, None, "a gradient overlaps"),
                         (5 * A, None, "two gradients"), (6 * A + 1, None, "dw is not aligned")):
        assert g(A, 160, 16, 2 * A, 160, 16, None, None, 3 * A, 4 * A, 5 * A, 160, 16, dw, db, 4, 10, 16, 4, 0, 0, None, 0, None) == gpu.EINVAL
        assert text in gpu.last_error()


def test_wait_selftest_limits():
    assert gpu.lib().abs_op_selftest_wait_timeout(0, None) == gpu.EINVAL
    assert gpu.lib().abs_op_selftest_wait_timeout(1000001, None) == gpu.EINVAL


def norm_grad(dy=A, ds=160, dp=16, x=2 * A, xs=160, xp=16, mean=3 * A, rstd=4 * A, dx=5 * A, dxs=160, dxp=16, n=4, pos=10, ch=16, groups=4, act=0,
              dtype=0):
    return gpu.lib().abs_group_norm_grad(dy, ds, dp, x, xs, xp, None, None, mean, rstd, dx, dxs, dxp, 6 * A, 7 * A, n, pos, ch, groups, act, dtype,
                                         None, 0, None)


@pytest.mark.parametrize("kw,text", [
    (dict(dy=0), "dy is null"), (dict(x=0), "x is null"), (dict(mean=0), "mean and rstd"), (dict(rstd=0), "mean and rstd"), (dict(dp=8), "position pitch"),
    (dict(dxs=100), "samples overlap"), (dict(dx=2 * A), "dx overlaps x"), (dict(dx=A + 4), "dx overlaps dy"), (dict(groups=5), "groups"),
])
def test_group_norm_grad_refuses(kw, text):
    assert norm_grad(**kw) == gpu.EINVAL
    assert text in gpu.last_error()


def test_tensors_that_are_not_on_a_gpu_are_refused():
    import torch
    x, w, y = torch.zeros(4, 8), torch.zeros(8, 16), torch.zeros(4, 16)
    m = torch.zeros(2, 3, 8)
    for call in (lambda: gpu.linear(x, w, None, None, y), lambda: gpu.linear_grad(y, x, w, None, x, w, None), lambda: gpu.dropout(x, None, x, 0.5, 1, 1),
                 lambda: gpu.group_norm(m, 2, None, None, m, None, None), lambda: gpu.group_norm_grad(m, m, 2, None, None, None, None, m, None, None),
                 lambda: gpu.linear(x.int(), w, None, None, y)):
        with pytest.raises(ValueError):
            call()


# Calls of abs_group_norm_scratch_bytes over every number of channels below and at a whole 16-byte vector, maps of a dataset, of single images
# and of more than 12 MB, in a process of their own: a fault of the host code ends that one only.
NORM_SCRATCH_SWEEP = """
from paper_2301_08895_b200 import abs as gpu
for channels in list(range(1, 10)) + [12, 13, 84, 255, 257, 4099]:
    for groups in {1, channels, *(d for d in (2, 3, 4, 7) if channels % d == 0)}:
        for samples, positions in ((1, 1), (20, 784), (700, 784), (1300, 784), (60000, 784), (1, 65536), (1, 262144), (1, 1000000), (1, 2 ** 31 - 1),
                                   (2 ** 31 // groups - 1, 1), (3, 5)):
            for dtype, size in ((gpu.FP32, 4), (gpu.BF16_FP32MASTER, 2)):
                for grad in (False, True):
                    n = gpu.group_norm_scratch_bytes(samples, positions, channels, groups, dtype, grad)
                    if samples * positions * channels * size > 24e6:      # read twice: statistics of every group in between
                        assert n >= samples * groups * 4 * (2 if grad else 3), (samples, positions, channels, groups, dtype, grad, n)
for case in ((1300, 784, 6, 3, gpu.BF16_FP32MASTER, False), (700, 784, 6, 3, gpu.BF16_FP32MASTER, True), (1, 262144, 3, 3, gpu.FP32, False),
             (1, 65536, 3, 3, gpu.FP32, True), (1, 1000000, 3, 1, gpu.BF16_FP32MASTER, False)):
    gpu.group_norm_scratch_bytes(*case)
print("swept")
"""


def test_group_norm_scratch_of_fewer_channels_than_a_vector():
    out = subprocess.run([sys.executable, "-c", NORM_SCRATCH_SWEEP], capture_output=True, text=True, timeout=600,
                         cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert out.returncode == 0, (out.returncode, out.stderr[-500:])
    assert out.stdout.strip() == "swept"


PAIRS = ((0, 2), (2, 0), (1, 1), (0, 1), (1, 0), (0, 0))                # the pairs of pieces that a product is taken as


def test_the_bound_of_products_in_pieces_sees_each_pair():
    """On the operands of the exact test of fp32 products in pieces: six pairs stay within 2^-22 of the product, any five do not."""
    x, w = helpers.one_product_operands(520, 64, 130, 5)
    a, b = helpers.bf16_pieces(x), helpers.bf16_pieces(w)
    want = x.astype(np.float64) @ w.astype(np.float64)
    terms = {p: a[p[0]] @ b[p[1]] for p in PAIRS}
    total = sum(terms.values())
    assert np.all(np.abs(total - want) <= 2.0 ** -23 * np.abs(want))
    for p in PAIRS:
        assert np.mean(np.abs(total - terms[p] - want) > 2.0 ** -22 * np.abs(want)) > 0.8


def test_long_sums_leave_the_tensor_cores_in_stretches():
    """A weight gradient over 16.5 million rows has 64 tiles for 74 pairs of CTAs, each a sum of 0.1 s in one go, as long as a kernel waits for anything:
    it needs room for fp32 sums outside tensor memory.  Those of a dataset of 60000 rows do not."""
    for rows, n in ((16_500_000, 2048), (5_000_000, 4096), (3_200_000, 8192)):
        assert gpu.linear_scratch_bytes(rows, n, n, gpu.ACT_NONE, gpu.BF16_FP32MASTER, True, 7) >= 4 * n * n
    for rows, n in ((60000, 4096), (8192, 4096)):
        assert gpu.linear_scratch_bytes(rows, n, n, gpu.ACT_NONE, gpu.BF16_FP32MASTER, True, 7) < 4 * n * n


def test_scratch_of_no_rows_and_of_every_alignment():
    """No rows need none; the query without known alignments covers all of them."""
    for dtype in (gpu.FP32, gpu.BF16_FP32MASTER):
        for grad in (False, True):
            for act in (gpu.ACT_NONE, gpu.ACT_GELU):
                for aligned in range(8):
                    for n_in, n_out in ((8, 8), (1, 1), (785, 10), (4096, 4096)):
                        assert gpu.linear_scratch_bytes(0, n_in, n_out, act, dtype, grad, aligned) == 0
                for rows, n_in, n_out in ((1, 1, 1), (2, 9, 9), (9, 4096, 64), (300, 256, 10), (1000, 785, 10), (60000, 784, 256), (8192, 4096, 4096),
                                          (1 << 27, 8, 8), (16_500_000, 2048, 2048)):
                    every = [gpu.linear_scratch_bytes(rows, n_in, n_out, act, dtype, grad, aligned) for aligned in range(8)]
                    assert every[0] == max(every), (rows, n_in, n_out, act, dtype, grad, every)
            for samples, positions in ((0, 5), (5, 0), (0, 0)):
                assert gpu.group_norm_scratch_bytes(samples, positions, 6, 3, dtype, grad) == 0


def test_planning_a_few_large_maps_is_quick():
    """The plan of a call is made on the host each time: for one sample of 512 x 512 x 128 as quickly as for many (two plans of 15 us when every number of
    ranges was tried, 2 us or less in all)."""
    f, out = gpu.lib().abs_group_norm_scratch_bytes, C.c_size_t(0)
    best = 1.0
    for _ in range(300):
        t0 = time.perf_counter()
        f(1, 262144, 128, 32, gpu.BF16_FP32MASTER, 1, C.byref(out))
        best = min(best, time.perf_counter() - t0)
    assert out.value > 0 and best < 12e-6
