"""Operators of a model's layers against their definitions in 64 bits.

Tolerances count roundings.  u = 2^-24 is half a step of fp32; a result stored in a type of half step h is off by at most
h |result| for that (and by half the smallest step below the normal range: 2^-25 in fp16).  A sum of N terms in fp32, whatever its order, is
off by at most N u times the sum of magnitudes.  Where inputs are small integers, every product and sum is exact in fp32 and the
comparison is for equality."""
import math

import numpy as np
import pytest
import torch

from oracle import adacgd_oracle as O
from paper_2211_00188_amd import engine as E
from paper_2211_00188_amd import layers as L

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
U = 2.0 ** -24
HALF = {F32: U, BF16: 2.0 ** -8, F16: 2.0 ** -11}
TINY = {F32: 0.0, BF16: 0.0, F16: 2.0 ** -25}


def gen(seed):
    return torch.Generator().manual_seed(seed)


def ints(shape, dtype, seed, most=3):
    return torch.randint(-most, most + 1, shape, generator=gen(seed)).to(dtype)


def normals(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=gen(seed)) * scale).to(dtype)


def gpu(t, pad=0, lead=0):
    """On the GPU, each row followed by `pad` elements of NaN; the data begins `lead` elements behind an aligned address."""
    shape = t.shape[:-1] + (t.shape[-1] + pad,)
    flat = torch.full((math.prod(shape) + lead,), float("nan"), dtype=t.dtype, device="cuda")
    view = flat[lead:].view(shape)[..., :t.shape[-1]]
    view.copy_(t)
    return view


def blank(shape, dtype, pad=0, lead=0):
    return gpu(torch.full(shape, 77.0, dtype=dtype), pad, lead)


def untouched(view, lead=0):
    """What lies between and before the rows of a matrix made by `blank` (no other element is NaN if all is well)."""
    flat = torch.as_strided(view, (view.storage_offset() + math.prod(view.shape[:-1]) * view.stride(-2),), (1,), 0)
    inside = torch.zeros_like(flat, dtype=torch.bool)
    torch.as_strided(inside, view.shape, view.stride(), view.storage_offset()).fill_(True)
    return bool(torch.isnan(flat[~inside]).all())


def offsets_of(sizes, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(sizes)]).astype(np.int64), device="cuda")


def spans(sizes, first=0):
    o = np.concatenate([[first], first + np.cumsum(sizes)]).astype(int)
    return [(int(a), int(b)) for a, b in zip(o, o[1:])]


# ---------------------------------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------------------------------
SHAPES = [
    # sizes of groups, n, k, elements between rows
    ([1], 1, 1, 0), ([1, 0, 2, 1], 33, 17, 0), ([1, 0, 2, 1], 40, 64, 3), ([5, 0, 130, 64, 1], 200, 96, 8), ([300, 17], 257, 129, 0),
    ([0, 0, 0], 64, 64, 0), ([700], 128, 512, 0), ([1] * 40, 64, 72, 0), ([2, 3, 0, 16, 17], 512, 1024, 0), ([1000, 24], 256, 264, 16),
    ([256, 512, 3], 512, 256, 0), ([63, 65, 127, 129, 31, 33], 96, 40, 0), ([4000], 40, 24, 0), ([0, 2500, 0, 0, 900], 136, 72, 8),
]


def product_case(sizes, n, k, pad, dtype, shared, seed, values):
    lead_rows, tail_rows = (3, 5) if pad else (0, 0)
    rows = lead_rows + sum(sizes) + tail_rows
    x, dy = values((rows, k), dtype, seed), values((rows, n), dtype, seed + 1)
    w = values((1 if shared else len(sizes), n, k), dtype, seed + 2)
    return lead_rows, rows, x, dy, w


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "%d-%dx%d+%d" % (len(s[0]), s[1], s[2], s[3]))
def test_products_of_integers_are_exact(dtype, shape):
    sizes, n, k, pad = shape
    for shared in (False, True):
        first, rows, x, dy, w = product_case(sizes, n, k, pad, dtype, shared, 11, ints)
        keep = torch.zeros(rows, dtype=torch.bool)
        keep[first:first + sum(sizes)] = True
        # rows of no group and weights of empty groups must not matter
        nan = float("nan")
        xg, dyg = gpu(torch.where(keep[:, None], x, nan), pad), gpu(torch.where(keep[:, None], dy, nan), pad)
        wn = w.clone()
        if not shared:
            for g, m in enumerate(sizes):
                if m == 0:
                    wn[g] = nan
        wg = gpu(wn, pad)
        wg = wg.expand(len(sizes), n, k) if shared else wg
        off = offsets_of(sizes, first)
        y64, dx64, dw64 = torch.full((rows, n), 77.0).double(), torch.full((rows, k), 77.0).double(), torch.zeros(len(sizes), n, k).double()
        for g, (a, b) in enumerate(spans(sizes, first)):
            wd = w[0 if shared else g].double()
            y64[a:b] = x[a:b].double() @ wd.t()
            dx64[a:b] = dy[a:b].double() @ wd
            dw64[g] = dy[a:b].double().t() @ x[a:b].double()
        for out in {dtype, F32}:
            y, dx, dw = blank((rows, n), out, pad), blank((rows, k), out, pad), blank((len(sizes), n, k), out, pad)
            L.group_matmul(xg, wg, off, out=y)
            L.group_matmul_dx(dyg, wg, off, out=dx)
            L.group_matmul_dw(dyg, xg, off, out=dw)
            for got, want, name in ((y, y64, "y"), (dx, dx64, "dx"), (dw, dw64, "dw")):
                assert torch.equal(got.cpu(), want.to(F32).to(out)), (name, shared, out)
                assert untouched(got), (name, shared, out)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("sizes,n,k", [
    ([5000, 0, 7041, 3, 500], 1032, 264), ([5000, 0, 7041, 3, 500], 264, 1032), ([157] * 20 + [0, 300, 1] + [150] * 20, 1032, 136),
    ([1500, 0, 2600, 700, 257, 900], 1032, 1040), ([4096] * 3, 1032, 1040), ([9000], 520, 264), ([30] * 70, 520, 264),
    ([1] * 100 + [0, 9001] + [3] * 400, 264, 136), ([2049, 2048, 5000, 0] + [2] * 300, 72, 136),
], ids=lambda v: str(len(v)) if isinstance(v, list) else str(v))
def test_products_of_many_tiles_are_exact(dtype, pad, sizes, n, k):
    """Sizes at which the larger tiles and the cut groups are used, each with whole and with ragged slices and slabs."""
    first = 3 if pad else 0
    rows, off = first + sum(sizes) + 2 * first, offsets_of(sizes, first)
    x, dy, w = (ints(s, dtype, i).cuda() for i, s in enumerate(((rows, k), (rows, n), (len(sizes), n, k))))
    y64, dx64 = torch.full((rows, n), 77.0, device="cuda").double(), torch.full((rows, k), 77.0, device="cuda").double()
    dw64 = torch.zeros((len(sizes), n, k), device="cuda").double()
    for g, (a, b) in enumerate(spans(sizes, first)):
        if b > a:
            y64[a:b] = x[a:b].double() @ w[g].double().t()
            dx64[a:b] = dy[a:b].double() @ w[g].double()
            dw64[g] = dy[a:b].double().t() @ x[a:b].double()
    x[:first] = dy[:first] = float("nan")
    x[rows - 2 * first:] = dy[rows - 2 * first:] = float("nan")
    xg, dyg, wg = gpu(x, pad), gpu(dy, pad), gpu(w, pad)
    for out in {dtype, F32}:
        y, dx, dw = blank((rows, n), out, pad), blank((rows, k), out, pad), blank((len(sizes), n, k), out, pad)
        L.group_matmul(xg, wg, off, out=y)
        L.group_matmul_dx(dyg, wg, off, out=dx)
        L.group_matmul_dw(dyg, xg, off, out=dw)
        for got, want, name in ((y, y64, "y"), (dx, dx64, "dx"), (dw, dw64, "dw")):
            assert torch.equal(got, want.float().to(out)), (name, out)
            assert untouched(got), (name, out)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("stride", [0, 8, 5])
def test_products_of_one_row_do_not_read_its_stride(dtype, stride):
    n, k = 72, 264
    x, dy, w = ints((1, k), dtype, 1).cuda(), ints((1, n), dtype, 2).cuda(), ints((1, n, k), dtype, 3).cuda()
    off, odd = offsets_of([1]), lambda t: torch.as_strided(t, t.shape, (stride, 1))
    out = dict(out=torch.empty((1, n, k), device="cuda"))
    assert torch.equal(L.group_matmul_dw(odd(dy), odd(x), off, **out)[0], (dy.double().t() @ x.double()).float())
    assert torch.equal(L.group_matmul(odd(x), w, off), (x.double() @ w[0].double().t()).float().to(dtype))
    assert torch.equal(L.group_matmul_dx(odd(dy), w, off), (dy.double() @ w[0].double()).float().to(dtype))
    one = ints((1, 1, k), dtype, 4).cuda()
    v = ints((30, k), dtype, 5).cuda()
    got = L.group_matmul(v, torch.as_strided(one, (1, 1, k), (k, stride, 1)), offsets_of([30]))
    assert torch.equal(got, (v.double() @ one[0].double().t()).float().to(dtype))


@pytest.mark.parametrize("dtype", TYPES)
def test_products_keep_infinities_and_nan_to_their_rows(dtype):
    for sizes, n, k in (([300, 200], 136, 264), ([2, 3], 136, 264), ([9000, 4000], 1032, 264)):
        x, w, off = normals((sum(sizes), k), dtype, 1).cuda(), normals((2, n, k), dtype, 2).cuda(), offsets_of(sizes)
        clean = L.group_matmul(x, w, off)
        bad = x.clone()
        rows = [1, sum(sizes) - 1]
        bad[1, 3], bad[-1, 7] = float("nan"), float("inf")
        got = L.group_matmul(bad, w, off)
        keep = torch.ones(sum(sizes), dtype=torch.bool, device="cuda")
        keep[rows] = False
        assert torch.equal(got[keep], clean[keep]) and torch.isnan(got[1]).all() and not torch.isfinite(got[-1]).any()


@pytest.mark.parametrize("dtype,small", [(F32, 2.0 ** -140), (BF16, 2.0 ** -130), (F16, 2.0 ** -20)])
def test_products_of_subnormal_numbers(dtype, small):
    """Subnormal elements count with their value, whatever tile they are in."""
    for rows, n, k in ((40, 48, 72), (2, 48, 264)):
        x = ints((rows, k), dtype, 1) * small
        w, off = ints((1, n, k), dtype, 2), offsets_of([rows])
        big = w * (1.0 if dtype == F16 else 2.0 ** 100)
        y = L.group_matmul(x.cuda(), big.to(dtype).cuda(), off, out=torch.empty((rows, n), device="cuda"))
        assert torch.equal(y.cpu(), (x.double() @ big[0].to(dtype).double().t()).float())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [([5, 0, 130, 64, 1], 200, 96, 1), ([700], 128, 512, 0), ([1, 1, 2], 320, 1024, 0), ([90, 1700], 264, 136, 0)],
                         ids=lambda s: "%d-%dx%d+%d" % (len(s[0]), s[1], s[2], s[3]))
def test_products_of_numbers(dtype, shape):
    sizes, n, k, pad = shape
    first, rows, x, dy, w = product_case(sizes, n, k, pad, dtype, False, 23, normals)
    xg, dyg, wg, off = gpu(x, pad), gpu(dy, pad), gpu(w, pad), offsets_of(sizes, first)
    y, dx, dw = L.group_matmul(xg, wg, off).cpu().double(), L.group_matmul_dx(dyg, wg, off).cpu().double(), L.group_matmul_dw(dyg, xg, off).cpu().double()

    def close(got, a, b, h):
        # every addition of a sum of N terms may round (or cut off) by a step, 2 u, of a partial sum
        want, size = a @ b, a.abs() @ b.abs()
        bound = 2 * U * a.shape[1] * size + h * want.abs() + TINY[dtype]
        assert (got - want).abs().le(bound).all(), ((got - want).abs() / bound).max()
    for g, (a, b) in enumerate(spans(sizes, first)):
        if b > a:
            xd, dyd, wd = x[a:b].double(), dy[a:b].double(), w[g].double()
            close(y[a:b], xd, wd.t(), HALF[dtype])
            close(dx[a:b], dyd, wd, HALF[dtype])
            close(dw[g], dyd.t(), xd, U)
        else:
            assert not dw[g].any()


@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_of_the_product_are_those_of_its_sum(dtype):
    """f = sum(dy * (x w^T)) is bilinear: f(x + e) - f(x) is exactly <e, dx>, and likewise for w.  Integers, so no rounding."""
    sizes, n, k = [9, 0, 40], 24, 56
    _, rows, x, dy, w = product_case(sizes, n, k, 0, dtype, False, 5, ints)
    ex, ew, off = ints(x.shape, dtype, 91), ints(w.shape, dtype, 92), offsets_of(sizes)

    def f(xx, ww):
        y = torch.empty((rows, n), device="cuda")
        return float((L.group_matmul(xx.cuda(), ww.cuda(), off, out=y).cpu().double() * dy.double()).sum())
    dx, dw = torch.empty((rows, k), device="cuda"), L.group_matmul_dw(dy.cuda(), x.cuda(), off).cpu().double()
    dx = L.group_matmul_dx(dy.cuda(), w.cuda(), off, out=dx).cpu().double()
    assert f(x + ex, w) - f(x, w) == float((ex.double() * dx).sum())
    assert f(x, w + ew) - f(x, w) == float((ew.double() * dw).sum())


@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_written_into_the_engines_array(dtype):
    """Matrices an odd number of elements apart that begin anywhere: a layer's place in ext [n, d]."""
    sizes, n, k, d, at = [40, 7, 0, 33], 24, 16, 24 * 16 + 1001, 501
    x, dy = ints((80, k), dtype, 1), ints((80, n), dtype, 2)
    ext = torch.full((4, d), 77.0, device="cuda")
    L.group_matmul_dw(dy.cuda(), x.cuda(), offsets_of(sizes), out=ext[:, at:at + n * k].unflatten(1, (n, k)))
    got = ext.cpu()
    for g, (a, b) in enumerate(spans(sizes)):
        assert torch.equal(got[g, at:at + n * k].view(n, k), (dy[a:b].double().t() @ x[a:b].double()).float())
    assert (got[:, :at] == 77).all() and (got[:, at + n * k:] == 77).all()


# ---------------------------------------------------------------------------------------------------
# layer norm
# ---------------------------------------------------------------------------------------------------
WIDTHS = [1, 2, 7, 64, 100, 256, 1001, 1024, 2048, 2056, 5003, 8192, 9000, 20001]


def norm64(x, w, b, eps):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    var = ((x - mean) ** 2).mean(1, keepdim=True)
    rstd = (var + eps) ** -0.5
    return (x - mean) * rstd * w.double() + b.double(), mean[:, 0], rstd[:, 0]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", WIDTHS)
def test_layer_norm(dtype, d):
    for rows, pad, lead in ((1, 0, 0), (5, 0, 0), (70, 8, 0), (9, 3, 1)):
        x = normals((rows, d), dtype, d + rows) + normals((rows, 1), dtype, d)
        w, b, eps = 1 + normals((d,), F32, 1, 0.1), normals((d,), F32, 2, 0.1), 1e-5
        y, mean, rstd = L.layer_norm(gpu(x, pad, lead), w.cuda(), b.cuda(), eps, out=blank((rows, d), dtype, pad, lead))
        want, m64, r64 = norm64(x, w, b, eps)
        # a lane adds at most N terms of a row, a few more joins them
        N = d / 64 + 20
        em = N * U * x.double().abs().mean(1) + U * m64.abs()
        assert (mean.cpu().double() - m64).abs().le(em).all()
        # var: its terms (x - mean)^2 are off by 2 |x - mean| (em + u |x - mean|) and their sum by N u; the error of the mean
        # itself enters by its square only.  rstd = (var + eps)^-1/2 halves that, and rounds three times
        var = r64 ** -2 - eps
        er = r64 * (0.5 * ((N + 6) * U * var + em ** 2) * r64 ** 2 + 4 * U)
        assert (rstd.cpu().double() - r64).abs().le(er).all()
        xc = (x.double() - m64[:, None]).abs()
        ey = w.double().abs() * (r64[:, None] * (em[:, None] + 3 * U * xc) + er[:, None] * xc) + 2 * U * (want.abs() + b.double().abs())
        got = y.cpu().double()
        bound = ey + HALF[dtype] * (want.abs() + ey) + TINY[dtype]
        assert (got - want).abs().le(bound).all(), ((got - want).abs() / bound).max()
        assert untouched(y)


def test_layer_norm_of_equal_elements_and_without_statistics():
    x = torch.full((3, 640), 1000.0, device="cuda")
    y, mean, rstd = L.layer_norm(x, bias=torch.arange(640.0, device="cuda"), eps=1e-4)
    assert torch.equal(y, torch.arange(640.0, device="cuda").expand(3, 640)) and (mean == 1000).all()
    assert (rstd.cpu().double() - 100.0).abs().le(100.0 * 4 * U).all()
    big = normals((33, 700), BF16, 3).cuda()
    a, mean, rstd = L.layer_norm(big)
    z, none, none2 = L.layer_norm(big, statistics=False)
    assert none is None and none2 is None and torch.equal(a, z)
    same, _, _ = L.layer_norm(big, out=big)                      # in place
    assert same.data_ptr() == big.data_ptr() and torch.equal(a, big)
    assert L.layer_norm(torch.empty((0, 64), device="cuda"))[0].shape == (0, 64)


def test_layer_norm_keeps_bad_rows_to_themselves():
    x = normals((40, 300), F32, 3)
    x[3, 7], x[9, 100], x[11, 5] = float("nan"), float("inf"), -float("inf")
    x[12] = 3e38                                                  # (the sum passes the largest number)
    dy, bad = normals((40, 300), F32, 4).cuda(), [3, 9, 11, 12]
    good = [r for r in range(40) if r not in bad]
    y, mean, rstd = L.layer_norm(x.cuda())
    dx, _, _ = L.layer_norm_backward(dy, x.cuda(), None, mean, rstd)
    z, zm, zr = L.layer_norm(x[good].cuda())
    dz, _, _ = L.layer_norm_backward(dy[good].contiguous(), x[good].cuda(), None, zm, zr)
    assert torch.equal(y[good], z) and torch.equal(dx[good], dz) and torch.isnan(y[[3, 9, 11]]).all()


def norm_grads64(dy, x, w, mean, rstd):
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    xh = (x - mean) * rstd
    c = dy * w.double()
    return rstd * (c - c.mean(1, keepdim=True) - xh * (c * xh).mean(1, keepdim=True)), dy * xh, dy


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", WIDTHS)
def test_layer_norm_gradients(dtype, d):
    for sizes, pad, lead in (([1], 0, 0), ([3, 0, 1, 30], 0, 0), ([65, 9], 8, 0), ([0, 17, 2, 0], 3, 1)):
        first, rows = (2, 2 + sum(sizes) + 3) if pad else (0, sum(sizes))
        x, dy, w = normals((rows, d), dtype, 7), normals((rows, d), dtype, 8), 1 + normals((d,), F32, 9, 0.1)
        mean, rstd = normals((rows,), F32, 10, 0.1), 1 + normals((rows,), F32, 12, 0.1).abs()      # (any are allowed)
        dx, dw, db = blank((rows, d), dtype, pad, lead), blank((len(sizes), d), F32, pad, lead), blank((len(sizes), d), F32, pad)
        L.layer_norm_backward(gpu(dy, pad, lead), gpu(x, pad, lead), w.cuda(), mean.cuda(), rstd.cuda(), offsets_of(sizes, first), dx, dw, db)
        dx64, pw, pb = norm_grads64(dy, x, w, mean, rstd)
        xh = ((x.double() - mean.double()[:, None]) * rstd.double()[:, None]).abs()
        ex = 3 * U * rstd.double()[:, None] * (x.double().abs() + mean.double().abs()[:, None])          # of xh
        c = (dy.double() * w.double()).abs()
        N = d / 64 + 24
        e1, e2 = N * U * c.mean(1, keepdim=True), (N * U * c * xh + c * ex).mean(1, keepdim=True)
        q = (c * xh).mean(1, keepdim=True)
        e = rstd.double()[:, None] * (4 * U * c + e1 + 2 * U * c.mean(1, keepdim=True) + xh * e2 + ex * q + 4 * U * xh * q) + 2 * U * dx64.abs()
        inside = slice(first, first + sum(sizes))
        got = dx.cpu().double()
        bound = (e + HALF[dtype] * (dx64.abs() + e) + TINY[dtype])[inside]
        assert (got - dx64).abs()[inside].le(bound).all(), ((got - dx64).abs()[inside] / bound).max()
        outside = torch.ones(rows, dtype=torch.bool)
        outside[inside] = False
        assert (got[outside] == 77).all() and untouched(dx) and untouched(dw) and untouched(db)
        for g, (a, b) in enumerate(spans(sizes, first)):
            n = b - a + 4
            bw = n * U * pw[a:b].abs().sum(0) + (dy[a:b].double().abs() * ex[a:b]).sum(0)
            assert (dw[g].cpu().double() - pw[a:b].sum(0)).abs().le(bw).all(), (g, d)
            assert (db[g].cpu().double() - pb[a:b].sum(0)).abs().le(n * U * pb[a:b].abs().sum(0)).all(), (g, d)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes,d", [([2000, 0, 1, 700], 72), ([1] * 300, 40), ([5000], 24), ([17, 5, 900], 2048), ([3, 2100], 1001)])
def test_gradients_of_weight_and_bias_by_group_are_exact_for_integers(dtype, sizes, d):
    rows = sum(sizes)
    x, dy = ints((rows, d), dtype, 1), ints((rows, d), dtype, 2)
    zero, one = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    _, dw, db = L.layer_norm_backward(dy.cuda(), x.cuda(), None, zero, one, offsets_of(sizes))
    for g, (a, b) in enumerate(spans(sizes)):
        assert torch.equal(dw[g].cpu(), (x[a:b].double() * dy[a:b].double()).sum(0).float())
        assert torch.equal(db[g].cpu(), dy[a:b].double().sum(0).float())


def test_layer_norm_gradients_against_differences():
    """Central differences of sum(dy * y) in 64 bits, along random directions."""
    rows, d, eps, h = 6, 40, 1e-5, 1e-5
    x, dy, w, b = normals((rows, d), F32, 1), normals((rows, d), F32, 2), 1 + normals((d,), F32, 3, 0.2), normals((d,), F32, 4)
    _, mean, rstd = L.layer_norm(x.cuda(), w.cuda(), b.cuda(), eps)
    dx, dw, db = (t.cpu().double() for t in L.layer_norm_backward(dy.cuda(), x.cuda(), w.cuda(), mean, rstd))
    f = lambda xx, ww, bb: float((norm64(xx, ww, bb, eps)[0] * dy.double()).sum())
    for seed in range(4):
        ex, ew, eb = (torch.randn(s, generator=gen(seed), dtype=torch.float64) for s in ((rows, d), (d,), (d,)))
        for diff, grad in ((f(x.double() + h * ex, w, b) - f(x.double() - h * ex, w, b), (ex * dx).sum()),
                           (f(x, w.double() + h * ew, b) - f(x, w.double() - h * ew, b), (ew * dw).sum()),
                           (f(x, w, b.double() + h * eb) - f(x, w, b.double() - h * eb), (eb * db).sum())):
            # the differences are good to h^2 times third derivatives and to 1e-16 |f| / h; the gradients to some 50 u of their terms
            assert abs(diff / (2 * h) - float(grad)) < 1e-4


# ---------------------------------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------------------------------
def draws(count, seed, step, layer, first):
    e = np.arange(count, dtype=np.uint64) + np.uint64(first)
    block = e >> np.uint64(3)
    words = np.stack(O.philox4x32_10((block & np.uint64(0xFFFFFFFF)).astype(np.uint32), (block >> np.uint64(32)).astype(np.uint32), np.uint32(step),
                                     np.uint32(layer + 1), seed & 0xFFFFFFFF, seed >> 32))
    word = words[((e & np.uint64(7)) >> np.uint64(1)).astype(np.int64), np.arange(count)].astype(np.uint32)
    return np.where(e & np.uint64(1), word >> 16, word & 0xFFFF).astype(np.int64)


def dropped(x, residual, p, seed, step=0, layer=0, first=0):
    cut = math.floor(p * 65536 + 0.5)
    keep = torch.from_numpy(draws(x.numel(), seed, step, layer, first) >= cut).view(x.shape)
    scale = torch.tensor(65536.0 / (65536 - cut) if cut < 65536 else 0.0, dtype=F32)
    out = torch.where(keep, x.float() * scale, 0.0)
    return (out if residual is None else out + residual.float()).to(x.dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d,pad,lead,first", [(1, 1, 0, 0, 0), (1, 1, 0, 0, 5), (3, 7, 0, 0, 0), (5, 64, 0, 0, 8), (9, 64, 8, 0, 0), (7, 100, 3, 1, 3), (33, 1000, 0, 0, 0),
                                                   (4, 5003, 0, 0, (1 << 35) - 2001), (2, 4096, 0, 0, (1 << 35) - 4096), (300, 520, 0, 2, 16), (1, 70000, 0, 0, 1)])
def test_dropout_draws_what_it_says(dtype, rows, d, pad, lead, first):
    x, res = normals((rows, d), dtype, 1), normals((rows, d), dtype, 2)
    x[0, 0] = float("nan")
    seed = 0xFEDCBA9876543210 + rows
    for p, step, layer in ((0.1, 0, 0), (0.5, 7, 3), (0.25, (1 << 32) - 1, (1 << 32) - 2)):
        for residual in (None, res):
            out = blank((rows, d), dtype, pad, lead)
            L.dropout(gpu(x, pad, lead), p, seed, step=step, layer=layer, first=first, out=out,
                      residual=None if residual is None else gpu(residual, pad, lead))
            want = dropped(x, residual, p, seed, step, layer, first)
            assert torch.equal(torch.nan_to_num(out.cpu().float(), 55.0), torch.nan_to_num(want.float(), 55.0)), (p, residual is None)
            assert untouched(out)


def test_dropout_of_nothing_and_of_everything():
    x = normals((40, 72), F32, 1).cuda()
    assert torch.equal(L.dropout(x, 0.0, 1), x) and torch.equal(L.dropout(x, 0.25 / 65536, 1), x)
    bad = torch.where(x > 0, float("inf"), float("nan"))
    assert (L.dropout(bad, 1.0, 1) == 0).all() and torch.equal(L.dropout(bad, 1.0, 1, residual=x), x)
    assert L.dropout(torch.empty((0, 8), device="cuda"), 0.5, 1).shape == (0, 8)
    y = x.clone()
    assert torch.equal(L.dropout(y, 0.3, 5, residual=x, out=y), L.dropout(x, 0.3, 5, residual=x))      # in place
    y = x.clone()
    assert torch.equal(L.dropout(x, 0.3, 5, residual=y, out=y), L.dropout(x, 0.3, 5, residual=x))


def test_dropout_of_pieces_is_that_of_the_batch_and_of_a_device_step_that_of_its_number():
    x = normals((64, 1000), BF16, 1).cuda()
    whole = L.dropout(x, 0.2, 9, step=5, layer=2)
    for cut in (1, 13, 40):
        parts = [L.dropout(x[a:b], 0.2, 9, step=5, layer=2, first=a * 1000) for a, b in ((0, cut), (cut, 64))]
        assert torch.equal(torch.cat(parts), whole)
    step = torch.tensor([5], device="cuda")
    assert torch.equal(L.dropout(x, 0.2, 9, step=step, layer=2), whole)
    assert not torch.equal(L.dropout(x, 0.2, 9, step=6, layer=2), whole)
    # the backward pass: kept where the forward pass kept
    ones = torch.ones_like(x)
    assert torch.equal(L.dropout(ones, 0.2, 9, step=5, layer=2) != 0, whole != 0)


# ---------------------------------------------------------------------------------------------------
# preference loss
# ---------------------------------------------------------------------------------------------------
def preference64(logits, targets, sizes, first, ref, beta, s):
    x = logits.double()
    tokens, v = x.shape
    counts = (targets >= 0) & (targets < v)
    for a, b in ((0, first), (first + sum(sizes), tokens)):
        counts[a:b] = False
    lse, logp = torch.zeros(tokens).double(), torch.zeros(tokens).double()
    lse[counts] = torch.logsumexp(x[counts], 1)
    logp[counts] = x[counts, targets[counts]] - lse[counts]
    ratio = torch.where(counts, logp - (0 if ref is None else ref.double()), 0.0)
    sums = torch.stack([ratio[a:b].sum() for a, b in spans(sizes, first)])
    margin = sums[0::2] - sums[1::2]
    z = beta * margin
    loss = (1 - s) * torch.logaddexp(-z, torch.zeros_like(z)) + s * torch.logaddexp(z, torch.zeros_like(z))
    slope = beta * (s * torch.sigmoid(z) - (1 - s) * torch.sigmoid(-z))
    return counts, lse, logp, margin, loss, slope


PREFERENCES = [
    # sizes of sequences, v, elements between rows, smoothing
    ([1, 1], 1, 0, 0.0), ([1, 2], 5, 0, 0.1), ([3, 0, 0, 4], 33, 0, 0.0), ([9, 40, 17, 1, 0, 0], 1000, 8, 0.0), ([5, 6, 7, 2], 1001, 3, 0.3), ([70, 30], 4096, 0, 0.0),
    ([2, 3], 20000, 0, 0.0), ([300, 290], 250, 2, 1.0),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", PREFERENCES, ids=lambda c: "%d-%d+%d" % (len(c[0]), c[1], c[2]))
def test_preference_loss_and_its_gradient(dtype, case):
    sizes, v, pad, s = case
    first, tokens = (2, 2 + sum(sizes) + 3) if pad else (0, sum(sizes))
    logits = normals((tokens, v), dtype, 3, 3.0)
    targets = torch.randint(0, v, (tokens,), generator=gen(4))
    targets[torch.rand(tokens, generator=gen(5)) < 0.25] = -100
    if tokens > 20:
        targets[10], targets[11] = v, 1 << 40                  # outside: do not count
        logits[targets < 0] = float("nan")                     # ... and their rows do not matter
    ref, beta = normals((tokens,), F32, 6) - math.log(v), 0.3
    pairs, dloss = len(sizes) // 2, normals((len(sizes) // 2,), F32, 7)
    lg, off, tg = gpu(logits, pad), offsets_of(sizes, first), targets.cuda()
    loss, margin, logp, lse = L.preference_loss(lg, tg, off, ref.cuda(), beta, s)
    counts, lse64, logp64, margin64, loss64, slope64 = preference64(logits, targets, sizes, first, ref, beta, s)
    inside = torch.zeros(tokens, dtype=torch.bool)
    inside[first:first + sum(sizes)] = True
    # exp is good to 2^-22 plus what its argument x - top lost, at most 2 u times its size, which weighs x - top by its own
    # probability (below 12 here); a lane adds v / 64 terms at most
    e = (v / 64 + 20) * U + 4 * U + 2 * U * 12
    el = e + U * lse64.abs()
    ep = e + U * logp64.abs() + U * (lse64.abs() + logp64.abs())
    assert (lse.cpu().double() - lse64).abs()[inside].le(el[inside]).all() and (logp.cpu().double() - logp64).abs()[inside].le(ep[inside]).all()
    em = torch.stack([torch.where(counts, ep, 0.0)[a:b].sum() for a, b in spans(sizes, first)])
    em = em[0::2] + em[1::2] + U * margin64.abs()
    assert (margin.cpu().double() - margin64).abs().le(em).all()
    assert (loss.cpu().double() - loss64).abs().le(beta * em + 2 * U * loss64 + 1e-30).all()
    out = blank((tokens, v), dtype, pad)
    L.preference_loss_backward(dloss.cuda(), lg, tg, off, margin, lse, beta, s, out=out)
    got = out.cpu().double()
    f = torch.zeros(tokens).double()
    ef = torch.zeros(tokens).double()
    for i, (a, b) in enumerate(spans(sizes, first)):
        f[a:b] = (1 - 2 * (i % 2)) * slope64[i // 2] * dloss[i // 2].double()
        ef[a:b] = beta ** 2 * em[i // 2] / 4 * dloss[i // 2].double().abs() + 2 * U * f[a].abs() if b > a else 0
    onehot = torch.zeros(tokens, v).double()
    onehot[counts, targets[counts]] = 1.0
    prob = torch.where(counts[:, None], torch.exp(logits.double() - lse64[:, None]), 0.0)
    want = f[:, None] * (onehot - prob)
    ex = prob * (el[:, None] + 4 * U + 2 * U * (logits.double() - lse64[:, None]).abs())
    bound = f.abs()[:, None] * (ex + U * (onehot - prob).abs()) + ef[:, None] * (onehot - prob).abs() + U * want.abs()
    bound = bound + HALF[dtype] * (want.abs() + bound) + TINY[dtype]
    want, bound = torch.where(counts[:, None], want, 0.0), torch.where(counts[:, None], bound, 0.0)
    assert (got - want).abs()[inside].le(bound[inside] + 1e-40).all(), ((got - want).abs() / (bound + 1e-30))[inside].max()
    assert (got[~inside] == 77).all() and untouched(out)


def test_preference_gradient_against_differences():
    sizes, v, beta, s, h = [4, 3, 2, 5], 30, 0.4, 0.1, 1e-5
    tokens = sum(sizes)
    logits, targets, ref = normals((tokens, v), F32, 1, 2.0), torch.randint(0, v, (tokens,), generator=gen(2)), normals((tokens,), F32, 3) - 3
    targets[2] = -1
    dloss, off = torch.tensor([0.7, -1.3]), offsets_of(sizes)
    loss, margin, logp, lse = L.preference_loss(logits.cuda(), targets.cuda(), off, ref.cuda(), beta, s)
    grad = L.preference_loss_backward(dloss.cuda(), logits.cuda(), targets.cuda(), off, margin, lse, beta, s).cpu().double()
    f = lambda x: float((preference64(x, targets, sizes, 0, ref, beta, s)[4] * dloss.double()).sum())
    for seed in range(4):
        e = torch.randn((tokens, v), generator=gen(seed), dtype=torch.float64)
        assert abs((f(logits.double() + h * e) - f(logits.double() - h * e)) / (2 * h) - float((e * grad).sum())) < 1e-5


def test_preference_loss_of_extreme_logits():
    """Columns masked by -inf or the type's lowest value, a target among them, margins far out, and no reference."""
    for dtype in TYPES:
        v, off = 300, offsets_of([2, 1, 1, 1])
        x = normals((5, v), dtype, 1)
        x[:, 100:] = -float("inf")
        x[1, 100:] = torch.finfo(dtype).min
        x[2, 5] = 60000.0                                      # everything on one column
        t = torch.tensor([3, 4, 5, 7, 200])                     # the last one's target is masked out: logp is -inf
        loss, margin, logp, lse = L.preference_loss(x.cuda(), t.cuda(), off, None, 1.0)
        want = x[:, :100].double().log_softmax(1)
        assert torch.isfinite(lse).all() and (logp[:4].cpu().double() - want[[0, 1, 2, 3], t[:4]]).abs().max() < 1e-5 and logp[4] == -float("inf")
        assert margin[1] == float("inf") and loss[1] == 0.0
        grad = L.preference_loss_backward(torch.ones(2, device="cuda"), x.cuda(), t.cuda(), off, margin, lse, 1.0)
        assert torch.isfinite(grad).all() and not grad[3:].any() and not grad[:, 100:].any()
        worse = x.clone()
        worse[0] = -float("inf")                               # nothing is left of this row: no number, but only there
        loss2, _, _, lse2 = L.preference_loss(worse.cuda(), t.cuda(), off, None, 1.0)
        assert torch.isnan(loss2[0]) and loss2[1] == loss[1] and torch.equal(lse2[1:], lse[1:])


def test_preference_loss_in_place_and_of_nothing():
    logits, off = normals((9, 130), BF16, 1).cuda(), offsets_of([4, 5])
    t = torch.arange(9, device="cuda")
    loss, margin, logp, lse = L.preference_loss(logits, t, off)
    d = torch.ones(1, device="cuda")
    want = L.preference_loss_backward(d, logits, t, off, margin, lse)
    assert torch.equal(L.preference_loss_backward(d, logits, t, off, margin, lse, out=logits), want)
    none = torch.empty((0, 130), dtype=BF16, device="cuda")
    loss, margin, logp, lse = L.preference_loss(none, t[:0], offsets_of([0, 0]))
    assert margin.item() == 0 and abs(loss.item() - math.log(2)) < 1e-7 and logp.shape == (0,)
    assert L.preference_loss_backward(d, none, t[:0], offsets_of([0, 0]), margin, lse).shape == (0, 130)
    assert L.preference_loss(none, t[:0], offsets_of([]))[0].shape == (0,)


# ---------------------------------------------------------------------------------------------------
# all of them
# ---------------------------------------------------------------------------------------------------
def every_call(dtype, seed=1):
    """(name, call, outputs) of each operator on tensors of its own; a call writes the same outputs whenever it is made."""
    rows, n, k, sizes = 700, 136, 264, [200, 0, 333, 167]
    off = offsets_of(sizes)
    x, dy, w = normals((rows, k), dtype, seed).cuda(), normals((rows, n), dtype, seed + 1).cuda(), normals((4, n, k), dtype, seed + 2).cuda()
    y, dx, dw = torch.empty((rows, n), dtype=dtype, device="cuda"), torch.empty_like(x), torch.empty((4, n, k), device="cuda")
    nw = normals((k,), F32, 4).cuda()
    ny, (nm, nr) = torch.empty_like(x), torch.randn((2, rows), generator=gen(3)).cuda()
    ndy, ndx, ndw, ndb = normals((rows, k), dtype, 5).cuda(), torch.empty_like(x), torch.empty((4, k), device="cuda"), torch.empty((4, k), device="cuda")
    drop = torch.empty_like(x)
    targets = torch.randint(0, k, (rows,), generator=gen(6)).cuda()
    out, saved = torch.empty_like(x), {}

    def loss():
        saved["loss"] = L.preference_loss(x, targets, off, None, 0.2)
        return saved["loss"]

    def grad():
        _, margin, _, lse = L.preference_loss(x, targets, off, None, 0.2)
        return [L.preference_loss_backward(torch.ones(2, device="cuda"), x, targets, off, margin, lse, 0.2, out=out)]
    return {
        "forward": lambda: [L.group_matmul(x, w, off, out=y)], "dx": lambda: [L.group_matmul_dx(dy, w, off, out=dx)],
        "dw": lambda: [L.group_matmul_dw(dy, x, off, out=dw)], "norm": lambda: list(L.layer_norm(x, nw, None, out=ny)),
        "norm back": lambda: list(L.layer_norm_backward(ndy, x, nw, nm, nr, off, ndx, ndw, ndb)),
        "dropout": lambda: [L.dropout(x, 0.1, 5, step=2, residual=ndy, out=drop)], "loss": lambda: list(loss()), "loss back": grad,
    }


@pytest.mark.parametrize("dtype", TYPES)
def test_the_same_call_gives_the_same_bits_on_any_stream(dtype):
    calls = every_call(dtype)
    want = {name: [t.clone() for t in call()] for name, call in calls.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = {name: [t.clone() for t in call()] for name, call in calls.items()}
    side.synchronize()
    for name in calls:
        assert all(torch.equal(a, b) for a, b in zip(want[name], got[name])), name


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_two_captured_graphs_replayed_between_eager_calls(dtype):
    first, second = every_call(dtype, 1), every_call(dtype, 50)
    want = [{name: [t.clone() for t in call()] for name, call in calls.items()} for calls in (first, second)]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for calls in (first, second):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append({name: call() for name, call in calls.items()})
        graphs.append(g)
    for replay in range(3):
        for i in (0, 1):
            for o in outs[i].values():
                for t in o:
                    t.fill_(0)
            graphs[i].replay()
            torch.cuda.synchronize()
            for name in want[i]:
                assert all(torch.equal(a, b) for a, b in zip(want[i][name], outs[i][name])), (replay, i, name)
            eager = {name: [t.clone() for t in call()] for name, call in (second if i == 0 else first).items()}
            assert all(torch.equal(a, b) for name in eager for a, b in zip(want[1 - i][name], eager[name]))


def test_a_captured_dropout_draws_anew_from_its_device_step():
    x, step = normals((20, 72), F32, 1).cuda(), torch.zeros(1, dtype=torch.int64, device="cuda")
    out = torch.empty_like(x)
    L.dropout(x, 0.5, 3, step=step, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.dropout(x, 0.5, 3, step=step, out=out)
        step.add_(1)
    step.fill_(4)
    for t in (4, 5, 6):
        g.replay()
        assert torch.equal(out.cpu(), dropped(x.cpu(), None, 0.5, 3, step=t))


def test_rows_more_than_four_gigabytes_apart():
    """Row numbers times strides pass 2^32 elements."""
    apart, rows, d = (1 << 27) + 64, 33, 64
    base = torch.empty(rows * apart, dtype=BF16, device="cuda")
    far = torch.as_strided(base, (rows, d), (apart, 1))
    near = normals((rows, d), BF16, 1).cuda()
    far.copy_(near)
    out = torch.as_strided(base, (rows, d), (apart, 1), 4096)
    off, w = offsets_of([20, 13]), normals((2, d, d), BF16, 2).cuda()
    mean, rstd = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    t = torch.arange(rows, device="cuda")
    _, margin, _, lse = L.preference_loss(near, t, off)
    one = torch.ones(1, device="cuda")
    for name, call in {
        "forward": lambda x, o: L.group_matmul(x, w, off, out=o), "dx": lambda x, o: L.group_matmul_dx(x, w, off, out=o),
        "norm": lambda x, o: L.layer_norm(x, out=o)[0], "norm back": lambda x, o: L.layer_norm_backward(x, x, None, mean, rstd, off, dx=o)[0],
        "dropout": lambda x, o: L.dropout(x, 0.3, 1, residual=x, out=o),
        "loss back": lambda x, o: L.preference_loss_backward(one, x, t, off, margin, lse, out=o),
    }.items():
        out.zero_()
        assert torch.equal(call(far, out), call(near, None)), name
    assert torch.equal(L.group_matmul_dw(far, far, off), L.group_matmul_dw(near, near, off))
    assert all(torch.equal(a, b) for a, b in zip(L.preference_loss(far, t, off), L.preference_loss(near, t, off)))
    assert all(torch.equal(a, b) for a, b in zip(L.layer_norm_backward(far, far, None, mean, rstd, off)[1:], L.layer_norm_backward(near, near, None, mean, rstd, off)[1:]))


def test_a_models_gradients_by_worker_and_the_engine_that_takes_them():
    """Every operator in its place: each worker's gradient of a norm, a residual block with dropout and a head under the preference
    loss, against automatic differentiation of that worker's own objective in 64 bits; then the engine's steps on them."""
    from paper_2211_00188_amd import experiments as X
    from paper_2211_00188_amd import workloads as W
    wl = W.preference(n=4, pairs=10, width=16, vocab=33, length=14, seed=5)
    model, step = X.PreferenceModel(wl, seed=3), 6
    ext = torch.full((wl.n, wl.d), float("nan"), device="cuda")
    loss = model.gradients(torch.from_numpy(wl.x0).cuda(), step, ext).cpu().double()
    keep = torch.from_numpy(draws(wl.features.size, 3, step, 0, 0) >= math.floor(wl.dropout * 65536 + 0.5)).view(wl.features.shape)
    scale = 65536 / (65536 - math.floor(wl.dropout * 65536 + 0.5))
    f, t, rows = torch.from_numpy(wl.features).double(), torch.from_numpy(wl.targets), wl.worker_rows()
    for i in range(wl.n):
        x = torch.from_numpy(wl.x0).double().requires_grad_()
        w = wl.parts(x)
        z = norm64(f, w["norm_weight"], w["norm_bias"], 1e-5)[0]
        u = z @ w["hidden"].t()
        assert u.abs().min() > 1e-5                             # (no element so near the kink that fp32 might pass it)
        logits = (u.clamp(min=0) * keep * scale + z) @ w["head"].t()
        lp = logits.log_softmax(1)
        counts = t >= 0
        ratio = torch.where(counts, lp.gather(1, t.clamp(min=0)[:, None])[:, 0] - torch.from_numpy(wl.ref).double(), 0.0)
        a, b = wl.worker_pairs[i:i + 2]
        s = wl.sequences
        margin = torch.stack([ratio[s[2 * p]:s[2 * p + 1]].sum() - ratio[s[2 * p + 1]:s[2 * p + 2]].sum() for p in range(a, b)])
        each = torch.nn.functional.softplus(-wl.beta * margin)
        assert (loss[a:b] - each.detach()).abs().max() < 1e-5
        each.mean().backward()
        for name, got in wl.parts(ext[i].cpu().double()).items():
            want = wl.parts(x.grad)[name]
            # a dozen operations one after the other, sums of some 40 to 140 terms in each: 12 * 140 u = 1e-4 of the largest
            assert (got - want).abs().max() <= 1e-4 * want.abs().max(), (i, name)
    levels, zeta = X.method_levels("adacgd", wl.d)
    x0 = torch.from_numpy(wl.x0).cuda()
    eng = E.AdaCGD(n=wl.n, d=wl.d, gamma=0.05, worker_levels=levels, zeta_worker=zeta, grad_mode=E.GRAD_EXTERNAL, x0=x0, grad0=ext)
    eng.step(ext)
    assert np.array_equal(eng.state(E.F_PREV_GRAD), ext.cpu().numpy())
    out = torch.empty(wl.d, device="cuda")
    assert np.array_equal(eng.state_into(E.F_X, out).cpu().numpy(), eng.state(E.F_X))
    eng.close()
    steps, bits, gn, mean_loss = X.run_preference(wl, "adacgd", 0.05, 2e4, max_steps=6)
    assert len(steps) > 2 and np.isfinite(gn).all() and np.isfinite(mean_loss).all() and (np.diff(bits) >= 0).all()


def test_the_binding_refuses_what_does_not_fit():
    x, w, off = torch.zeros((8, 16), device="cuda"), torch.zeros((2, 4, 16), device="cuda"), offsets_of([3, 5])
    for call in (lambda: L.group_matmul(x, w[:, :, :8], off), lambda: L.group_matmul(x, w[:1], off), lambda: L.group_matmul(x.t(), w, off),
                 lambda: L.group_matmul(x, w, off.cpu()), lambda: L.group_matmul(x, w, off.int()), lambda: L.group_matmul(x, w, off[::2]),
                 lambda: L.group_matmul(x, w, off, out=torch.zeros((8, 5), device="cuda")), lambda: L.group_matmul_dw(x, x[:7], off),
                 lambda: L.group_matmul_dw(x, x, off, out=torch.zeros((16, 16), device="cuda").expand(2, 16, 16)),
                 lambda: L.layer_norm(x, weight=torch.zeros(15, device="cuda")), lambda: L.layer_norm(x, weight=torch.zeros(16, device="cuda", dtype=BF16)),
                 lambda: L.layer_norm_backward(x, x, None, x[:, 0], x[0], off), lambda: L.dropout(x, 0.5, -1), lambda: L.dropout(x, 0.5, 1, step=1 << 32),
                 lambda: L.dropout(x, 1.5, 1), lambda: L.dropout(x, 0.5, 1, residual=x[:4]), lambda: L.preference_loss(x, off, off),
                 lambda: L.preference_loss(x, torch.zeros(8, dtype=torch.int64, device="cuda"), offsets_of([3])),
                 lambda: L.preference_loss(x, torch.zeros(8, dtype=torch.int32, device="cuda"), off)):
        with pytest.raises((ValueError, E.AdaCGDError)):
            call()
    with pytest.raises(TypeError):
        L.layer_norm(x.double())
    with pytest.raises(E.AdaCGDError):
        L.group_matmul(x, w.to(BF16), off)


def test_a_captured_product_of_large_tiles():
    sizes = [5000, 0, 7041, 3, 500]
    off, x, w = offsets_of(sizes), normals((sum(sizes), 264), BF16, 1).cuda(), normals((5, 1032, 264), BF16, 2).cuda()
    y, dw = torch.empty((sum(sizes), 1032), dtype=BF16, device="cuda"), torch.empty((5, 1032, 264), device="cuda")
    want = L.group_matmul(x, w, off), L.group_matmul_dw(L.group_matmul(x, w, off), x, off)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.group_matmul(x, w, off, out=y)
        L.group_matmul_dw(y, x, off, out=dw)
    for _ in range(3):
        y.zero_(), dw.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(dw, want[1])
        assert torch.equal(L.group_matmul(x, w, off), want[0])


@pytest.mark.parametrize("bad", [[0, 12000, -3, 9000, 1 << 40], [1 << 62, 0, 5000, 4000, 12544], [12544] * 5])
def test_offsets_that_break_the_rule_stay_inside_large_tiles(bad):
    off, rows = torch.tensor(bad, device="cuda"), 12544
    x, w, y, dw = blank((rows, 264), BF16, 8), gpu(normals((4, 1032, 264), BF16, 1), 8), blank((rows, 1032), BF16, 8), blank((4, 1032, 264), F32, 8)
    L.group_matmul(x, w, off, out=y)
    L.group_matmul_dx(y, w, off, out=x)
    L.group_matmul_dw(y, x, off, out=dw)
    torch.cuda.synchronize()
    assert untouched(x) and untouched(y) and untouched(dw)


@pytest.mark.parametrize("bad", [[0, 900, 20, 60], [-5, 30, 40, 1 << 62], [-(1 << 62), 5, 3, 60], [60, 40, 20, 0], [100, 100, 100, 100]])
def test_offsets_that_break_the_rule_stay_inside(bad):
    """They are clamped where they are read: results are unspecified, everything around the matrices keeps its values."""
    off, rows = torch.tensor(bad, device="cuda"), 60
    x, w, y, dw = blank((rows, 40), F32, 8), gpu(normals((3, 24, 40), F32, 1), 8), blank((rows, 24), F32, 8), blank((3, 24, 40), F32, 8)
    L.group_matmul(x, w, off, out=y)
    L.group_matmul_dw(y, x, off, out=dw)
    dx, nw, nb = blank((rows, 40), F32, 8), blank((3, 40), F32, 8), blank((3, 40), F32, 8)
    L.layer_norm_backward(x, x, None, torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda"), off, dx, nw, nb)
    o2 = torch.cat([off, off[-1:]])
    t = torch.zeros(rows, dtype=torch.int64, device="cuda")
    _, margin, _, lse = L.preference_loss(x, t, o2)
    L.preference_loss_backward(torch.ones(2, device="cuda"), x, t, o2, margin, lse, out=dx)
    torch.cuda.synchronize()
    assert all(untouched(v) for v in (x, y, dw, dx, nw, nb))


# ---------------------------------------------------------------------------------------------------
# logits far from zero
# ---------------------------------------------------------------------------------------------------
def gradient_and_its_bound(logits, targets, off, sizes, beta=0.4, s=0.1, out=None):
    """The kernel's gradient, the one in 64 bits at the margin that the kernel is given, and a bound on their difference without a term in |lse|."""
    tokens, v = logits.shape
    dtype, dloss = logits.dtype, 0.5 + normals((len(sizes) // 2,), F32, 77).abs()
    lg, tg = logits.cuda(), targets.cuda()
    _, margin, _, lse = L.preference_loss(lg, tg, off, None, beta, s)
    got = L.preference_loss_backward(dloss.cuda(), lg, tg, off, margin, lse, beta, s, out=lg if out == "in place" else None).cpu().double()
    z = beta * margin.cpu().double()
    slope = beta * (s * torch.sigmoid(z) - (1 - s) * torch.sigmoid(-z)) * dloss.double()
    f = torch.cat([torch.full((m,), 1.0 - 2 * (i % 2)).double() * slope[i // 2] for i, m in enumerate(sizes)])[:, None]
    p = torch.softmax(logits.double(), 1)
    onehot = torch.zeros(tokens, v).double()
    onehot[torch.arange(tokens), targets] = 1.0
    want = f * (onehot - p)
    # exp(x - l) is off by 4 u and by 2 u |x - l| (its argument, rounded twice), the sum of these by their weighted mean and by its
    # additions, (v / 64 + 20) u; a reciprocal and a product of them, the difference, and the product with f, rounded too, take one u each
    away = (logits.double() - lse.cpu().double()[:, None]).abs()
    each = 4 * U + 2 * U * away
    ep = p * (each + (p * each).sum(1, keepdim=True) + (v / 64 + 20) * U + 2 * U)
    bound = f.abs() * (ep + U * (onehot - p).abs()) + 2 * U * want.abs()
    return got, want, bound + HALF[dtype] * (want.abs() + bound) + TINY[dtype] + 1e-38


@pytest.mark.parametrize("offset", [0.0, 100.0, 1000.0, -1e4, 1e6])
@pytest.mark.parametrize("dtype,sizes,v", [(F32, [9, 40, 17, 1], 1000), (F32, [2, 1], 20000), (F32, [600, 700], 300), (F16, [9, 40, 17, 1], 1000), (BF16, [9, 40], 9001)],
                         ids=lambda t: str(t).replace("torch.", ""))
def test_preference_gradient_does_not_depend_on_the_logits_offset(dtype, sizes, v, offset):
    logits = (torch.randn((sum(sizes), v), generator=gen(1)) * 2 + min(offset, 6e4 if dtype == F16 else offset)).to(dtype)
    targets = torch.randint(0, v, (sum(sizes),), generator=gen(2))
    for out in (None, "in place"):
        got, want, bound = gradient_and_its_bound(logits, targets, offsets_of(sizes), sizes, out=out)
        assert (got - want).abs().le(bound).all(), (out, ((got - want).abs() / bound).max())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("v", [300, 20000])
def test_preference_gradient_of_rows_that_are_masked_with_the_lowest_value_throughout(dtype, v):
    """All of a row's elements alike, far below zero: each has probability 1 / v."""
    logits = torch.full((5, v), torch.finfo(dtype).min, dtype=dtype)
    logits[3], logits[4] = torch.finfo(dtype).max, 1000.0
    targets, sizes = torch.tensor([3, 4, 5, 7, 8]), [2, 1, 1, 1]
    got, want, bound = gradient_and_its_bound(logits, targets, offsets_of(sizes), sizes)
    assert (got - want).abs().le(bound).all(), ((got - want).abs() / bound).max()
    again, _, _ = gradient_and_its_bound(logits, targets, offsets_of(sizes), sizes, out="in place")
    assert torch.equal(again, got)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [3, 7, 64, 100, 300, 1001, 2056, 5003, 9000, 20001])
def test_layer_norm_gradients_of_rows_whose_mean_is_large_beside_their_spread(dtype, d):
    """Equal elements of 1e37, rstd = eps^-1/2: xhat is 0, though mean times rstd passes the largest number.  dx = rstd (c - mean(c))."""
    rows, rstd = 6, 316.25
    x = torch.full((rows, d), 1e37).to(dtype)
    dy, w, mean = normals((rows, d), dtype, 5), 1 + normals((d,), F32, 6, 0.1), x[:, 0].float()
    dx, dw, db = L.layer_norm_backward(dy.cuda(), x.cuda(), w.cuda(), mean.cuda(), torch.full((rows,), rstd, device="cuda"), offsets_of([4, 2]))
    c = dy.double() * w.double()
    want = rstd * (c - c.mean(1, keepdim=True))
    # a sum of d terms, d / 64 + 24 of them one after the other; each c rounds once, its mean twice more, dx twice
    bound = rstd * (2 * U * c.abs() + (d / 64 + 28) * U * c.abs().mean(1, keepdim=True)) + 2 * U * want.abs()
    bound = bound + HALF[dtype] * (want.abs() + bound)
    assert (dx.cpu().double() - want).abs().le(bound).all() and not dw.any() and torch.isfinite(db).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes", [[262144], [3, 262144, 0, 70]], ids=lambda s: str(len(s)))
def test_groups_sums_of_many_slices(dtype, sizes):
    """One row of a long group weighs 2^24, 383 far ones 1 each, which a sum in fp32 that goes from the one to the others would lose."""
    n = k = 64
    first = sizes[0] if len(sizes) > 1 else 0
    x, dy = torch.zeros((sum(sizes), k)), torch.zeros((sum(sizes), n))
    x[first], dy[first] = 4096.0, 4096.0
    far = first + 65536 + 512 * torch.arange(383)
    x[far], dy[far] = 1.0, 1.0
    dw = L.group_matmul_dw(dy.to(dtype).cuda(), x.to(dtype).cuda(), offsets_of(sizes)).cpu()
    want = torch.tensor(2 ** 24 + 383, dtype=torch.float64).float()
    assert (dw[1 if len(sizes) > 1 else 0] == want).all(), (dw.max() - want)
    # numbers: at most 4096 rows are added up in fp32, each addition a step, 2 u, of a partial sum, before the parts are joined
    x, dy = torch.randn((sum(sizes), k), generator=gen(1)).to(dtype).cuda(), torch.randn((sum(sizes), n), generator=gen(2)).to(dtype).cuda()
    dw = L.group_matmul_dw(dy, x, offsets_of(sizes))
    for g, (a, b) in enumerate(spans(sizes)):
        xd, dyd = x[a:b].double(), dy[a:b].double()
        want, size = (dyd.t().contiguous() @ xd), (dyd.abs().t().contiguous() @ xd.abs())
        assert (dw[g].double() - want).abs().le(2 * U * min(4096, b - a) * size + U * want.abs()).all(), g


# ---------------------------------------------------------------------------------------------------
# more rows than one launch has blocks: each row as in a call that has it in its first turn
# ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows,d,dtype", [(70001, 64, F32), (40001, 100, BF16), (20003, 500, F16), (9001, 1000, BF16), (4999, 1501, F32), (5001, 4000, BF16), (4100, 5003, F16),
                                          (4099, 8192, F32), (4100, 9000, BF16), (2500, 9000, F32), (2100, 20001, BF16)])
def test_layer_norm_of_many_rows_is_that_of_few(rows, d, dtype):
    x = torch.randn((rows, d), generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(dtype)
    w, b = 1 + normals((d,), F32, 1, 0.1).cuda(), normals((d,), F32, 2, 0.1).cuda()
    y, mean, rstd = L.layer_norm(x, w, b)
    dx, dw, db = L.layer_norm_backward(x, x, w, mean, rstd)
    for a in range(0, rows, 1999):
        part = slice(a, a + 1999)
        py, pm, pr = L.layer_norm(x[part], w, b)
        assert torch.equal(y[part], py) and torch.equal(mean[part], pm) and torch.equal(rstd[part], pr)
        assert torch.equal(dx[part], L.layer_norm_backward(x[part], x[part], w, pm, pr)[0])
    # dbias: the rows of a slice, 1/1024 of all or a few, are added up in fp32, the slices in fp64
    size = x.double().abs().sum(0)
    assert (db[0].double() - x.double().sum(0)).abs().le((rows / 1024 + 20) * 2 * U * size).all()
    same, _, _ = L.layer_norm(x, w, b, out=x)
    assert torch.equal(same, y)


@pytest.mark.parametrize("rows,d,pad", [(17001, 1003, 0), (70001, 24, 3), (33000, 9, 1), (3, 6000001, 5)])      # (rows without gaps are one row)
def test_dropout_of_many_elements_is_that_of_few(rows, d, pad):
    x = gpu(torch.randn((rows, d), generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(BF16), pad)
    whole = L.dropout(x, 0.2, 9, step=5, residual=x, out=gpu(x, pad))
    if rows > 100:
        parts = [L.dropout(x[a:a + 7000], 0.2, 9, step=5, residual=x[a:a + 7000], first=a * d) for a in range(0, rows, 7000)]
        assert torch.equal(torch.cat(parts), whole)
    else:
        step = 4000000
        for r in range(rows):
            for a in range(0, d, step):
                piece = x[r:r + 1, a:a + step]
                assert torch.equal(L.dropout(piece, 0.2, 9, step=5, residual=piece, first=r * d + a), whole[r:r + 1, a:a + step])
    assert untouched(whole)


def test_preference_loss_of_many_tokens_is_that_of_few():
    tokens, v = 4500000, 9
    x = torch.randn((tokens, v), generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    t = torch.randint(-1, v, (tokens,), generator=torch.Generator("cuda").manual_seed(2), device="cuda")
    off = torch.arange(0, tokens + 1, 3, device="cuda")[:2 * (tokens // 6) + 1]
    loss, margin, logp, lse = L.preference_loss(x, t, off, None, 0.3)
    one = torch.ones(len(loss), device="cuda")
    grad = L.preference_loss_backward(one, x, t, off, margin, lse, 0.3)
    for a in (0, 2100000, tokens - 1200000):                       # (token rows; multiples of 6, 1200000 of them each)
        rows, pairs = slice(a, a + 1200000), slice(a // 6, a // 6 + 200000)
        o = off[:400001]
        part = L.preference_loss(x[rows], t[rows], o, None, 0.3)
        assert all(torch.equal(p, w) for p, w in zip(part, (loss[pairs], margin[pairs], logp[rows], lse[rows])))
        assert torch.equal(L.preference_loss_backward(one[pairs], x[rows], t[rows], o, part[1], part[3], 0.3), grad[rows])
    assert torch.equal(L.preference_loss_backward(one, x, t, off, margin, lse, 0.3, out=x), grad)


@pytest.mark.parametrize("dtype", TYPES)
def test_dropout_of_the_last_elements_that_64_bits_number(dtype):
    x, first = normals((3, 24), dtype, 1), (1 << 64) - 72
    assert torch.equal(L.dropout(x.cuda(), 0.3, 5, first=first).cpu(), dropped(x, None, 0.3, 5, first=first))
    with pytest.raises(E.AdaCGDError, match="2\\^64"):
        L.dropout(x.cuda(), 0.3, 5, first=first + 1)
