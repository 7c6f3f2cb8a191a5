"""The encoder operators (neuroute_ops.h) against plain implementations in 64
bits, at the sizes, strides and values where they can go wrong.

Tolerances. u is the largest relative error of a rounding to a type of 8, 11 or
24 significant bits (2^-8 bf16, 2^-11 fp16, 2^-24 fp32). A sum of c products
in fp32, in any order and rounded or truncated at every step, is off by at most
(c + 16) 2^-23 times the sum of the products' magnitudes. An activation's
Lipschitz constant is at most 1.13, and its fp32 evaluation adds at most 2^-20
of its argument's magnitude."""
import math

import numpy as np
import pytest

from gpu_util import need_cuda

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -149}
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
HALF = [F16, BF16]


@pytest.fixture(scope="module")
def ops():
    need_cuda()
    from paper_2608_15438_gb300 import ops as o

    yield o
    o.check(0)  # no bounded wait expired


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rows(g, m, n, dtype, pad=0, offset=0, scale=1.0):
    """[m x n] cut out of a wider buffer, its first value `offset` elements in."""
    buf = torch.randn(m * (n + pad) + offset, generator=g, device="cuda") * scale
    return buf.to(dtype)[offset:].view(m, n + pad)[:, :n]


def act64(z, act):
    if act == "relu":
        return torch.clamp(z, min=0), (z > 0).double()
    if act == "gelu":
        c = 0.5 * torch.erfc(-z / math.sqrt(2))
        return z * c, c + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    return z, torch.ones_like(z)


def held64(x):
    """What a checkpoint of x stands for, from the definition, on the CPU."""
    v = x.double().cpu().numpy()
    out = np.empty_like(v)
    for c in range(0, v.shape[1], 32):
        part = v[:, c:c + 32]
        top = np.abs(part).max(1)
        with np.errstate(divide="ignore", invalid="ignore"):
            e = np.floor(np.log2(np.where(top > 0, top, 1.0) / 127.5)) + 1  # least e with top < 127.5 2^e
        e = np.where(top < 127.5 * 2.0 ** (e - 1), e - 1, e)  # log2 off by one at a power of two
        e = np.where(top >= 127.5 * 2.0 ** e, e + 1, e)
        e = np.clip(np.where(top > 0, e, -126), -126, 121)
        step = 2.0 ** e[:, None]
        out[:, c:c + 32] = np.clip(np.rint(part / step), -127, 127) * step
    return torch.from_numpy(out).to(x.device)


def near(got, want, tol, what=""):
    """|got - want| <= tol elementwise, the type's largest finite value and infinities aside."""
    d = (got.double() - want).abs()
    bad = ~(d <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst by {float((d - tol).max())}"


def linear64(x, w, bias, act, residual):
    z = x.double() @ w.double().T
    s = x.double().abs() @ w.double().abs().T
    if bias is not None:
        z, s = z + bias.double(), s + bias.double().abs()
    y = act64(z, act)[0]
    if residual is not None:
        y = y + residual.double()
        s = s + residual.double().abs()
    return y, z, s


# one row to many, both sides of tiles of 32, 64, 128 and 256, odd widths
SHAPES = [(1, 1, 1), (1, 16, 16), (1, 1536, 512), (2, 7, 5), (3, 64, 1), (4, 128, 1000), (5, 129, 257),
          (8, 96, 384), (9, 64, 64), (16, 2048, 96), (17, 100, 33), (64, 512, 250), (127, 65, 129), (128, 64, 256),
          (129, 128, 255), (130, 200, 520), (257, 771, 1013), (300, 1536, 640), (1000, 96, 24), (2500, 40, 72)]


@pytest.mark.parametrize("i,shape", list(enumerate(SHAPES)))
@pytest.mark.parametrize("dtype", HALF)
def test_linear_forward(ops, i, shape, dtype):
    m, k, n = shape
    g = gen(i)
    act = ["none", "relu", "gelu", "silu"][i % 4]
    x, w = rows(g, m, k, dtype, pad=[0, 3, 8][i % 3]), rows(g, n, k, dtype, pad=[0, 8, 1][i % 3], scale=k ** -0.5)
    bias = [None, torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda").to(dtype)][i % 3]
    for residual in (None, rows(g, m, n, dtype, pad=i % 2)):
        for out in (None, F32):
            y, z = ops.linear(x, w, bias, act=act, residual=residual, save="z", out_dtype=out)
            y64, z64, s = linear64(x, w, bias, act, residual)
            acc = (k + 16) * 2.0 ** -23 * s
            assert y.dtype == (out or dtype) and z.dtype == dtype
            near(y, y64, U[y.dtype] * y64.abs() + 1.13 * acc + 2.0 ** -20 * z64.abs() + TINY[y.dtype], "y")
            near(z, z64, U[dtype] * z64.abs() + acc + TINY[dtype], "z")
            assert torch.equal(y, ops.linear(x, w, bias, act=act, residual=residual, out_dtype=out))
            # the pre-activations in 8 bits: within a step of the group's scale, and half a step of it exactly
            y8, c = ops.linear(x, w, bias, act=act, residual=residual, save="z8", out_dtype=out)
            assert torch.equal(y, y8)
            top = torch.nn.functional.pad(z64.abs() + acc, (0, -n % 32)).view(m, -1, 32).amax(2)
            step = torch.exp2(torch.floor(torch.log2(top / 127.5)) + 1).repeat_interleave(32, 1)[:, :n]
            near(ops.checkpoint8_read(c), z64, 0.5 * step * 1.001 + acc + 2 * TINY[dtype], "z8")
            assert torch.equal(c.codes[:, n:], torch.zeros_like(c.codes[:, n:]))


def grads64(dy, x, w, z, act):
    sl = act64(z.double(), act)[1] if z is not None else 1.0
    dz = dy.double() * sl
    return (dz, dz @ w.double(), dz.T @ x.double(), dz.sum(0),
            dz.abs() @ w.double().abs(), dz.abs().T @ x.double().abs(), dz.abs().sum(0))


@pytest.mark.parametrize("i,shape", list(enumerate(SHAPES)))
@pytest.mark.parametrize("dtype", HALF)
def test_linear_backward(ops, i, shape, dtype):
    m, k, n = shape
    g = gen(100 + i)
    act = ["gelu", "silu", "none", "relu"][i % 4]
    x, w = rows(g, m, k, dtype, pad=[0, 1, 8][i % 3]), rows(g, n, k, dtype, pad=[0, 8, 3][i % 3], scale=k ** -0.5)
    z = rows(g, m, n, dtype, pad=[0, 8, 1][i % 3]) if act != "none" else None
    u = U[dtype]
    for dy_dtype in (dtype, F32):
        dy = rows(g, m, n, dy_dtype, pad=[8, 0, 1][i % 3], scale=0.25)
        dz, dx64, dw64, db64, sx, sw, sb = grads64(dy, x, w, z, act)
        # dz is rounded to 16 bits for the products, its slope good to 2^-19
        e = u + 2.0 ** -19
        for bdt in (dtype, F32):
            dx, dw, db = ops.linear_backward(dy, x, w, z=z, act=act, bias_dtype=bdt)
            near(dx, dx64, u * dx64.abs() + (e + (n + 16) * 2.0 ** -23) * sx + (n + 1) * TINY[dtype], "dx")
            near(dw, dw64, u * dw64.abs() + (e + (m + 16) * 2.0 ** -23) * sw + (m * 4 + 1) * TINY[dtype], "dw")
            near(db, db64, U[bdt] * db64.abs() + (2.0 ** -19 + (m + 16) * 2.0 ** -23) * sb + TINY[bdt], "db")
            again = ops.linear_backward(dy, x, w, z=z, act=act, bias_dtype=bdt)
            assert all(torch.equal(a, b) for a, b in zip((dx, dw, db), again))
    part = ops.linear_backward(dy, x, w, z=z, act=act, need=(False, True, False))
    assert part[0] is None and part[2] is None and torch.equal(part[1], dw)
    part = ops.linear_backward(dy, x, w, z=z, act=act, need=(True, False, True))
    assert part[1] is None and torch.equal(part[0], dx) and torch.equal(part[2], db)


@pytest.mark.parametrize("shape", [(1, 33, 7), (40, 100, 96), (300, 257, 130), (513, 64, 320)])
@pytest.mark.parametrize("act,x_act", [("gelu", "none"), ("none", "gelu"), ("silu", "relu"), ("none", "none")])
def test_linear_backward_from_checkpoints(ops, shape, act, x_act):
    m, k, n = shape
    for dtype in HALF:
        g = gen(m)
        x, w, z = rows(g, m, k, dtype), rows(g, n, k, dtype, scale=k ** -0.5), rows(g, m, n, dtype)
        dy = rows(g, m, n, dtype, scale=0.25)
        x8, z8 = ops.checkpoint8(x), ops.checkpoint8(z) if act != "none" else None
        xv = act64(held64(x), x_act)[0]
        zv = held64(z) if act != "none" else None
        u = U[dtype]
        dx, dw, db = ops.linear_backward(dy, x8, w, z=z8, act=act, x_act=x_act)
        dz, dx64, dw64, db64, sx, sw, sb = grads64(dy, xv, w, zv, act)
        e = 2 * u + 2.0 ** -18  # dz, and x_act's value, in 16 bits
        near(dx, dx64, u * dx64.abs() + (e + (n + 16) * 2.0 ** -23) * sx + (n + 1) * TINY[dtype], "dx")
        near(dw, dw64, u * dw64.abs() + (e + (m + 16) * 2.0 ** -23) * sw + (m * 8 + 1) * TINY[dtype], "dw")
        near(db, db64, U[F32] * db64.abs() + (2.0 ** -18 + (m + 16) * 2.0 ** -23) * sb, "db")


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
def test_linear_gradients_against_differences(ops, act):
    """Central differences of sum(dy y) in 64 bits, y from the formula on the same 16-bit inputs."""
    g = gen(7)
    m, k, n = 6, 20, 12
    x, w, dy = rows(g, m, k, BF16), rows(g, n, k, BF16, scale=0.3), rows(g, m, n, BF16)
    b = torch.randn(n, generator=g, device="cuda")
    _, z = ops.linear(x, w, b, act=act, save="z")
    zc = z if act != "none" else None
    dx, dw, db = ops.linear_backward(dy, x, w, z=zc, act=act)

    def total(x_, w_, b_):
        return float((dy.double() * act64(x_ @ w_.T + b_, act)[0]).sum())

    X, W, B, h = x.double(), w.double(), b.double(), 1e-5
    for t, grad, which in ((X, dx, 0), (W, dw, 1), (B[None], db[None], 2)):
        for r, c in ((0, 0), (t.shape[0] - 1, t.shape[1] - 1), (t.shape[0] // 2, 3)):
            p = []
            for s in (h, -h):
                v = t.clone()
                v[r, c] += s
                a = [X, W, B]
                a[which] = v[0] if which == 2 else v
                p.append(total(*a))
            want = (p[0] - p[1]) / (2 * h)
            # z in 16 bits moves a slope by up to 2^-9 |z| times the second derivative (at most 1.2);
            # dz and the gradient are rounded to 16 bits: 2^-8 of the sum of magnitudes bounds the three
            mag = 1.0 + float((dy.double().abs() @ W.abs()).max() + (dy.double().abs().T @ X.abs()).max())
            if act == "relu":  # slopes from z's sign: exact unless the 16-bit z is zero
                assert (z != 0).all()
            assert abs(float(grad[r, c]) - want) <= 2.0 ** -7 * mag


NORMS = [(1, 1), (3, 2), (2, 7), (5, 31), (1, 32), (33, 33), (64, 96), (7, 128), (130, 387), (9, 1000), (700, 1536),
         (3, 4097), (40, 8192), (2, 20001)]


def norm_tol(x64, n):
    """How far fp32 statistics move xh: the mean by (n + 16) 2^-24 mean|x|, rstd by as much relatively."""
    sd = x64.var(1, unbiased=False, keepdim=True).add(1e-5).sqrt()
    return ((n + 16) * 2.0 ** -23 * (1 + x64.abs().mean(1, keepdim=True) / sd)) + 2.0 ** -20


@pytest.mark.parametrize("i,shape", list(enumerate(NORMS)))
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_layer_norm(ops, i, shape, dtype):
    m, n = shape
    g = gen(i)
    x = rows(g, m, n, dtype, pad=[0, 8, 1][i % 3], offset=i % 2) + 0.5
    if i % 2:
        x = torch.nn.functional.pad(x, (1, 2))[:, 1:1 + n]
    wdt = F32 if i % 2 else dtype
    w = (1 + 0.3 * torch.randn(n, generator=g, device="cuda")).to(wdt)
    b = torch.randn(n, generator=g, device="cuda").to(wdt)
    u = U[dtype]
    for from8 in (False, True):
        xin = ops.checkpoint8(x) if from8 else x
        x64 = held64(x) if from8 else x.double()
        mean64 = x64.mean(1)
        rstd64 = (x64.var(1, unbiased=False) + 1e-5).rsqrt()
        xh = (x64 - mean64[:, None]) * rstd64[:, None]
        t = norm_tol(x64, n)
        y, mean, rstd = ops.layer_norm(xin, w, b, save=True)
        y64 = xh * w.double() + b.double()
        near(y, y64, u * y64.abs() + t * (1 + xh.abs()) * w.double().abs() + 2.0 ** -22 * b.double().abs() + TINY[dtype], "y")
        near(mean, mean64, (n + 16) * 2.0 ** -23 * x64.abs().mean(1), "mean")
        near(rstd, rstd64, rstd64 * t[:, 0], "rstd")
        y1 = ops.layer_norm(xin)
        near(y1, xh, u * xh.abs() + t * (1 + xh.abs()) + TINY[dtype], "plain")
        # gradients
        dy = rows(g, m, n, dtype, pad=[1, 0, 8][i % 3])
        dres = rows(g, m, n, dtype) if i % 2 else None
        dx, dw, db = ops.layer_norm_backward(dy, xin, w, mean, rstd, residual_grad=dres)
        xh = (x64 - mean.double()[:, None]) * rstd.double()[:, None]
        gy = dy.double() * w.double()
        r = rstd.double()[:, None]
        dx64 = r * (gy - gy.mean(1, keepdim=True) - xh * (gy * xh).mean(1, keepdim=True))
        if dres is not None:
            dx64 = dx64 + dres.double()
        # three fp32 terms; the mean in xh costs 2^-22 of |x| and |mean| by cancellation
        exh = 2.0 ** -22 * (1 + (x64.abs() + mean.double().abs()[:, None]) * r)
        sums = (n + 32) * 2.0 ** -23
        mag = r * (gy.abs() + gy.abs().mean(1, keepdim=True) * (1 + sums / 2.0 ** -20)
                   + xh.abs() * (gy * xh).abs().mean(1, keepdim=True) * (1 + sums / 2.0 ** -20))
        lost = r * (exh * (gy * xh).abs().mean(1, keepdim=True) + xh.abs() * (gy.abs() * exh).mean(1, keepdim=True))
        near(dx, dx64, u * dx64.abs() + 2.0 ** -20 * mag + lost + TINY[dtype], "dx")
        dw64, db64 = (dy.double() * xh).sum(0), dy.double().sum(0)
        sw = (dy.double() * xh).abs().sum(0)
        uw = U[dw.dtype]
        assert dw.dtype == db.dtype == wdt
        near(dw, dw64, uw * dw64.abs() + (m + 32) * 2.0 ** -23 * sw + (dy.double().abs() * exh).sum(0) + TINY[wdt], "dw")
        near(db, db64, uw * db64.abs() + (m + 32) * 2.0 ** -23 * dy.double().abs().sum(0) + TINY[wdt], "db")
        again = ops.layer_norm_backward(dy, xin, w, mean, rstd, residual_grad=dres)
        assert all(torch.equal(a, b_) for a, b_ in zip((dx, dw, db), again))
        only = ops.layer_norm_backward(dy, xin, w, mean, rstd, residual_grad=dres, param_grads=False)
        assert only[1] is None and only[2] is None and torch.equal(only[0], dx)


@pytest.mark.parametrize("shape", [(1, 1), (9, 3), (2, 9), (7, 57), (8, 63), (100, 65), (5, 121), (3000, 131), (17, 249),
                                   (16, 250), (33, 255), (700, 387), (65, 1021), (4000, 1659), (6, 2041), (13, 2045),
                                   (300, 2500), (11, 4088), (9, 4089), (10, 4095), (21, 5095), (5, 8184), (4, 8187)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("pad,offset", [(0, 0), (1, 3), (8, 7)])
def test_layer_norm_rows_that_start_alike(ops, shape, dtype, pad, offset):
    """Matrices of one width, pitch and distance from an aligned address, as contiguous ones have."""
    from paper_2608_15438_gb300 import neuroute as nr

    m, n = shape
    g = gen(n + pad)
    x, dy, dres, out, dx = (rows(g, m, n, dtype, pad=pad, offset=offset) for _ in range(5))
    # what lies around the rows is not theirs, and stays
    around = []
    for t in (x, dy, dres, out, dx):
        whole = t.as_strided((t.untyped_storage().nbytes() // t.element_size(),), (1,), 0)
        kept = t.clone()
        whole.fill_(float("nan"))
        t.copy_(kept)
        around.append((whole, torch.isnan(whole)))
    w, b = 1 + 0.3 * torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
    u, x64 = U[dtype], x.double()
    mean64, rstd64 = x64.mean(1), (x64.var(1, unbiased=False) + 1e-5).rsqrt()
    xh = (x64 - mean64[:, None]) * rstd64[:, None]
    t = norm_tol(x64, n)
    ld, dt, f32 = n + pad, ops._DT[dtype], ops._DT[F32]
    mean, rstd = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    packed = ops._NORM.pack(m, n, dt, f32, 1e-5, x.data_ptr(), ld, 0, w.data_ptr(), b.data_ptr(), out.data_ptr(), ld,
                            mean.data_ptr(), rstd.data_ptr(), 0, 0, 0, 0, 0, 0, 0, 0)
    assert nr.lib().nr_layer_norm_forward(packed, 0, ops._stream(0)) == 0
    y64 = xh * w.double() + b.double()
    near(out, y64, u * y64.abs() + t * (1 + xh.abs()) * w.double().abs() + 2.0 ** -22 * b.double().abs() + TINY[dtype], "y")
    near(mean, mean64, (n + 16) * 2.0 ** -23 * x64.abs().mean(1), "mean")
    near(rstd, rstd64, rstd64 * t[:, 0], "rstd")
    for res in (None, dres):
        dw, db = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        packed = ops._NORM.pack(m, n, dt, f32, 0.0, x.data_ptr(), ld, 0, w.data_ptr(), 0, 0, 0, mean.data_ptr(),
                                rstd.data_ptr(), dy.data_ptr(), ld, 0 if res is None else res.data_ptr(), ld,
                                dx.data_ptr(), ld, dw.data_ptr(), db.data_ptr())
        need = nr.lib().nr_layer_norm_backward_workspace(packed, 0)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        for turn in range(2):
            before = [v.clone() for v in (dx, dw, db)]
            assert nr.lib().nr_layer_norm_backward(packed, 0, ws.data_ptr(), need, ops._stream(0)) == 0
            assert turn == 0 or all(torch.equal(v, k) for v, k in zip((dx, dw, db), before))
        r = rstd.double()[:, None]
        xh = (x64 - mean.double()[:, None]) * r
        gy = dy.double() * w.double()
        dx64 = r * (gy - gy.mean(1, keepdim=True) - xh * (gy * xh).mean(1, keepdim=True))
        if res is not None:
            dx64 = dx64 + res.double()
        # the bounds of test_layer_norm
        exh = 2.0 ** -22 * (1 + (x64.abs() + mean.double().abs()[:, None]) * r)
        sums = (n + 32) * 2.0 ** -23
        mag = r * (gy.abs() + gy.abs().mean(1, keepdim=True) * (1 + sums / 2.0 ** -20)
                   + xh.abs() * (gy * xh).abs().mean(1, keepdim=True) * (1 + sums / 2.0 ** -20))
        lost = r * (exh * (gy * xh).abs().mean(1, keepdim=True) + xh.abs() * (gy.abs() * exh).mean(1, keepdim=True))
        near(dx, dx64, u * dx64.abs() + 2.0 ** -20 * mag + lost + TINY[dtype], "dx")
        dw64, db64 = (dy.double() * xh).sum(0), dy.double().sum(0)
        sw = (dy.double() * xh).abs().sum(0)
        near(dw, dw64, U[F32] * dw64.abs() + (m + 32) * 2.0 ** -23 * sw + (dy.double().abs() * exh).sum(0) + TINY[F32], "dw")
        near(db, db64, U[F32] * db64.abs() + (m + 32) * 2.0 ** -23 * dy.double().abs().sum(0) + TINY[F32], "db")
    for whole, nans in around:
        assert torch.equal(torch.isnan(whole), nans)


def test_layer_norm_gradients_against_differences(ops):
    g = gen(3)
    m, n = 4, 24
    x, dy = rows(g, m, n, F32), rows(g, m, n, F32)
    w, b = 1 + 0.3 * torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
    _, mean, rstd = ops.layer_norm(x, w, b, save=True)
    dx, dw, db = ops.layer_norm_backward(dy, x, w, mean, rstd)

    def total(x_, w_, b_):
        xh = (x_ - x_.mean(1, keepdim=True)) * (x_.var(1, unbiased=False, keepdim=True) + 1e-5).rsqrt()
        return float((dy.double() * (xh * w_ + b_)).sum())

    X, W, B, h = x.double(), w.double(), b.double(), 1e-5
    for r, c in ((0, 0), (3, 23), (2, 11)):
        for which, grad in ((0, float(dx[r, c])), (1, float(dw[c])), (2, float(db[c]))):
            p = []
            for s in (h, -h):
                a = [X.clone(), W.clone(), B.clone()]
                if which == 0:
                    a[0][r, c] += s
                else:
                    a[which][c] += s
                p.append(total(*a))
            # the difference is good to h^2 and 1e-16 / h; the operator to fp32 sums of 24 terms
            assert abs(grad - (p[0] - p[1]) / (2 * h)) <= 1e-5 * (1 + abs(grad))


@pytest.mark.parametrize("shape", [(1, 1), (3, 31), (2, 32), (5, 33), (130, 100), (64, 1536), (1, 5000)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_checkpoint_holds_the_defined_values(ops, shape, dtype):
    m, n = shape
    g = gen(n)
    x = rows(g, m, n, dtype, pad=3, scale=1.0)
    x = x * torch.exp2(torch.randint(-8, 9, (m, n), generator=g, device="cuda").to(dtype))
    x[0, 0] = 127.5 / 64  # the least value that takes the next scale, when it leads its group
    if n > 40:
        x[0, 32:64] = 0.0
        x[0, 33] = 127.5 / 64
        x[-1, :32] = 0.0
    x = torch.nn.functional.pad(x, (0, 5))[:, :n]
    c = ops.checkpoint8(x)
    assert c.shape == (m, n) and c.dtype == dtype
    want = held64(x)
    got = ops.checkpoint8_read(c)
    assert torch.equal(got.double(), want.to(dtype).double())
    assert torch.equal(c.codes[:, n:], torch.zeros_like(c.codes[:, n:]))
    for act in ("relu", "gelu", "silu"):
        a64 = act64(want, act)[0]
        near(ops.checkpoint8_read(c, act=act), a64, U[dtype] * a64.abs() + 2.0 ** -20 * want.abs() + TINY[dtype], act)


def test_checkpoint_extremes(ops):
    inf, nan = float("inf"), float("nan")
    x = torch.zeros(6, 64, device="cuda")
    x[1, 3], x[2, 40], x[3, 0] = inf, nan, -inf
    x[4, 5], x[4, 33] = 3.4028234663852886e38, 2.0 ** -149
    x[5] = torch.linspace(-1, 1, 64, device="cuda") * 2.0 ** -125
    got = ops.checkpoint8_read(ops.checkpoint8(x))
    assert torch.equal(got[0], torch.zeros(64, device="cuda"))
    assert got[1, :32].isnan().all() and (got[1, 32:] == 0).all()
    assert got[2, 32:].isnan().all() and (got[2, :32] == 0).all()
    assert got[3, :32].isnan().all()
    assert got[4, 5].isfinite() and abs(float(got[4, 5]) / 3.4028234663852886e38 - 1) < 0.01 and got[4, 33] == 0
    assert torch.equal(got[5].double(), held64(x[5:6])[0])
    h = torch.full((1, 32), 65504.0, device="cuda", dtype=F16)  # 64 x 2^10 would be infinite in fp16
    assert torch.equal(ops.checkpoint8_read(ops.checkpoint8(h)), h)


def test_non_finite_values_stay_in_their_rows(ops):
    g = gen(1)
    for m in (4, 200):
        x, w, r = rows(g, m, 96, BF16), rows(g, 80, 96, BF16, scale=0.1), rows(g, m, 80, BF16)
        good = ops.linear(x, w, None, act="gelu", residual=r)
        x[1, 5], x[2, 7] = float("nan"), float("inf")
        y = ops.linear(x, w, None, act="gelu", residual=r)
        keep = [i for i in range(m) if i not in (1, 2)]
        assert torch.equal(y[keep], good[keep]) and y[1].isnan().all()
        assert not y[2][w[:, 7] > 0].isfinite().any()
        yn = ops.layer_norm(x)
        assert yn[1].isnan().all() and yn[2].isnan().all() and yn[keep].isfinite().all()
        xg = x.clone()
        dy = rows(g, m, 80, BF16)
        dy[3, 2] = float("nan")
        dx, dw, db = ops.linear_backward(dy, xg, w)
        assert dx[3].isnan().all() and dx[0].isfinite().all() and dw[2].isnan().all() and db[2].isnan()
        assert torch.equal(db.isnan(), torch.arange(80, device="cuda") == 2)


def test_odd_bases_repeated_rows_and_transposed_refusals(ops):
    g = gen(9)
    for off in (1, 2, 4, 8):
        x, w = rows(g, 150, 64, F16, offset=off), rows(g, 72, 64, F16, offset=off, scale=0.1)
        y64, z64, s = linear64(x, w, None, "none", None)
        near(ops.linear(x, w), y64, U[F16] * y64.abs() + 80 * 2.0 ** -23 * s + TINY[F16])
    x = rows(g, 1, 64, F16).expand(150, 64)  # one row read 150 times
    y64, z64, s = linear64(x, w, None, "none", None)
    near(ops.linear(x, w), y64, U[F16] * y64.abs() + 80 * 2.0 ** -23 * s + TINY[F16])
    assert torch.equal(ops.layer_norm(x), ops.layer_norm(x.contiguous()))
    assert torch.equal(ops.checkpoint8(x).codes, ops.checkpoint8(x.contiguous()).codes)
    dy = rows(g, 1, 72, F16).expand(150, 72)  # the gradient of a sum over rows
    for a, b in zip(ops.linear_backward(dy, x, w), ops.linear_backward(dy.contiguous(), x.contiguous(), w)):
        assert torch.equal(a, b)


def test_empty_batches(ops):
    w, b = torch.ones(24, 16, device="cuda", dtype=BF16), torch.ones(24, device="cuda")
    x = torch.empty(0, 16, device="cuda", dtype=BF16)
    y, z = ops.linear(x, w, b, act="gelu", save="z")
    assert y.shape == z.shape == (0, 24)
    y, c = ops.linear(x, w, b, act="gelu", save="z8")
    assert c.shape == (0, 24) and ops.checkpoint8_read(c).shape == (0, 24)
    dx, dw, db = ops.linear_backward(y, ops.checkpoint8(x), w, z=c, act="gelu")
    assert dx.shape == (0, 16) and (dw == 0).all() and (db == 0).all() and dw.shape == (24, 16)
    yn, mean, rstd = ops.layer_norm(x, save=True)
    dx, dw, db = ops.layer_norm_backward(yn, x, None, mean, rstd)
    assert dx.shape == (0, 16) and (dw == 0).all() and (db == 0).all() and mean.shape == (0,)


def test_other_streams(ops):
    g = gen(4)
    x, w, b = rows(g, 2000, 256, BF16), rows(g, 256, 256, BF16, scale=0.06), torch.zeros(256, device="cuda")
    want = ops.linear(ops.layer_norm(x), w, b, act="gelu")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = ops.linear(ops.layer_norm(x, stream=s), w, b, act="gelu", stream=s)
    with torch.cuda.stream(s):
        also = ops.linear(ops.layer_norm(x), w, b, act="gelu")
        c = ops.checkpoint8_read(ops.checkpoint8(x, stream=s), stream=s)
    s.synchronize()
    assert torch.equal(got, want) and torch.equal(also, want)
    assert torch.equal(c.double(), held64(x).to(BF16).double())


def test_graph_capture(ops):
    """The calls allocate through torch and synchronise nothing: a graph replays them on new inputs."""
    g = gen(6)
    x, w = rows(g, 300, 128, BF16), rows(g, 192, 128, BF16, scale=0.1)
    dy = rows(g, 300, 192, BF16)

    def step():
        h, mean, rstd = ops.layer_norm(x, save=True)
        y, z = ops.linear(h, w, act="gelu", save="z8")
        dh, dw, db = ops.linear_backward(dy, h, w, z=z, act="gelu")
        return (y, dw, db) + ops.layer_norm_backward(dh, x, None, mean, rstd)

    step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    x.copy_(rows(g, 300, 128, BF16))
    graph.replay()
    got = [t.clone() for t in out]
    assert all(torch.equal(a, b) for a, b in zip(got, step()))


def test_offsets_past_32_bits(ops):
    """Outputs and inputs of more than 2^32 bytes and 2^31 elements: the last rows are as those of a small call."""
    m, n = 360_000, 6144
    x = torch.zeros(m, 32, device="cuda", dtype=BF16)
    g = gen(8)
    tail = rows(g, 200, 32, BF16)
    x[-200:] = tail
    w = rows(g, n, 32, BF16, scale=0.2)
    y, z8 = ops.linear(x, w, act="gelu", save="z8")
    ys, zs = ops.linear(tail, w, act="gelu", save="z8")
    assert torch.equal(y[-200:], ys) and torch.equal(z8.codes[-200:], zs.codes) and (y[:1000] == 0).all()
    yn = ops.layer_norm(y)
    assert torch.equal(yn[-200:], ops.layer_norm(ys))
    c = ops.checkpoint8(y)
    assert torch.equal(c.codes[-200:], ops.checkpoint8(ys).codes)
    del yn
    dy = torch.zeros(m, n, device="cuda", dtype=BF16)
    dy[-200:] = ys
    dx, dw, db = ops.linear_backward(dy, x, w, z=z8, act="gelu")
    dxs, dws, dbs = ops.linear_backward(ys, tail, w, z=zs, act="gelu")
    # a small batch's products may be summed in parts: the order is fixed for given sizes only
    sx = (ys.double().abs() * 1.13) @ w.double().abs()
    near(dx[-200:], dxs.double(), 2 * U[BF16] * dxs.double().abs() + 2 * (n + 16) * 2.0 ** -23 * sx, "dx")
    d = dws.double()
    # the same products in another order: 2^-8 for the rounding of dz and dw, as above
    mag = ys.double().abs().T @ tail.double().abs() * 1.13
    near(dw, d, 2.0 ** -7 * mag + 1e-30, "dw")
    near(db, dbs.double(), 2.0 ** -12 * ys.double().abs().sum(0) + 1e-30, "db")


def test_refusals(ops):
    x, w = torch.zeros(8, 16, device="cuda", dtype=BF16), torch.zeros(24, 16, device="cuda", dtype=BF16)
    b = torch.zeros(24, device="cuda")
    bad = [
        (ValueError, "dtype", lambda: ops.linear(x.float(), w)),
        (ValueError, "dtype", lambda: ops.linear(x, w.half())),
        (ValueError, "shape", lambda: ops.linear(x, w[:, :8])),
        (ValueError, "shape", lambda: ops.linear(x[0], w)),
        (ValueError, "stride", lambda: ops.linear(x, torch.zeros(16, 24, device="cuda", dtype=BF16).T)),
        (ValueError, "cuda", lambda: ops.linear(x, w.cpu())),
        (ValueError, "CUDA", lambda: ops.linear(x.cpu(), w)),
        (ValueError, "bias", lambda: ops.linear(x, w, b[:8])),
        (ValueError, "bias", lambda: ops.linear(x, w, b.half())),
        (ValueError, "contiguous", lambda: ops.linear(x, w, torch.zeros(48, device="cuda")[::2])),
        (ValueError, "act", lambda: ops.linear(x, w, act="tanh")),
        (ValueError, "save", lambda: ops.linear(x, w, save="y")),
        (ValueError, "out_dtype", lambda: ops.linear(x, w, out_dtype=F16)),
        (ValueError, "residual", lambda: ops.linear(x, w, residual=x)),
        (ValueError, "widths", lambda: ops.linear(x[:, :0], w[:, :0])),
        (TypeError, "Tensor", lambda: ops.linear(np.zeros((8, 16), np.float16), w)),
        (ValueError, "z:", lambda: ops.linear_backward(torch.zeros(8, 24, device="cuda", dtype=BF16), x, w, act="gelu")),
        (ValueError, "x_act", lambda: ops.linear_backward(torch.zeros(8, 24, device="cuda", dtype=BF16), x, w, x_act="gelu")),
        (ValueError, "x:", lambda: ops.linear_backward(torch.zeros(8, 24, device="cuda", dtype=BF16), x[:4], w)),
        (ValueError, "made from", lambda: ops.linear_backward(torch.zeros(8, 24, device="cuda", dtype=BF16),
                                                              ops.checkpoint8(x.half()), w)),
        (ValueError, "bias_dtype", lambda: ops.linear_backward(torch.zeros(8, 24, device="cuda", dtype=BF16), x, w,
                                                               bias_dtype=F16)),
        (ValueError, "eps", lambda: ops.layer_norm(x, eps=0.0)),
        (ValueError, "weight", lambda: ops.layer_norm(x, b)),
        (ValueError, "bias", lambda: ops.layer_norm(x, b[:16], b[:16].to(BF16))),
        (ValueError, "mean", lambda: ops.layer_norm_backward(x, x, None, b[:4], b[:8])),
        (ValueError, "mean", lambda: ops.layer_norm_backward(x, x, None, None, None)),
        (ValueError, "residual_grad", lambda: ops.layer_norm_backward(x, x, None, b[:8], b[:8], residual_grad=x.float())),
        (ValueError, "dtype", lambda: ops.checkpoint8(x.to(torch.int8))),
        (TypeError, "Checkpoint8", lambda: ops.checkpoint8_read(x)),
        (ValueError, "codes", lambda: ops.Checkpoint8(torch.zeros(8, 16, device="cuda", dtype=torch.int8),
                                                      torch.zeros(8, 1, device="cuda", dtype=torch.uint8), (8, 16), BF16)),
        (ValueError, "scales", lambda: ops.Checkpoint8(torch.zeros(8, 32, device="cuda", dtype=torch.int8),
                                                       torch.zeros(8, 2, device="cuda", dtype=torch.uint8), (8, 16), BF16)),
    ]
    for kind, text, call in bad:
        with pytest.raises(kind, match=text):
            call()


def test_expired_waits_are_reported(ops):
    """With a limit that expires at once every role of the product kernel gives
    up; the call ends, the check reports it once, and the next call is right."""
    from paper_2608_15438_gb300 import neuroute as nr

    g = gen(2)
    for m, k, n in ((100, 256, 64), (2000, 512, 512)):  # one CTA a tile, a pair
        x, w = rows(g, m, k, BF16), rows(g, n, k, BF16, scale=k ** -0.5)
        want = ops.linear(x, w)
        ops.check(0)
        assert nr.lib().nr_ops_wait_limit(-1) == 0
        try:
            ops.linear(x, w)
            with pytest.raises(nr.NRError, match="DEVICE_CHECK"):
                ops.check(0)
        finally:
            assert nr.lib().nr_ops_wait_limit(0) == 0
        ops.check(0)
        assert torch.equal(ops.linear(x, w), want)
