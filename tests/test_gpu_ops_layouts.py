"""The encoder operators through the C ABI with every matrix at a pitch and an
address of its own, and at widths that take every form of a kernel: values
against 64 bits under the bounds of test_gpu_ops.py, and the bytes around the
outputs as they were."""
import pytest

from gpu_util import need_cuda

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_ops import BF16, F16, F32, HALF, TINY, U, act64, gen, grads64, held64, linear64, near, norm_tol  # noqa: E402

FILL = 0xA5


@pytest.fixture(scope="module")
def ops():
    need_cuda()
    from paper_2608_15438_gb300 import ops as o

    yield o
    o.check(0)


class Out:
    """[m x n] at a pitch of n + pad and `offset` elements past an aligned address,
    in a buffer of bytes that have to stay around it."""

    def __init__(self, m, n, dtype, pad=0, offset=0):
        e = torch.empty(0, dtype=dtype).element_size()
        ld = n + pad
        self.buf = torch.full(((offset + m * ld + 64) * e,), FILL, dtype=torch.uint8, device="cuda")
        flat = self.buf.view(dtype)
        self.t = flat.as_strided((m, n), (ld, 1), offset)
        self.ld = ld
        own = torch.zeros(flat.shape, dtype=torch.bool, device="cuda")
        own.as_strided((m, n), (ld, 1), offset).fill_(True)
        self.around = ~own.repeat_interleave(e)

    def ptr(self):
        return self.t.data_ptr()

    def check(self, what):
        changed = int((self.buf[self.around] != FILL).sum())
        assert changed == 0, f"{what}: {changed} bytes around the matrix changed"


def inp(g, m, n, dtype, pad=0, offset=0, scale=1.0, shift=0.0):
    """An input laid out likewise, NaN around it."""
    o = Out(m, n, dtype, pad, offset)
    o.buf.view(dtype).fill_(float("nan"))
    o.t.copy_(torch.randn(m, n, generator=g, device="cuda") * scale + shift)
    return o


def call(fn, workspace, packed, device=0):
    from paper_2608_15438_gb300 import neuroute as nr
    from paper_2608_15438_gb300 import ops as o

    L = nr.lib()
    if workspace is None:
        assert getattr(L, fn)(packed, device, o._stream(device)) == 0
        return
    need = getattr(L, workspace)(packed, device)
    assert need >= 0
    ws = torch.full((need + 256,), FILL, dtype=torch.uint8, device="cuda")
    assert getattr(L, fn)(packed, device, ws.data_ptr(), need, o._stream(device)) == 0
    assert (ws[need:] == FILL).all(), "past the scratch"


# (pad, offset) of x, w, residual, y, z, dx and so on: aligned, alike, all different
LAYOUTS = {"aligned": [(0, 0)] * 6, "pitched": [(8, 8)] * 6, "odd": [(3, 1), (1, 5), (5, 3), (7, 2), (2, 7), (9, 4)],
           "even": [(2, 2), (6, 4), (4, 6), (2, 4), (6, 2), (4, 2)], "outputs": [(0, 0)] * 3 + [(3, 1), (1, 3), (5, 7)]}
# few rows, one CTA a tile and a pair, whole and ragged blocks, sums in parts
LINEAR = [(1, 40, 24), (3, 129, 257), (8, 96, 33), (9, 64, 64), (17, 100, 1), (130, 200, 520), (129, 2048, 96),
          (257, 771, 1013), (700, 64, 264)]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("i,shape", list(enumerate(LINEAR)))
@pytest.mark.parametrize("dtype", HALF)
def test_linear_forward(ops, layout, i, shape, dtype):
    m, k, n = shape
    g, at = gen(i), LAYOUTS[layout]
    act = ["gelu", "none", "silu", "relu"][i % 4]
    x, w = inp(g, m, k, dtype, *at[0]), inp(g, n, k, dtype, *at[1], scale=k ** -0.5)
    r = inp(g, m, n, dtype, *at[2])
    b = torch.randn(n, generator=g, device="cuda")
    y64, z64, s = linear64(x.t, w.t, b, act, r.t)
    acc = (k + 16) * 2.0 ** -23 * s
    for ydt in (dtype, F32):
        for save in ("", "z", "z8"):
            y = Out(m, n, ydt, *at[3])
            groups = -(-n // 32)
            z = Out(m, n, dtype, *at[4]) if save == "z" else Out(m, groups * 32, torch.int8)
            sc = Out(m, groups, torch.uint8)
            packed = ops._LINEAR.pack(m, k, n, ops._DT[dtype], ops._DT[ydt], ops._DT[F32], ops.ACTIVATIONS[act], x.ptr(), x.ld,
                                      0, 0, w.ptr(), w.ld, b.data_ptr(), r.ptr(), r.ld, y.ptr(), y.ld, z.ptr() if save else 0,
                                      z.ld if save == "z" else 0, sc.ptr() if save == "z8" else 0, 0, 0, 0, 0, 0, 0)
            call("nr_linear_forward", "nr_linear_forward_workspace", packed)
            near(y.t, y64, U[ydt] * y64.abs() + 1.13 * acc + 2.0 ** -20 * z64.abs() + TINY[ydt], "y")
            for o, what in ((y, "y"), (z, "z"), (sc, "scales")):
                o.check(what)
            if save == "z":
                near(z.t, z64, U[dtype] * z64.abs() + acc + TINY[dtype], "z")
            elif save == "z8":
                v = ops.checkpoint8_read(ops.Checkpoint8(z.t.contiguous(), sc.t.contiguous(), (m, n), dtype))
                top = torch.nn.functional.pad(z64.abs() + acc, (0, -n % 32)).view(m, -1, 32).amax(2)
                step = torch.exp2(torch.floor(torch.log2(top / 127.5)) + 1).repeat_interleave(32, 1)[:, :n]
                near(v, z64, 0.5 * step * 1.001 + acc + 2 * TINY[dtype], "z8")
            else:
                assert (z.buf == FILL).all() and (sc.buf == FILL).all()


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("i,shape", list(enumerate(LINEAR)))
@pytest.mark.parametrize("dtype", HALF)
def test_linear_backward(ops, layout, i, shape, dtype):
    m, k, n = shape
    g, at, u = gen(40 + i), LAYOUTS[layout], U[dtype]
    act = ["silu", "gelu", "relu", "none"][i % 4]
    x, w = inp(g, m, k, dtype, *at[0]), inp(g, n, k, dtype, *at[1], scale=k ** -0.5)
    z = inp(g, m, n, dtype, *at[2])
    for ydt in (dtype, F32):
        dy = inp(g, m, n, ydt, *at[4], scale=0.25)
        dx, dw = Out(m, k, dtype, *at[3]), Out(1, n * k, dtype, 0, at[5][1])
        db = Out(1, n, F32, 0, at[5][1])
        packed = ops._LINEAR.pack(m, k, n, ops._DT[dtype], ops._DT[ydt], ops._DT[F32], ops.ACTIVATIONS[act], x.ptr(), x.ld, 0, 0,
                                  w.ptr(), w.ld, 0, 0, 0, 0, 0, z.ptr(), z.ld, 0, dy.ptr(), dy.ld, dx.ptr(), dx.ld, dw.ptr(),
                                  db.ptr())
        call("nr_linear_backward", "nr_linear_backward_workspace", packed)
        _, dx64, dw64, db64, sx, sw, sb = grads64(dy.t, x.t, w.t, z.t if act != "none" else None, act)
        # a slope is good to 2^-20 absolutely (GELU's and SiLU's cross zero), dz is rounded to 16 bits for the products
        d, sl = dy.t.double().abs(), 0.0 if act in ("none", "relu") else 2.0 ** -20
        near(dx.t, dx64, u * dx64.abs() + (u + (n + 16) * 2.0 ** -23) * sx + sl * d @ w.t.double().abs() + (n + 1) * TINY[dtype], "dx")
        near(dw.t.view(n, k), dw64,
             u * dw64.abs() + (u + (m + 16) * 2.0 ** -23) * sw + sl * d.T @ x.t.double().abs() + (m * 4 + 1) * TINY[dtype], "dw")
        near(db.t[0], db64, U[F32] * db64.abs() + sl * d.sum(0) + (m + 16) * 2.0 ** -23 * sb + TINY[F32], "db")
        for o, what in ((dx, "dx"), (dw, "dw"), (db, "dbias")):
            o.check(what)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("shape", [(1, 1), (5, 33), (130, 100), (9, 51), (64, 1536), (3, 771), (2, 5000)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_checkpoint(ops, layout, shape, dtype):
    from paper_2608_15438_gb300 import neuroute as nr

    m, n = shape
    g, at, groups = gen(n), LAYOUTS[layout], -(-n // 32)
    x = inp(g, m, n, dtype, *at[0])
    codes, scales = Out(m, groups * 32, torch.int8), Out(m, groups, torch.uint8, 0, at[5][1])
    L, st = nr.lib(), ops._stream(0)
    assert L.nr_checkpoint8_write(x.ptr(), ops._DT[dtype], m, n, x.ld, codes.ptr(), scales.ptr(), 0, st) == 0
    want = held64(x.t)
    codes.check("codes"), scales.check("scales")
    for act in ("none", "silu"):
        y = Out(m, n, dtype, *at[3])
        assert L.nr_checkpoint8_read(codes.ptr(), scales.ptr(), m, n, ops.ACTIVATIONS[act], y.ptr(), ops._DT[dtype], y.ld, 0, st) == 0
        y.check("y")
        if act == "none":
            assert torch.equal(y.t.double(), want.to(dtype).double())
        else:
            a64 = act64(want, act)[0]
            near(y.t, a64, U[dtype] * a64.abs() + 2.0 ** -20 * want.abs() + TINY[dtype], act)


# warps with three and six eights a thread, blocks of one, two and four, several rows' groups a block, long rows
NORM = [(5, 264), (300, 512), (41, 768), (130, 1000), (700, 1024), (9, 1600), (66, 2048), (7, 2504), (5, 4000), (5, 5000),
        (9, 8200), (4, 9001), (3, 16384), (2, 16385), (1300, 48), (33, 257), (12, 1601)]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("shape", NORM)
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_layer_norm(ops, layout, shape, dtype):
    m, n = shape
    g, at, u = gen(m + n), LAYOUTS[layout], U[dtype]
    x, dy, res = inp(g, m, n, dtype, *at[0], shift=0.5), inp(g, m, n, dtype, *at[1]), inp(g, m, n, dtype, *at[2])
    wdt = F32 if n % 2 else dtype
    w = inp(g, 1, n, wdt, 0, at[5][0], scale=0.3, shift=1.0).t[0]
    b = inp(g, 1, n, wdt, 0, at[5][1]).t[0]
    held = ops.checkpoint8(x.t)
    for from8 in (False, True):
        x64 = held64(x.t) if from8 else x.t.double()
        src = (held.codes.data_ptr(), 0, held.scales.data_ptr()) if from8 else (x.ptr(), x.ld, 0)
        mean64, rstd64 = x64.mean(1), (x64.var(1, unbiased=False) + 1e-5).rsqrt()
        xh = (x64 - mean64[:, None]) * rstd64[:, None]
        t = norm_tol(x64, n)
        y, mean, rstd = Out(m, n, dtype, *at[3]), Out(1, m, F32), Out(1, m, F32)
        call("nr_layer_norm_forward", None,
             ops._NORM.pack(m, n, ops._DT[dtype], ops._DT[wdt], 1e-5, *src, w.data_ptr(), b.data_ptr(), y.ptr(), y.ld, mean.ptr(),
                            rstd.ptr(), 0, 0, 0, 0, 0, 0, 0, 0))
        y64 = xh * w.double() + b.double()
        near(y.t, y64, u * y64.abs() + t * (1 + xh.abs()) * w.double().abs() + 2.0 ** -22 * b.double().abs() + TINY[dtype], "y")
        near(mean.t[0], mean64, (n + 16) * 2.0 ** -23 * x64.abs().mean(1), "mean")
        near(rstd.t[0], rstd64, rstd64 * t[:, 0], "rstd")
        for o, what in ((y, "y"), (mean, "mean"), (rstd, "rstd")):
            o.check(what)
        for dres in (None, res):
            dx, dw, db = Out(m, n, dtype, *at[4]), Out(1, n, wdt, 0, at[5][1]), Out(1, n, wdt, 0, at[5][0])
            call("nr_layer_norm_backward", "nr_layer_norm_backward_workspace",
                 ops._NORM.pack(m, n, ops._DT[dtype], ops._DT[wdt], 0.0, *src, w.data_ptr(), 0, 0, 0, mean.ptr(), rstd.ptr(),
                                dy.ptr(), dy.ld, 0 if dres is None else dres.ptr(), 0 if dres is None else dres.ld, dx.ptr(), dx.ld,
                                dw.ptr(), db.ptr()))
            mu, r = mean.t[0].double()[:, None], rstd.t[0].double()[:, None]
            xr = (x64 - mu) * r
            gy = dy.t.double() * w.double()
            dx64 = r * (gy - gy.mean(1, keepdim=True) - xr * (gy * xr).mean(1, keepdim=True))
            if dres is not None:
                dx64 = dx64 + dres.t.double()
            exh = 2.0 ** -22 * (1 + (x64.abs() + mu.abs()) * r)
            sums = (n + 32) * 2.0 ** -23
            mag = r * (gy.abs() + gy.abs().mean(1, keepdim=True) * (1 + sums / 2.0 ** -20)
                       + xr.abs() * (gy * xr).abs().mean(1, keepdim=True) * (1 + sums / 2.0 ** -20))
            lost = r * (exh * (gy * xr).abs().mean(1, keepdim=True) + xr.abs() * (gy.abs() * exh).mean(1, keepdim=True))
            near(dx.t, dx64, u * dx64.abs() + 2.0 ** -20 * mag + lost + TINY[dtype], "dx")
            dd = dy.t.double()
            dw64, db64, sw = (dd * xr).sum(0), dd.sum(0), (dd * xr).abs().sum(0)
            near(dw.t[0], dw64, U[wdt] * dw64.abs() + (m + 32) * 2.0 ** -23 * sw + (dd.abs() * exh).sum(0) + TINY[wdt], "dw")
            near(db.t[0], db64, U[wdt] * db64.abs() + (m + 32) * 2.0 ** -23 * dd.abs().sum(0) + TINY[wdt], "db")
            for o, what in ((dx, "dx"), (dw, "dweight"), (db, "dbias")):
                o.check(what)
