"""The residual encoder's autograd functions on the CPU, with a plain stand-in
for the operators: gradients of gradients, gradients as autograd lays them
out, and what is kept for the backward pass. The stand-in takes the operators' arguments and
refuses what they refuse."""
import gc
import weakref

import pytest
import torch

from paper_2608_15438_gb300 import residual

ACTS = {"none": lambda z: z, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}


class Held:
    """A checkpoint's stand-in: 32 columns share a power of two."""

    def __init__(self, codes, scales, shape, dtype):
        self.codes, self.scales, self.shape, self.dtype = codes, scales, tuple(shape), dtype

    @property
    def device(self):
        return self.codes.device


class PlainOps:
    Checkpoint8 = Held

    @staticmethod
    def _rows(*ts):
        for t in ts:
            if t is not None and t.stride(1) != 1:
                raise ValueError("rows must be contiguous (stride(1) == 1)")

    @staticmethod
    def checkpoint8(x):
        m, n = x.shape
        g = -(-n // 32)
        v = torch.nn.functional.pad(x.detach().float(), (0, g * 32 - n)).view(m, g, 32)
        e = torch.floor(torch.log2(v.abs().amax(2).clamp(min=1e-30) / 127.5)) + 1
        codes = torch.round(v / torch.exp2(e)[:, :, None]).clamp(-127, 127).to(torch.int8).view(m, g * 32)
        return Held(codes, (e + 133).to(torch.uint8), (m, n), x.dtype)

    @staticmethod
    def read(c):
        if not isinstance(c, Held):
            return c.float()
        m, n = c.shape
        step = torch.exp2(c.scales.float() - 133)[:, :, None]
        return (c.codes.view(m, -1, 32).float() * step).view(m, -1)[:, :n]

    @classmethod
    def linear(cls, x, w, bias=None, act="none", residual=None, save=None, out_dtype=None):
        cls._rows(x, w, residual)
        z = x.float() @ w.float().T + bias.float()
        y = ACTS[act](z)
        if residual is not None:
            y = y + residual.float()
        y = y.to(out_dtype or x.dtype)
        z = z.to(x.dtype)
        return y if save is None else (y, cls.checkpoint8(z) if save == "z8" else z)

    @classmethod
    def linear_backward(cls, dy, x, w, z=None, act="none", x_act="none", need=(True, True, True)):
        cls._rows(dy, w)
        dz = dy.float().contiguous()  # one order of sums for every layout
        if act != "none":
            with torch.enable_grad():
                v = cls.read(z).clone().requires_grad_()
                (s,) = torch.autograd.grad(ACTS[act](v).sum(), v)
            dz = dz * s
        xv = ACTS[x_act](cls.read(x))
        return ((dz @ w.float()).to(w.dtype) if need[0] else None, (dz.T @ xv).to(w.dtype) if need[1] else None,
                dz.sum(0) if need[2] else None)

    @classmethod
    def layer_norm(cls, x, weight, bias, eps=1e-5, save=False):
        v = cls.read(x)
        mean, rstd = v.mean(1), (v.var(1, unbiased=False) + eps).rsqrt()
        y = ((v - mean[:, None]) * rstd[:, None] * weight + bias).to(x.dtype)
        return (y, mean, rstd) if save else y

    @classmethod
    def layer_norm_backward(cls, dy, x, weight, mean, rstd, residual_grad=None):
        cls._rows(dy, residual_grad)
        xh = (cls.read(x) - mean[:, None]) * rstd[:, None]
        g = dy.float() * weight
        dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        if residual_grad is not None:
            dx = dx + residual_grad.float()
        return dx.to(dy.dtype), (dy.float() * xh).sum(0), dy.float().contiguous().sum(0)

    @staticmethod
    def check(device=0):
        pass


@pytest.fixture(autouse=True)
def plain(monkeypatch):
    monkeypatch.setattr(residual, "ops", PlainOps)


def encoder(hold8, D=24, width=32, b=6):
    return residual.ResidualEncoder(D, width, 2, b, hold8=hold8, device="cpu", seed=1)


def rows(m, D, seed=0):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.randn(m, D, generator=g)


def test_the_stand_in_gives_the_encoders_gradients():
    """Against autograd through the formulas in 64 bits; a path of a gradient crosses
    at most ten roundings to 8 significant bits."""
    model, x = encoder(False), rows(40, 24)
    p = {n: v.detach().double().clone().requires_grad_() for n, v in model.named_parameters()}
    r = x.bfloat16().double() @ p["stem.0"].T + p["stem.1"]
    norm = torch.nn.functional.layer_norm
    for i in range(2):
        q = [p[f"blocks.{i}.{j}"] for j in range(6)]
        r = r + ACTS["gelu"](norm(r, (32,), q[0], q[1]) @ q[2].T + q[3]) @ q[4].T + q[5]
    want = norm(r, (32,), p["head.0"], p["head.1"]) @ p["head.2"].T + p["head.3"]
    dl = rows(40, 6, 1)
    want.backward(dl.double())
    model(x).backward(dl)
    for n, v in model.named_parameters():
        assert float((v.grad.double() - p[n].grad).norm() / p[n].grad.norm()) <= 0.04, n


@pytest.mark.parametrize("hold8", [False, True])
def test_gradients_of_gradients_are_refused(hold8):
    """The backward passes have no derivatives of their own: a penalty on a
    gradient says so instead of losing its share."""
    model = encoder(hold8)
    x = rows(40, 24).requires_grad_()
    out = model(x)
    dx, = torch.autograd.grad(out, x, torch.ones(40, 6), create_graph=True)
    with pytest.raises(RuntimeError, match="gradients of gradients"):
        (out.sum() + (dx * dx).sum()).backward()


@pytest.mark.parametrize("part", ["_Linear", "_Norm"])
def test_gradients_of_gradients_are_refused_by_each_function(part):
    x = rows(8, 16).bfloat16().requires_grad_()
    if part == "_Linear":
        y = residual._Linear.apply(x, torch.nn.Parameter(rows(4, 16, 2)), torch.nn.Parameter(rows(1, 4, 3)[0]), torch.float32)
    else:
        y = residual._Norm.apply(x, torch.nn.Parameter(torch.ones(16)), torch.nn.Parameter(torch.zeros(16)))
    dx, = torch.autograd.grad(y, x, torch.ones_like(y), create_graph=True)
    assert dx.requires_grad
    with pytest.raises(RuntimeError, match="gradients of gradients"):
        dx.float().pow(2).sum().backward()


def test_a_graph_that_is_not_differentiated_again_is_served():
    model, x = encoder(True), rows(40, 24)
    dl = rows(40, 6, 1)
    want = torch.autograd.grad(model(x), model.stem[0], dl)[0]
    got = torch.autograd.grad(model(x), model.stem[0], dl, create_graph=True)[0]
    assert torch.equal(got, want)


def kept(model, x, monkeypatch):
    """The loss of a step, and weak references to what its forward pass held."""
    refs = []
    for name in ("checkpoint8", "linear"):
        fn = getattr(PlainOps, name)

        def spy(*args, _fn=fn, **kw):
            out = _fn(*args, **kw)
            for v in out if isinstance(out, tuple) else (out,):
                refs.extend(weakref.ref(t) for t in ((v.codes, v.scales) if isinstance(v, Held) else (v,)))
            return out

        monkeypatch.setattr(PlainOps, name, staticmethod(spy))
    return model(x).square().mean(), refs


@pytest.mark.parametrize("hold8", [False, True])
def test_a_backward_pass_releases_what_was_held(hold8, monkeypatch):
    """Also while the loss is still at hand, as in a loop that keeps it for its log."""
    loss, refs = kept(encoder(hold8), rows(40, 24), monkeypatch)
    gc.collect()
    assert sum(r() is not None for r in refs) >= (8 if hold8 else 6)
    loss.backward()
    gc.collect()
    assert [r() for r in refs if r() is not None] == []
    assert loss.grad_fn is not None


@pytest.mark.parametrize("hold8", [False, True])
def test_hooks_see_all_that_is_held(hold8):
    """Saved-tensor hooks (offloading, checkpointing) get every activation of a block:
    the 8-bit codes and scales of its input and pre-activations, or the input,
    the pre-activations, the norm's output and the activation in 16 bits."""
    seen = []

    def pack(t):
        seen.append((t.dtype, tuple(t.shape)))
        return t.clone()

    model, x = encoder(hold8), rows(40, 24)
    dl = rows(40, 6, 1)
    want = torch.autograd.grad(model(x), list(model.parameters()), dl)
    with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t):
        out = model(x)
    got = torch.autograd.grad(out, list(model.parameters()), dl)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    if hold8:
        for item in ((torch.int8, (40, 32)), (torch.uint8, (40, 1)), (torch.int8, (40, 128)), (torch.uint8, (40, 4))):
            assert seen.count(item) == 2, item
    else:
        assert seen.count((torch.bfloat16, (40, 128))) == 4  # z and a of two blocks
        assert seen.count((torch.bfloat16, (40, 32))) == 4 + 2  # r and h; the head norm's input and output


def test_a_changed_input_of_a_block_is_noticed():
    p = [v for v in encoder(False).blocks[0]]
    r = rows(40, 32).bfloat16().requires_grad_()
    s = r * 1.0
    y = residual._Block.apply(s, *p, "gelu", False)
    with torch.no_grad():
        s.mul_(2.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward(torch.ones_like(y))


def test_a_graph_kept_for_a_second_pass_gives_the_same_gradients():
    for hold8 in (False, True):
        model, x = encoder(hold8), rows(40, 24)
        out, dl = model(x), rows(40, 6, 1)
        a = torch.autograd.grad(out, list(model.parameters()), dl, retain_graph=True)
        b = torch.autograd.grad(out, list(model.parameters()), dl)
        assert all(torch.equal(u, v) for u, v in zip(a, b))


LAYOUTS = {"sum": lambda y: y.sum(), "mean": lambda y: y.mean(), "rows": lambda y: y.sum(0).square().sum(),
           "columns": lambda y: y.sum(1).square().sum(),
           "transposed": lambda y: (y.T.contiguous() * torch.arange(1.0, y.shape[0] + 1)).sum(),
           "half": lambda y: y[:, ::2].square().sum()}


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("hold8", [False, True])
def test_gradients_come_in_any_layout(hold8, layout):
    """Autograd brings expanded and transposed gradients; they give what contiguous ones give."""
    model, x = encoder(hold8), rows(40, 24)
    leaf = model(x).detach().requires_grad_()
    LAYOUTS[layout](leaf).backward()
    want = torch.autograd.grad(model(x), list(model.parameters()), leaf.grad.contiguous())
    got = torch.autograd.grad(LAYOUTS[layout](model(x)), list(model.parameters()))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("layout", ["sum", "transposed"])
@pytest.mark.parametrize("part", ["linear", "norm", "block8", "block16"])
def test_each_function_takes_a_gradient_in_any_layout(part, layout):
    x = rows(8, 32).bfloat16().requires_grad_()
    g, b = torch.ones(32), torch.zeros(32)
    if part == "linear":
        y = residual._Linear.apply(x, rows(12, 32, 2), torch.zeros(12), torch.float32)
    elif part == "norm":
        y = residual._Norm.apply(x, g, b)
    else:
        y = residual._Block.apply(x, *[v.detach() for v in encoder(False).blocks[0]], "gelu", part == "block8")
    dy = torch.ones(1, 1, dtype=y.dtype).expand(y.shape) if layout == "sum" else rows(y.shape[1], 8, 4).to(y.dtype).T
    want, = torch.autograd.grad(y, x, dy.contiguous(), retain_graph=True)
    assert torch.equal(torch.autograd.grad(y, x, dy)[0], want)


def test_rows_to_encode_come_in_any_layout():
    model, x = encoder(True), rows(24, 40).T
    assert torch.equal(model(x), model(x.contiguous()))
    assert torch.equal(model.encode(x), model.encode(x.contiguous()))


@pytest.mark.parametrize("batch", [1 << 17, 16])
def test_no_rows_give_no_logits(batch):
    model = encoder(True)
    out = model.encode(torch.empty(0, 24), batch=batch)
    assert out.shape == (0, 6) and out.dtype == torch.float32
    assert torch.equal(model.encode(rows(40, 24), batch=batch), model.encode(rows(40, 24)))
