"""AdamW states whose parameters become other tensors between steps, and averages and norms at the ends of fp32's range."""
import pytest

from gpu_util import need_cuda

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.fixture
def ops():
    need_cuda()
    from paper_2608_15438_gb300 import ops as o

    return o


@pytest.mark.parametrize("old,new", [(F32, BF16), (BF16, F16), (F16, F32)])
@pytest.mark.parametrize("bits", [32, 8])
def test_another_type_at_the_same_address(ops, old, new, bits):
    """The step is the one that a state over the new tensor takes, and what lies behind it stays."""
    g = torch.Generator(device="cuda").manual_seed(1)
    n = 500
    buf = torch.ones(4 * n, device="cuda")
    p = torch.nn.Parameter(buf.view(old)[:n])
    x = torch.randn(n, generator=g, device="cuda")
    s = ops.AdamWState([p], bits=bits)
    ops.adamw_step(s, [x], 1e-2)
    address = p.data_ptr()
    p.data = buf.view(new)[:n]
    assert p.data_ptr() == address and p.dtype == new
    p.data.copy_(torch.randn(n, generator=g, device="cuda"))
    twin = p.detach().clone()
    t = ops.AdamWState([twin], bits=bits, m=s.m.clone() if bits == 32 else [c.clone() for c in s.m],
                       v=s.v.clone() if bits == 32 else [c.clone() for c in s.v], step=s.step.clone())
    behind = buf.view(new)[n:].clone()
    ops.adamw_step(s, [x], 1e-2)
    ops.adamw_step(t, [x], 1e-2)
    assert torch.equal(p.detach(), twin) and torch.equal(buf.view(new)[n:], behind)


def test_a_transposed_parameter_is_refused(ops):
    from paper_2608_15438_gb300.optim import AdamW

    p = torch.nn.Parameter(torch.randn(64, 64, device="cuda"))
    opt = AdamW([p], lr=1e-2)
    p.grad = torch.ones_like(p)
    opt.step()
    before = p.detach().clone()
    p.data = p.data.t()
    p.grad = torch.randn_like(p)
    with pytest.raises(ValueError, match="does not fit"):
        opt.step()
    assert torch.equal(p.detach(), before.t()) and int(opt.state.step) == 1


@pytest.mark.parametrize("bits,offset", [(32, 0), (32, 1), (8, 0), (8, 1)])
@pytest.mark.parametrize("eps", [1e-20, 1e-12, 2e-11, 5.7e-11, 5.8e-11, 1e-8])
@pytest.mark.parametrize("b2", [0.0, 0.95, 0.999, 1 - 1e-6])
@pytest.mark.parametrize("t", [1, 5])
def test_averages_below_the_normal_numbers(ops, bits, offset, eps, b2, t):
    """Squares of gradients down to nothing: their root counts beside eps however small it is. m' and v' are those that
    the step holds to (three roundings, from zeros one and two); the update from them is allowed 2^-20 of itself, as
    elsewhere: 1 - beta^t good to 2^-22, root and reciprocal, four roundings."""
    import math

    import numpy as np

    f, n, b1, lr = np.float32, 4096, 0.9, 1e-2
    rng = np.random.default_rng(int(1e3 * b2) + t)
    x = (10.0 ** rng.uniform(-23.0, -15.0, n) * rng.choice([-1.0, 1.0], n)).astype(f)
    grads, params = torch.zeros(n + offset, device="cuda")[offset:], torch.zeros(n + offset, device="cuda")[offset:]
    grads.copy_(torch.from_numpy(x))
    s = ops.AdamWState([params], bits=bits)
    s.step.fill_(t - 1)
    ops.adamw_step(s, [grads], lr, betas=(b1, b2), eps=eps, weight_decay=0.0)
    m, v = f(1 - b1) * x, (f(1 - b2) * x) * x
    assert (v < 2.0 ** -126).any() and (v > 2.0 ** -126).any()
    if bits == 32:
        assert np.array_equal(s.m.cpu().numpy(), m) and np.array_equal(s.v.cpu().numpy(), v)
    root = 1.0 if b2 == 0.0 else math.sqrt(-1.0 / math.expm1(t * math.log(b2)))
    want = -lr / -math.expm1(t * math.log(b1)) * m.astype(np.float64) / (np.sqrt(v.astype(np.float64)) * root + eps)
    got = params.cpu().numpy().astype(np.float64)
    assert (np.abs(got - want) <= 2.0 ** -20 * np.abs(want)).all()


@pytest.mark.parametrize("dtype,offset", [(F32, 0), (BF16, 0), (F32, 1), (BF16, 1)])
@pytest.mark.parametrize("n", [1000, 1 << 20, (1 << 27) + 77])
def test_norms_of_gradients_near_two_to_the_60(ops, n, dtype, offset):
    """Gradients below 2^60, many of them: their squares' sum is past fp32's range, the norm is not."""
    top = 2.0 ** 60 * (1 - 2.0 ** -8)
    x = torch.full((n + offset,), top, device="cuda", dtype=dtype)[offset:]
    x[::2].neg_()
    x[:7] = 1.0
    want = top * (n - 7) ** 0.5
    assert abs(float(ops.grad_norm([x])) - want) <= 2.0 ** -20 * want
    p = torch.zeros(n + offset, device="cuda", dtype=BF16)[offset:]
    s = ops.AdamWState([p])
    norm = ops.adamw_step(s, [x], 1e-3, max_norm=1.0, weight_decay=0.0)
    assert abs(float(norm) - want) <= 2.0 ** -20 * want and int(s.step) == 1
    m = 0.1 * top / want
    assert abs(float(s.m[8]) + m) <= 2.0 ** -18 * m and abs(float(s.m[9]) - m) <= 2.0 ** -18 * m
    x[n // 2] = float("inf")
    assert not float(ops.grad_norm([x])) < float("inf")
    x[n // 2] = float("nan")
    assert not float(ops.grad_norm([x])) < float("inf")


def test_steps_from_several_threads(ops):
    """Each on a state and a stream of its own."""
    import threading

    def states(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        params = [torch.randn(k, generator=g, device="cuda") for k in (70000 + seed, 33)]
        grads = [torch.randn(p.shape, generator=g, device="cuda") for p in params]
        return ops.AdamWState(params, bits=8 if seed % 2 else 32), grads

    def steps(seed, state, grads):
        for _ in range(40):
            ops.adamw_step(state, grads, 1e-3, max_norm=0.1 * (seed + 1), seed=seed)

    want = [states(i) for i in range(4)]
    for i, w in enumerate(want):
        steps(i, *w)
    got = [states(i) for i in range(4)]
    torch.cuda.synchronize()

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            steps(i, *got[i])

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for (a, _), (b, _) in zip(got, want):
        assert int(a.step) == 40 and all(torch.equal(x, y) for x, y in zip(a._tensors(), b._tensors()))
