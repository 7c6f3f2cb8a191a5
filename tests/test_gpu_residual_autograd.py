"""The residual encoder's autograd functions on the operators themselves: gradients
in any layout, saved-tensor hooks, refused gradients of gradients, no rows."""
import pytest

from gpu_util import need_cuda

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture
def model_of():
    need_cuda()
    from paper_2608_15438_gb300 import ops
    from paper_2608_15438_gb300.residual import ResidualEncoder

    yield lambda hold8: ResidualEncoder(40, 64, 2, 12, hold8=hold8, seed=2)
    ops.check(0)


def rows(m, n, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(m, n, generator=g, device="cuda")


LOSSES = {"sum": lambda y: y.sum(), "mean": lambda y: y.mean(), "columns": lambda y: y.sum(1).square().sum(),
          "transposed": lambda y: (y.T.contiguous() * torch.arange(1.0, y.shape[0] + 1, device="cuda")).sum()}


@pytest.mark.parametrize("loss", LOSSES)
@pytest.mark.parametrize("hold8", [False, True])
def test_gradients_come_in_any_layout(model_of, hold8, loss):
    model, x = model_of(hold8), rows(300, 40, 1)
    leaf = model(x).detach().requires_grad_()
    LOSSES[loss](leaf).backward()
    want = torch.autograd.grad(model(x), list(model.parameters()), leaf.grad.contiguous())
    got = torch.autograd.grad(LOSSES[loss](model(x)), list(model.parameters()))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("hold8", [False, True])
def test_held_activations_can_be_offloaded(model_of, hold8):
    model, x, dl = model_of(hold8), rows(300, 40, 2), rows(300, 12, 3)
    want = torch.autograd.grad(model(x), list(model.parameters()), dl)
    with torch.autograd.graph.save_on_cpu():
        out = model(x)
    got = torch.autograd.grad(out, list(model.parameters()), dl)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("hold8", [False, True])
def test_gradients_of_gradients_are_refused(model_of, hold8):
    model, x = model_of(hold8), rows(300, 40, 4).requires_grad_()
    dx, = torch.autograd.grad(model(x), x, torch.ones(300, 12, device="cuda"), create_graph=True)
    assert dx.isfinite().all()
    with pytest.raises(RuntimeError, match="gradients of gradients"):
        dx.square().sum().backward()


def test_no_rows_and_rows_in_any_layout(model_of):
    model, x = model_of(True), rows(40, 300, 5).T
    out = model.encode(x[:0])
    assert out.shape == (0, 12) and out.dtype == torch.float32
    assert torch.equal(model.encode(x), model.encode(x.contiguous()))
