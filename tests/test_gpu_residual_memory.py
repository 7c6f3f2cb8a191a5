"""What the residual encoder's training step holds on the GPU, and for how long."""
import pytest

from gpu_util import need_cuda

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

SLACK = 1 << 20  # the loss, and the allocator's blocks of 512 bytes


@pytest.mark.parametrize("hold8", [True, False])
def test_held_activations_end_with_the_backward_pass(hold8):
    """Also while the loss is still at hand: a second step's peak is the first's."""
    need_cuda()
    from paper_2608_15438_gb300 import ops
    from paper_2608_15438_gb300.residual import ResidualEncoder

    m, width, blocks = 8192, 256, 3
    model = ResidualEncoder(96, width, blocks, 16, hold8=hold8, seed=5)
    x = torch.randn(m, 96, device="cuda")
    model(x).square().mean().backward()  # the library's and the allocator's first use
    peaks, loss = [], None
    for _ in range(3):
        for p in model.parameters():
            p.grad = None
        torch.cuda.synchronize()
        start = torch.cuda.memory_allocated()
        torch.cuda.reset_peak_memory_stats()
        loss = model(x).square().mean()
        held = torch.cuda.memory_allocated() - start
        # a unit of width of the block's input and four of its pre-activations at 33/32 bytes, or ten in 16 bits
        assert held >= m * width * blocks * (5 * 33 / 32 if hold8 else 20)
        loss.backward()
        grads = sum(p.grad.numel() * 4 for p in model.parameters())
        assert torch.cuda.memory_allocated() - start <= grads + SLACK
        peaks.append(torch.cuda.max_memory_allocated() - start)
    assert peaks[1] <= peaks[0] + SLACK and peaks[2] <= peaks[0] + SLACK
    assert float(loss.detach()) > 0
    ops.check(0)
