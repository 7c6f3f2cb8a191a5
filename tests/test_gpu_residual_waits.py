"""The residual encoder after a bounded wait that expired: its outputs are
undefined, and neither training nor encoding goes on with them."""
import pytest

from gpu_util import need_cuda

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture
def expired():
    """Waits expire when first tested, for the test's own calls only."""
    need_cuda()
    from paper_2608_15438_gb300 import neuroute as nr
    from paper_2608_15438_gb300 import ops

    ops.check(0)

    class Limit:
        def __enter__(self):
            assert nr.lib().nr_ops_wait_limit(-1) == 0

        def __exit__(self, *_):
            assert nr.lib().nr_ops_wait_limit(0) == 0

    yield Limit()
    nr.lib().nr_ops_status(0)  # reported, or forgotten with a failed test


def test_encoding_raises(expired):
    from paper_2608_15438_gb300 import neuroute as nr
    from paper_2608_15438_gb300 import ops
    from paper_2608_15438_gb300.residual import ResidualEncoder

    model = ResidualEncoder(96, 64, 2, 16, seed=1)
    x = torch.randn(500, 96, device="cuda")
    want = model.encode(x)
    with expired, pytest.raises(nr.NRError, match="DEVICE_CHECK"):
        model.encode(x)
    assert torch.equal(model.encode(x), want)
    with expired:
        model.encode(x, check=False)
    with pytest.raises(nr.NRError, match="DEVICE_CHECK"):
        ops.check(0)


def test_training_ends_with_the_epoch(expired):
    from paper_2608_15438_gb300 import neuroute as nr
    from paper_2608_15438_gb300.residual import train_residual

    x = torch.randn(256, 96, device="cuda")
    seen = []
    with expired, pytest.raises(nr.NRError, match="DEVICE_CHECK"):
        train_residual(x, 1.0, 64, 1, 16, epochs=3, batch=128, log=seen.append)
    assert seen == []
    _, hist = train_residual(x, 1.0, 64, 1, 16, epochs=2, batch=128)
    assert len(hist) == 2


def test_encoding_can_be_captured(expired):
    from paper_2608_15438_gb300.residual import ResidualEncoder

    model = ResidualEncoder(96, 64, 2, 16, seed=1)
    x = torch.randn(64, 96, device="cuda")
    want = model.encode(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        model.encode(x)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = model.encode(x)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
