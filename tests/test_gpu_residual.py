"""The residual encoder on the library's operators: its gradients against torch
autograd in 64 bits, training with L_sim, and an index searched through its
logits."""
import pytest

from gpu_util import need_cuda

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def reference(model, x):
    """The same encoder in 64 bits, on copies of the parameters."""
    p = {n: v.detach().double().clone().requires_grad_() for n, v in model.named_parameters()}
    F = torch.nn.functional

    def norm(r, g, b):
        return F.layer_norm(r, (r.shape[1],), g, b, eps=1e-5)

    r = x.double() @ p["stem.0"].T + p["stem.1"]
    for i in range(len(model.blocks)):
        q = [p[f"blocks.{i}.{j}"] for j in range(6)]
        r = r + F.gelu(norm(r, q[0], q[1]) @ q[2].T + q[3]) @ q[4].T + q[5]
    return norm(r, p["head.0"], p["head.1"]) @ p["head.2"].T + p["head.3"], p


@pytest.mark.parametrize("hold8", [False, True])
@pytest.mark.parametrize("m,D,width,b", [(64, 96, 64, 16), (300, 128, 96, 20)])
def test_gradients(hold8, m, D, width, b):
    """A path of a gradient crosses at most ten roundings to 8 significant bits
    (2^-8 each, so 0.04 in all); holding in 8 bits adds an error of at most 0.015
    of the values' deviation (half of a step of 2 / 127.5 of a group's largest
    value, uniform) at three places."""
    need_cuda()
    from paper_2608_15438_gb300 import ops
    from paper_2608_15438_gb300.residual import ResidualEncoder

    torch.manual_seed(m)
    model = ResidualEncoder(D, width, 2, b, hold8=hold8, seed=3)
    x = torch.randn(m, D, device="cuda").bfloat16()
    dl = torch.randn(m, b, device="cuda")
    out = model(x)
    assert out.dtype == torch.float32 and out.shape == (m, b)
    out.backward(dl)
    want, p = reference(model, x)
    want.backward(dl.double())
    tol = 0.04 + (0.045 if hold8 else 0.0)
    assert float((out.detach().double() - want.detach()).norm() / want.detach().norm()) <= 0.04
    for name, v in model.named_parameters():
        g = p[name].grad
        assert float((v.grad.double() - g).norm() / g.norm()) <= tol, name
    same = model.encode(x.float())
    assert torch.equal(same, out.detach())
    ops.check(0)


def test_training_and_an_index_of_its_logits():
    need_cuda()
    import synth
    from paper_2608_15438_gb300 import neuroute as nr
    from paper_2608_15438_gb300.builder import config
    from paper_2608_15438_gb300.residual import recall_at_10, train_residual

    w = synth.WORKLOADS["tiny"]
    x = synth.DeviceRows(w, synth.SEED_DATA, device=0).rows(0, 16384)
    last = {}
    for hold8 in (True, False):
        model, hist = train_residual(x, w.in_scale, 128, 2, 12, epochs=4, batch=2048, lr=1e-3, seed=1, hold8=hold8)
        assert hist[-1][1] < 0.5 * hist[0][1]
        last[hold8] = hist[-1][1]
    # held in 8 bits, the loss falls as it does in 16
    assert abs(last[True] / last[False] - 1.0) < 0.25
    n = x.shape[0]
    bd = nr.Builder(config(w.dtype, w.dim, w.hidden, 12, w.k_max, w.t), n,
                    tuple(synth.encoder_weights(w)[:2]) + tuple(a[:12] for a in synth.encoder_weights(w)[2:4]), 0)
    bd.set_logits(model.encode(x, w.in_scale), 0)
    torch.cuda.synchronize()
    bd.finish()
    bd.place(x, 0)
    ix = bd.end()
    qs = torch.from_numpy(synth.queries(w, 500)).cuda()
    ids, _ = ix.search_logits(qs, model.encode(qs, w.in_scale), 10, 4096, 4096)
    torch.cuda.synchronize()
    assert recall_at_10(qs, [x], ids, n) > 0.99  # every bucket probed, every cluster kept
    ids, _ = ix.search_logits(qs, model.encode(qs, w.in_scale), 10, 64, 256)
    torch.cuda.synchronize()
    assert recall_at_10(qs, [x], ids, n) > 0.5
    ix.close()
