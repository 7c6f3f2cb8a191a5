"""The vectors' gradients of the block norm where every sum is a whole number that fp32 holds: equality, so that
no row, group or block of rows can be lost. Statistics are given: whole means and deviations of one. The magnitudes of a
column's terms add up to less than 2^24 (asserted), so that fp32 sums in any order are exact."""
import pytest

from test_gpu_block import BF16, F16, F32, TYPES, gen, ops  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SIZES = [(1, 3), (5, 1), (40000, 48), (9001, 264), (9001, 387), (3001, 771), (2500, 1536), ((1 << 20) + 3, 64), (70001, 9),
         (1217, 2049), (4099, 3100), (701, 8192), (305, 6145), (303, 8200)]


def whole(g, m, n, dtype, most, pad=0):
    """[m x n] of whole numbers up to `most` in magnitude, at a pitch of n + pad."""
    return torch.randint(-most, most + 1, (m, n + pad), generator=g, device="cuda", dtype=torch.int8).to(dtype)[:, :n]


def column_sums(*factors):
    terms = factors[0].double()
    for f in factors[1:]:
        terms = terms * f.double()
    assert float(terms.abs().sum(0).max()) < 2 ** 24
    return terms.sum(0)


@pytest.mark.parametrize("m,n", SIZES)
@pytest.mark.parametrize("k", range(5))
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_before_the_next_block(ops, m, n, k, kind):  # noqa: F811
    dt, st = TYPES[k]
    g = gen(n + k)
    dh, y = whole(g, m, n, dt, 1, k % 3), whole(g, m, n, st, 2, k % 3)
    mean = whole(g, 1, m, F32, 1) if kind == "layer" else torch.zeros(1, m, device="cuda")
    stats = torch.cat([mean, torch.ones_like(mean)]) if kind == "layer" else torch.ones_like(mean)
    w, b = whole(g, 1, n, F32, 2)[0].clone(), whole(g, 1, n, F32, 2)[0].clone()
    want_w, want_b = column_sums(dh, y.double() - mean.t()), column_sums(dh)
    d = ops.block_norm_backward(dh, None, y, None, stats, pre=kind, weight=w, bias=b)
    assert torch.equal(d.weight.double(), want_w) and torch.equal(d.bias.double(), want_b)
    d = ops.block_norm_backward(dh, None, y, None, stats, pre=kind, weight=w)
    assert torch.equal(d.weight.double(), want_w)


@pytest.mark.parametrize("m,n", SIZES)
@pytest.mark.parametrize("k", range(5))
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_after_a_block(ops, m, n, k, kind):  # noqa: F811
    dt, st = TYPES[k]
    g = gen(n + k)
    vt = dt if k == 2 else F32
    dy, u = whole(g, m, n, st, 1, k % 3), whole(g, m, n, dt, 2, k % 3)
    mean = whole(g, 1, m, F32, 1) if kind == "layer" else torch.zeros(1, m, device="cuda")
    stats = torch.cat([mean, torch.ones_like(mean)]) if kind == "layer" else torch.ones_like(mean)
    pw, pb, scale = (whole(g, 1, n, vt, 2)[0].clone() for _ in range(3))
    A, S = column_sums(dy, u.double() - mean.t()), column_sums(dy)
    want = {"scale": pw.double() * A + pb.double() * S, "post_weight": scale.double() * A, "post_bias": scale.double() * S}
    assert max(float(w.abs().max()) for w in want.values()) < 2 ** 24
    d = ops.block_norm_backward(None, dy, None, u, stats, scale=scale, post=kind, post_weight=pw, post_bias=pb, pre="none")
    for name, v in want.items():
        assert torch.equal(getattr(d, name), v.to(vt)), name
    d = ops.block_norm_backward(None, dy, None, u, stats, scale=scale, post=kind, post_weight=pw, pre="none")
    assert torch.equal(d.scale, (pw.double() * A).to(vt)) and torch.equal(d.post_weight, want["post_weight"].to(vt))


def test_rows_past_two_to_the_32_bytes(ops):  # noqa: F811
    m, n, part = (1 << 25) + 7, 64, 1 << 22
    g = gen(1)
    dh, y = whole(g, m, n, BF16, 1), whole(g, m, n, BF16, 1)
    dh[1::3] = 0.0
    want, most = torch.zeros(2, n, dtype=torch.float64, device="cuda"), torch.zeros(2, n, dtype=torch.float64, device="cuda")
    for s in range(0, m, part):
        a, b = dh[s:s + part].double(), y[s:s + part].double()
        for k, t in enumerate((a * b, a)):
            want[k] += t.sum(0)
            most[k] += t.abs().sum(0)
    assert float(most.max()) < 2 ** 24
    ones = torch.ones(n, device="cuda")
    d = ops.block_norm_backward(dh, None, y, None, torch.ones(1, m, device="cuda"), pre="rms", weight=ones, bias=ones)
    assert torch.equal(d.weight.double(), want[0]) and torch.equal(d.bias.double(), want[1])
