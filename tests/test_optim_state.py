"""What optim.AdamW takes over of a saved state, without a GPU: tensors that say they are on one."""
import copy

import pytest
import torch

from paper_2608_15438_gb300.optim import AdamW


@pytest.fixture(autouse=True)
def on_a_device(monkeypatch):
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True))
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)


def over(*shapes, **kw):
    opt = AdamW([torch.nn.Parameter(torch.zeros(s)) for s in shapes], **kw)
    if opt.state.bits == 32:
        opt.state.m.copy_(torch.arange(opt.state.size))
    opt.state.step.fill_(3)
    return opt


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("mine,theirs", [([64, 32], [32, 64]), ([40], [50]), ([1, 33], [32, 40]), ([(8, 4)], [(4, 8)]), ([32], [(32, 1)]),
                                         ([32, 0], [0, 32]), ([32], [32, 0])], ids=str)
def test_a_state_of_other_tensors_is_refused(mine, theirs, bits):
    opt, saved = over(*mine, bits=bits), over(*theirs, bits=bits).state_dict()
    kept = copy.deepcopy(opt.state_dict())
    with pytest.raises(ValueError, match="other sizes"):
        opt.load_state_dict(saved)
    now = opt.state_dict()
    for k in ("m", "v"):
        for a, b in zip([kept[k]] if bits == 32 else kept[k], [now[k]] if bits == 32 else now[k]):
            assert torch.equal(a, b)
    assert int(now["step"]) == 3


def test_a_state_of_the_same_tensors_is_taken():
    a, b = over((8, 4), 5, lr=3.0), over((8, 4), 5, lr=1.0)
    a.state.m.mul_(2.0)
    b.load_state_dict(copy.deepcopy(a.state_dict()))
    assert torch.equal(a.state.m, b.state.m) and b.lr == 3.0
    saved = a.state_dict()
    del saved["shapes"]  # saved before shapes were: held to the sum of sizes
    b.load_state_dict(saved)
    with pytest.raises(ValueError, match="other sizes"):
        over(100).load_state_dict(saved)


def test_masters_of_fp32_tensors_are_refused():
    """They hold the values of the state's first day."""
    def of(*types):
        return AdamW([torch.nn.Parameter(torch.zeros(32, dtype=t)) for t in types])

    F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
    of(BF16, F32).load_state_dict(of(BF16, F32).state_dict())
    of(F16, F32).load_state_dict(of(BF16, BF16).state_dict())
    with pytest.raises(ValueError, match="masters"):
        of(BF16, BF16).load_state_dict(of(BF16, F32).state_dict())
    of(F32, F32).load_state_dict(of(F32, F32).state_dict())


def test_settings_are_copies():
    """Neither optimizer sees what is set on the other afterwards; a rate in a tensor, which a captured step reads, stays
    where it is."""
    a, b = over((8, 4), 5, weight_decay=0.1, lr=torch.tensor([1e-3])), over((8, 4), 5, lr=5.0)
    saved = a.state_dict()
    b.load_state_dict(saved)
    assert b.weight_decay == [0.1, 0.0] and float(b.lr) == float(torch.tensor(1e-3))
    a.weight_decay[0], b.weight_decay[1] = 0.7, 0.3
    a.lr.fill_(9.0)
    assert saved["weight_decay"] == [0.1, 0.0]
    assert (a.weight_decay, b.weight_decay) == ([0.7, 0.0], [0.1, 0.3]) and float(b.lr) < 1.0
    at = b.lr
    b.load_state_dict(a.state_dict())
    assert b.lr is at and float(at) == 9.0
    b.load_state_dict(over((8, 4), 5, lr=2.0).state_dict())
    assert b.lr == 2.0
