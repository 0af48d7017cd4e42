"""Activations next to the largest bfloat16: 127 steps of their group may lie past it, and are read back as it, not as infinity."""
import pytest
import torch

from paper_2502_01703_amd import binding as Q
import plain_gradients as plain

pytestmark = pytest.mark.gpu
DEV = "cuda"
MOST = torch.finfo(torch.bfloat16).max


def _say(msg):
    print("[case] " + msg, flush=True)


def _inputs(T, D, seed):
    """Groups whose largest value is one of the 20 largest bfloat16 numbers, of either sign."""
    g = torch.Generator().manual_seed(seed)
    X = torch.randn(T, D, generator=g) * 1e37
    top = (torch.tensor(MOST).bfloat16().view(torch.int16) - torch.randint(0, 20, (T, -(-D // 128)), generator=g)).to(torch.int16).view(torch.bfloat16).float()
    sign = torch.randint(0, 2, top.shape, generator=g) * 2.0 - 1
    for group in range(top.shape[1]):
        X[:, group * 128 + (7 * group) % 5] = top[:, group] * sign[:, group]
    return X.bfloat16()


@pytest.mark.parametrize("T,D", [(64, 256), (33, 133)])
def test_the_largest_numbers_are_read_back(T, D):
    _say("largest activations T=%d D=%d" % (T, D))
    X = _inputs(T, D, T)
    codes, steps = plain.checkpoint(X)
    q, s = Q.checkpoint8(X.to(DEV))
    assert torch.equal(q.cpu().long(), codes) and torch.equal(s.cpu().double(), steps)
    v = plain.values(codes, steps)
    assert (v.abs() > MOST).any(), "the groups are what the test is about"
    assert torch.equal(Q.checkpoint8_read(q, s, torch.float32).cpu(), v.float())
    assert torch.equal(Q.checkpoint8_read(q, s).cpu(), v.clamp(-MOST, MOST).bfloat16())


def test_the_largest_numbers_in_gradients():
    """Expanded activations (many rows, bfloat16 results) and codes as they are; bounds as derived in test_gpu_checkpoint.py (127.5 u for
    127.99 u is within the rounding to bfloat16 that they allow)."""
    T, D, R = 600, 4096, 4096
    codes, steps = Q.checkpoint8(_inputs(T, D, 5).to(DEV))
    y = (torch.randn(T, R, generator=torch.Generator().manual_seed(6)) * 1e-30).bfloat16().to(DEV)
    x = codes.double() * steps.double().repeat_interleave(Q.CHECKPOINT_GROUP, 1)
    ends = torch.tensor([0, T], device=DEV)
    ref, size = torch.mm(y.double().t().contiguous(), x), torch.mm(y.double().abs().t().contiguous(), x.abs())
    for dtype in (torch.bfloat16, torch.float32):
        _say("gradient of the largest activations %s" % dtype)
        G = Q.checkpoint8_grad(y, codes, steps, ends, dtype=dtype)[0].double()
        bound = (T + 64) * 2.0 ** -23 * size
        if dtype == torch.bfloat16:
            bound = bound + 2.0 ** -8 * size * (1 + 2.0 ** -8) + 2.0 ** -8 * ref.abs()
        assert ((G - ref).abs() <= bound).all()
