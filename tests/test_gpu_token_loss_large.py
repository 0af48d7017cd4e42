"""The most tokens that a call takes, and more tiles of logits than a launch takes.  Bounds as derived in test_gpu_token_loss.py."""
import pytest
import torch

from paper_2502_01703_amd import binding as Q
from test_gpu_token_loss import _check, _say

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _many(T, D, V, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    W = (torch.randn(V, D, generator=g, device=DEV) / D ** 0.5).bfloat16()
    y = torch.randint(-1, V, (T,), generator=g, device=DEV)
    return torch.randn(T, D, generator=g, device=DEV).bfloat16(), W, y, torch.rand(T, generator=g, device=DEV)


def test_the_most_tokens():
    T, D, V = (1 << 24) - 256, 8, 40
    _say("loss of %d tokens" % T)
    H, W, y, w = _many(T, D, V, 1)
    nll, lse, dH, _ = Q.token_loss(H, W, y, w)
    step = 1 << 21
    for a in range(0, T, step):
        part = slice(a, a + step)
        _check(H[part], W, y[part], w[part], (nll[part], lse[part], dH[part], None))


@pytest.mark.parametrize("V", [1 << 17, (1 << 17) - 77])
def test_more_tiles_than_a_launch_takes(V):
    """The loss alone of 2^22 tokens: pieces of the vocabulary, whose parts lie beside each other."""
    T, D = 1 << 22, 8
    _say("loss of %d tokens, V=%d" % (T, V))
    H, W, y, w = _many(T, D, V, 2)
    y[5], y[T - 1], y[T - 2] = V - 1, 0, V - 300
    nll, lse, _, _ = Q.token_loss(H, W, y, w, want_dH=False)
    for part in (slice(0, 1500), slice(T // 2 - 700, T // 2 + 700), slice(T - 1500, T)):
        _check(H[part], W, y[part], w[part], (nll[part], lse[part], None, None))
