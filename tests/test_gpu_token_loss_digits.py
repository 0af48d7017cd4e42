"""Tokens whose target is all but certain: the loss, 1 - p(target) and with it the gradients keep their digits on every path.

Bounds.  With o = sum of exp(z - z_target) over the other entries, nll = log(1 + o) and 1 - p(target) = o / (1 + o).  The logits of a
token are each within ez = (D + 64) 2^-23 max_v sum_d |h w| of their value, so that a term of o is relative e^(2 ez) - 1 <=
2 ez (1 + 2 ez) off for 2 ez <= 1; exponentials of rounded arguments and the sums of fewer than 200 additions on any path add less than 2^-12.  So nll, an entry of
delta and 1 - p(target) are relative `rel` = 2 ez (1 + 2 ez) + 2^-12 off at most (their denominators 1 + o by less than that of o), delta's other entries by 2^-8 more where they are rounded
to bfloat16; a gradient sums these, its fp32 sums' (count of terms + 64) 2^-23 of the terms, and 2^-8 of the result."""
import pytest
import torch

from paper_2502_01703_amd import binding as Q
from test_gpu_token_loss import _say

pytestmark = pytest.mark.gpu
DEV = "cuda"
WANT = [(False, False), (True, False), (False, True), (True, True)]


def _confident(T, D, V, c, seed):
    """Each token's target stands c above the mean of the other logits, which are c / sqrt(D) wide; targets all differ."""
    g = torch.Generator().manual_seed(seed)
    W = torch.randn(V, D, generator=g)
    W = W / W.norm(dim=1, keepdim=True)
    y = torch.randperm(V, generator=g)[:T]
    return (c * W[y]).bfloat16().to(DEV), W.bfloat16().to(DEV), y.to(DEV), (torch.rand(T, generator=g) + 0.5).to(DEV)


def _check_small(H, W, y, w, got, least, most):
    nll, lse, dH, dW = got
    h, W64, at = H.double(), W.double(), y[:, None]
    D, V = W.shape[1], W.shape[0]
    z = torch.mm(h, W64.t().contiguous())
    ez = (D + 64) * 2.0 ** -23 * torch.mm(h.abs(), W64.abs().t().contiguous()).amax(1)
    assert (2 * ez <= 1).all()
    rel = 2 * ez * (1 + 2 * ez) + 2.0 ** -12
    o = torch.exp(z - z.gather(1, at)).scatter_(1, at, 0.0)
    total = o.sum(1)
    ref = torch.log1p(total)
    assert (ref > least).all() and (ref < most).all(), "the tokens are what the test is about"
    assert ((nll.double() - ref).abs() <= ref * rel).all()
    ref_lse = torch.logsumexp(z, 1)
    assert ((lse.double() - ref_lse).abs() <= ez + 2.0 ** -15 + 2.0 ** -22 * ref_lse.abs()).all()
    weight = w.double()[:, None]
    others = weight * o / (1 + total)[:, None]
    pull = weight[:, 0] * total / (1 + total)
    delta = others.scatter(1, at, -pull[:, None])
    off = others * (rel[:, None] + 2.0 ** -8)
    off.scatter_(1, at, (pull * rel)[:, None])
    if dH is not None:
        r = torch.mm(delta, W64)
        bound = torch.mm(off, W64.abs()) + (V + 64) * 2.0 ** -23 * torch.mm(delta.abs() + off, W64.abs())
        assert ((dH.double() - r).abs() <= bound + 2.0 ** -8 * (r.abs() + bound)).all()
    if dW is not None:
        r = torch.mm(delta.t().contiguous(), h)
        bound = torch.mm(off.t().contiguous(), h.abs()) + (len(y) + 64) * 2.0 ** -23 * torch.mm((delta.abs() + off).t().contiguous(), h.abs())
        assert ((dW.double() - r).abs() <= bound + 2.0 ** -8 * (r.abs() + bound)).all()


# one pass of few tokens, tiles, D in parts (100 x 2048, 300 x 2056), W packed (odd D), dW in one pass or two
@pytest.mark.parametrize("T,D,V", [(1, 256, 1000), (2, 1024, 3000), (4, 256, 1000), (4, 4096, 2000), (20, 256, 1000), (30, 257, 1000), (60, 512, 2000), (100, 2048, 2000),
                                   (130, 256, 1000), (300, 2056, 1500), (400, 256, 1000), (400, 301, 1000)])
@pytest.mark.parametrize("c", [13.0, 17.0, 21.0, 26.0])
def test_small_losses_keep_their_digits(T, D, V, c):
    _say("small losses T=%d D=%d V=%d c=%g" % (T, D, V, c))
    H, W, y, w = _confident(T, D, V, c, T + D)
    for want in WANT:
        _check_small(H, W, y, w, Q.token_loss(H, W, y, w, want_dH=want[0], want_dW=want[1]), 1e-11, 2e-2)


@pytest.mark.parametrize("c", [22.0, 30.0])
@pytest.mark.parametrize("T", [20, 40])
def test_small_losses_over_several_pieces(T, c):
    """More entries than a piece holds; a token's target stands out along a column of its own."""
    _say("small losses of millions of entries T=%d c=%g" % (T, c))
    g = torch.Generator().manual_seed(T)
    D, V = 48, 4300000
    W = torch.randn(V, D, generator=g) / 32
    y = torch.randperm(V, generator=g)[:T]
    W[y] = torch.eye(T, D)
    H = (c * torch.eye(T, D) + 0.1 * torch.randn(T, D, generator=g)).bfloat16().to(DEV)
    W, y, w = W.bfloat16().to(DEV), y.to(DEV), (torch.rand(T, generator=g) + 0.5).to(DEV)
    for want in WANT:
        _check_small(H, W, y, w, Q.token_loss(H, W, y, w, want_dH=want[0], want_dW=want[1]), 1e-11, 2e-2)
