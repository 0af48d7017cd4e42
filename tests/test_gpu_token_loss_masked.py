"""Batches in which no token has a target: every output is zeros, whatever the workspace held before."""
import pytest
import torch

from paper_2502_01703_amd import binding as Q
from test_gpu_token_loss import _check, _inputs, _say

pytestmark = pytest.mark.gpu
DEV = "cuda"
WANT = [(False, False), (True, False), (False, True), (True, True)]


# packed into several pieces; read in place; more entries than a piece holds; more tokens than two terms are kept for
@pytest.mark.parametrize("T,D,V", [(4, 1001, 50257), (30, 1001, 50257), (30, 512, 3000), (3, 8, 4300000), (20, 12, 4300000), (40, 1001, 9000), (200, 64, 3000)])
@pytest.mark.parametrize("want", WANT)
def test_no_target_in_any_token(T, D, V, want):
    _say("loss without targets T=%d D=%d V=%d dH=%s dW=%s" % (T, D, V, *want))
    H, W, y, w = _inputs(T, D, V, 21)
    ws = torch.full((Q.token_loss_workspace(T, D, V, *want),), 0xFF, dtype=torch.uint8, device=DEV)
    got = Q.token_loss(H, W, torch.full_like(y, -100), w, want_dH=want[0], want_dW=want[1], ws=ws)
    for x in got:
        assert x is None or (x == 0).all()


@pytest.mark.parametrize("T", [4, 30])
def test_a_micro_batch_without_targets_replayed(T):
    """Replays of one graph: a batch with targets, one without, and one with again; the workspace is spoiled in between."""
    D, V = 1001, 50257
    Q.init()
    held = _inputs(T, D, V, 22, masked=0.0)
    ws = torch.full((Q.token_loss_workspace(T, D, V, False, True),), 0xFF, dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        Q.token_loss(*held, want_dH=False, want_dW=True, ws=ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = Q.token_loss(*held, want_dH=False, want_dW=True, ws=ws)
    for i, masked in enumerate((0.0, 1.0, 0.5, 1.0)):
        _say("loss replay %d, %g of T=%d masked" % (i, masked, T))
        for a, b in zip(held, _inputs(T, D, V, 23 + i, masked=masked)):
            a.copy_(b)
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        _check(*held, out)
