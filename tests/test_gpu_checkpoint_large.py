"""Checkpoints and gradients of more work items than a launch takes."""
import pytest
import torch

from paper_2502_01703_amd import binding as Q

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _say(msg):
    print("[case] " + msg, flush=True)


def _whole(X, places):
    """Written and read: every number within half a step (and the rounding of the type), groups at `places` as in a call for them alone."""
    codes, step = Q.checkpoint8(X)
    back = Q.checkpoint8_read(codes, step, X.dtype)
    assert int(codes.min()) >= -127
    for rows, cols in places:
        c, s = Q.checkpoint8(X[rows, cols].contiguous())
        first = cols.start // Q.CHECKPOINT_GROUP
        assert torch.equal(codes[rows, cols], c) and torch.equal(step[rows, first:first + s.shape[1]], s)
        assert torch.equal(back[rows, cols], Q.checkpoint8_read(c, s, X.dtype))
        x, b = X[rows, cols].double(), back[rows, cols].double()
        half = s.double().repeat_interleave(Q.CHECKPOINT_GROUP, 1)[:, :x.shape[1]] / 2
        assert ((x - b).abs() <= half + torch.finfo(X.dtype).eps / 2 * (x.abs() + half)).all()


def test_more_rows_than_a_launch_takes():
    T = (1 << 29) + 1001
    _say("checkpoint of %d rows" % T)
    X = torch.randn(T, 1, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV, dtype=torch.bfloat16)
    edge = 32 * ((1 << 24) - 1)
    _whole(X, [(slice(a, b), slice(0, 1)) for a, b in ((0, 5000), (edge - 3000, edge + 3000), (T - 2000, T))])


def test_the_longest_row():
    D = (1 << 31) - 1
    _say("checkpoint of a row of %d" % D)
    X = torch.empty(1, D, device=DEV, dtype=torch.bfloat16)
    g = torch.Generator(device=DEV).manual_seed(2)
    for a in range(0, D, 1 << 28):
        X[:, a:a + (1 << 28)].normal_(generator=g)
    _whole(X, [(slice(0, 1), slice(a, b)) for a, b in ((0, 12800), ((1 << 30) - 1280, (1 << 30) + 1280), (D - 127 - 1280, D))])
