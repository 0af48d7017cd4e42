"""The loss over the vocabulary, without a GPU: what the entry point refuses."""
import ctypes
import random

from paper_2502_01703_amd import binding

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
one = ctypes.c_void_p(16)           # never dereferenced: every call below ends on the host


def test_refusals():
    L = binding.lib()

    def call(H=one, ldH=64, W=one, ldW=64, dt=1, T=4, D=64, V=100, target=one, weight=None, nll=one, lse=None, dH=one, ldDH=64, dW=one, ldDW=64,
             ws=one, wsb=1 << 40):
        return L.qless_token_loss(H, ldH, W, ldW, dt, T, D, V, target, weight, nll, lse, dH, ldDH, dW, ldDW, ws, wsb, None)
    for bad in (dict(T=-1), dict(D=0), dict(V=0), dict(ldH=63), dict(ldW=63), dict(ldDH=63), dict(ldDW=63), dict(H=None), dict(W=None),
                dict(target=None), dict(nll=None)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(dt=0), dict(dt=2), dict(D=65537, ldH=65537, ldW=65537, ldDH=65537, ldDW=65537), dict(T=1 << 30)):
        assert call(**bad) == UNSUPPORTED, bad
    need = L.qless_token_loss_workspace(4, 64, 100, 1, 1)
    assert need > L.qless_token_loss_workspace(4, 64, 100, 1, 0) > L.qless_token_loss_workspace(4, 64, 100, 0, 0) > 0
    for bad in (dict(wsb=need - 1), dict(ws=None), dict(ws=ctypes.c_void_p(24))):
        assert call(**bad) == WORKSPACE, bad
    assert call(T=0, dW=None, H=None, target=None, nll=None, ws=None, wsb=0) == OK
    for shape in ((-1, 64, 100, 1, 1), (4, 0, 100, 1, 1), (4, 64, 0, 1, 1)):
        assert L.qless_token_loss_workspace(*shape) == 0


def test_workspace_does_not_hold_the_logits():
    L = binding.lib()
    T, D, V = 65536, 4096, 131072
    assert L.qless_token_loss_workspace(T, D, V, 1, 1) < T * V * 2 // 4


def test_vocabularies_that_32_bits_do_not_count_are_refused():
    L = binding.lib()
    for V in (1 << 30, (1 << 31) - 1):
        for T in (1, 100):
            assert L.qless_token_loss(one, 64, one, 64, 1, T, 64, V, one, None, one, None, one, 64, None, 0, one, 1 << 62, None) == UNSUPPORTED


def test_a_workspace_for_more_outputs_serves_fewer():
    L = binding.lib()
    for T, D, V in ((1, 64, 100), (1, 4096, 32000), (2, 8192, 7), (4, 4096, 1000), (31, 100, 5000), (40, 8192, 4000), (300, 264, 3001), (9000, 40, 100000)):
        loss, dH, dW, both = (L.qless_token_loss_workspace(T, D, V, *want) for want in ((0, 0), (1, 0), (0, 1), (1, 1)))
        assert 0 < loss <= dH <= both and loss <= dW <= both


def test_a_workspace_for_more_outputs_serves_fewer_at_random_sizes():
    L, r = binding.lib(), random.Random(1)
    for _ in range(5000):
        T, D, V = (int(2 ** r.uniform(0, top)) for top in (17, 13, 19))
        loss, dH, dW, both = (L.qless_token_loss_workspace(T, D, V, *want) for want in ((0, 0), (1, 0), (0, 1), (1, 1)))
        assert 0 < loss <= dH <= both and loss <= dW <= both, (T, D, V)


def test_more_tokens_than_a_launch_takes_are_refused():
    """256 threads a token, of fewer than 2^32; tiles of 256 x 256 of dH, of 512 threads."""
    L = binding.lib()

    def status(T, D, dH, dW):
        return L.qless_token_loss(one, D, one, D, 1, T, D, 100, one, None, one, None, dH, D, dW, D, None, 0, None)
    most = (1 << 24) - 256
    for T, D in ((most + 1, 8), (1 << 24, 64), ((1 << 30) - 1, 8), (1 << 23, 65536), (most, 32769)):
        for dH, dW in ((None, None), (one, None), (None, one), (one, one)):
            assert status(T, D, dH, dW) == UNSUPPORTED, (T, D)
            assert L.qless_token_loss_workspace(T, D, 100, dH is not None, dW is not None) == 0
    for T, D in ((most, 8), (most, 32000), (1 << 22, 65536)):
        assert status(T, D, one, None) == WORKSPACE
        assert L.qless_token_loss_workspace(T, D, 100, 1, 0) > 0
