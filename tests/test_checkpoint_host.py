"""8-bit activation checkpoints, without a GPU: what the entry points refuse, and the plain form the GPU tests compare with."""
import ctypes
import math

import pytest
import torch

from paper_2502_01703_amd import binding
import plain_gradients as plain

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
one = ctypes.c_void_p(16)           # never dereferenced: every call below ends on the host


def test_write_and_read_refusals():
    L = binding.lib()
    w, r = L.qless_checkpoint8, L.qless_checkpoint8_read
    assert w(one, 1, -1, 64, 64, one, 64, one, 1, None) == INVALID
    assert w(one, 1, 4, 0, 64, one, 64, one, 1, None) == INVALID
    assert w(one, 1, 4, 64, 63, one, 64, one, 1, None) == INVALID
    assert w(one, 1, 4, 64, 64, one, 63, one, 1, None) == INVALID
    assert w(one, 1, 4, 129, 129, one, 129, one, 1, None) == INVALID
    assert w(one, 2, 4, 64, 64, one, 64, one, 1, None) == UNSUPPORTED
    for null in range(3):
        p = [one, one, one]
        p[null] = None
        assert w(p[0], 1, 4, 64, 64, p[1], 64, p[2], 1, None) == INVALID
        assert r(p[1], 64, p[2], 1, 4, 64, p[0], 1, 64, None) == INVALID
    assert r(one, 64, one, 1, 4, 64, one, 1, 63, None) == INVALID
    assert r(one, 64, one, 1, 4, 64, one, 5, 64, None) == UNSUPPORTED
    assert w(None, 1, 0, 64, 0, None, 0, None, 0, None) == OK
    assert r(None, 0, None, 0, 0, 64, None, 0, 0, None) == OK


def test_gradient_refusals():
    L = binding.lib()
    f = L.qless_checkpoint8_grad

    def call(dY=one, dtY=1, ldY=16, R=16, codes=one, ldC=256, step=one, ldS=2, D=256, T=100, off=one, n=3, G=one, dtG=0, ldG=4096, ws=one, wsb=1 << 40):
        return f(dY, dtY, ldY, R, codes, ldC, step, ldS, D, T, off, n, G, dtG, ldG, ws, wsb, None)
    for bad in (dict(R=0), dict(n=-1), dict(T=-1), dict(D=0), dict(ldY=15), dict(ldC=255), dict(ldS=1), dict(ldG=4095), dict(dY=None),
                dict(codes=None), dict(step=None), dict(off=None), dict(G=None)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(dtY=2), dict(dtG=7), dict(n=65536)):
        assert call(**bad) == UNSUPPORTED, bad
    long = dict(T=100000, n=1)
    need = L.qless_checkpoint8_grad_workspace(100000, 1, 16, 256)
    assert need > 0
    assert call(wsb=need - 1, **long) == WORKSPACE
    assert call(ws=None, wsb=need, **long) == WORKSPACE
    assert call(ws=ctypes.c_void_p(8), wsb=need, **long) == WORKSPACE
    assert call(n=0, G=None, off=None) == OK
    for shape in ((-1, 1, 16, 256), (10, 0, 16, 256), (10, 1, 0, 256), (10, 1, 16, 0)):
        assert L.qless_checkpoint8_grad_workspace(*shape) == 0


def test_plain_steps():
    assert plain.step_of(127.0) == 1.0 and plain.step_of(254.0) == 2.0 and plain.step_of(0.0) == 0.0
    assert plain.step_of(127.0 * (1 + 2.0 ** -23)) == 1 + 2.0 ** -7
    assert plain.step_of(1e-40) == 2.0 ** -126
    assert math.isnan(plain.step_of(float("inf"))) and math.isnan(plain.step_of(float("nan")))
    for top in torch.rand(200, generator=torch.Generator().manual_seed(1)).tolist():
        s = plain.step_of(top)
        m = math.frexp(s)[0] * 256
        assert m == int(m) and 127 * s >= top
        assert 127 * (s - 2.0 ** (math.frexp(s)[1] - 8)) < top or m == 128


def test_plain_codes_round_to_even():
    X = torch.tensor([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, 126.5, 0.4999999]])
    codes, steps = plain.checkpoint(X)
    assert steps.item() == 1.0 and codes.tolist() == [[127, 0, 2, 2, 0, -2, 126, 0]]


def test_gradient_sizes_that_32_bits_do_not_count_are_refused():
    """Rows and columns up to 2^30, fewer than 2^24 tiles of an example, tensors of up to 2^40 numbers; what is refused asks for no workspace."""
    L = binding.lib()

    def status(T, n, R, D):
        return L.qless_checkpoint8_grad(one, 1, R, R, one, D, one, -(-D // 128), D, T, one, n, one, 0, R * D, None, 0, None)
    for T, n, R, D in ((1, 1, (1 << 30) + 1, 1), (1, 1, (1 << 31) - 1, 1), (1, 1, 1, (1 << 30) + 1), (1, 1, 1, (1 << 31) - 1), (100, 2, (1 << 31) - 1, (1 << 31) - 1),
                       (10, 1, 1 << 21, 1 << 20), (1, 1, 1 << 30, 1), (1, 1, 1 << 29, 129), (1 << 30, 1, 1 << 11, 16), (1 << 30, 1, 16, 1 << 11), ((1 << 40) + 1, 1, 1, 1), (1 << 62, 1, 1, 1)):
        assert status(T, n, R, D) == UNSUPPORTED, (T, n, R, D)
        assert L.qless_checkpoint8_grad_workspace(T, n, R, D) == 0, (T, n, R, D)
    for T, n, R, D in ((1 << 40, 1, 1, 1), (1 << 30, 1, 1 << 10, 1 << 10)):
        assert L.qless_checkpoint8_grad_workspace(T, n, R, D) > 0
        assert status(T, n, R, D) == WORKSPACE, (T, n, R, D)
