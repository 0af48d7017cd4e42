"""The loss over the vocabulary and its gradients against their formulas in 64 bits.

Bounds.  A logit is a sum of D exact products added in fp32, each of at most D + 64 additions off by at most one step of a partial sum:
|error| <= ez = (D + 64) 2^-23 max_v sum_d |h w|.  A sum of exponentials is relative 2^-15 off at most (fewer than 200 additions on any
path, each 2^-23, and exponentials of arguments that were rounded), its logarithm as much absolutely: lse within ez + 2^-15 + 2^-22 |lse|,
nll within twice that (el).  A probability is then relative er = 3 (el + 2^-15) off, delta = weight (softmax - onehot) by that and by its
rounding to bfloat16, 2^-8 of itself; a gradient sums these errors, adds its own fp32 sums' (count of terms + 64) 2^-23 of the terms and
the rounding of the result, 2^-8 of it."""
import pytest
import torch

from paper_2502_01703_amd import binding as Q

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _say(msg):
    print("[case] " + msg, flush=True)


def _inside(X, left, right):
    wide = torch.full((X.shape[0], left + X.shape[1] + right), 7, dtype=X.dtype, device=DEV)
    wide[:, left:left + X.shape[1]] = X.to(DEV)
    return wide[:, left:left + X.shape[1]], wide


def _inputs(T, D, V, seed, masked=0.3, scale=4.0):
    g = torch.Generator().manual_seed(seed)
    W = torch.randn(V, D, generator=g) / D ** 0.5
    y = torch.randint(0, V, (T,), generator=g)
    H = torch.randn(T, D, generator=g) + 2 * scale * torch.rand(T, 1, generator=g) * W[y]
    out = torch.rand(T, generator=g) < masked
    y[out] = torch.tensor([-100, -1, V, 1 << 40])[torch.randint(0, 4, (int(out.sum()),), generator=g)]
    w = torch.rand(T, generator=g) - 0.2
    return H.bfloat16().to(DEV), W.bfloat16().to(DEV), y.to(DEV), w.to(DEV)


def _check(H, W, y, w, got):
    """All outputs of a call within the bounds above."""
    nll, lse, dH, dW = got
    live = ((y >= 0) & (y < W.shape[0])).nonzero()[:, 0]
    rest = torch.ones(len(y), dtype=torch.bool, device=DEV)
    rest[live] = False
    assert not nll[rest].any() and not lse[rest].any()
    assert dH is None or not dH[rest].any()
    if len(live) == 0:
        assert dW is None or not dW.any()
        return
    h, W64, t = H[live].double(), W.double(), y[live][:, None]
    D, V = W.shape[1], W.shape[0]
    z = torch.mm(h, W64.t().contiguous())
    ez = (D + 64) * 2.0 ** -23 * torch.mm(h.abs(), W64.abs().t().contiguous()).amax(1)
    ref_lse = torch.logsumexp(z, 1)
    ref = ref_lse - z.gather(1, t)[:, 0]
    el = 2 * (ez + 2.0 ** -15 + 2.0 ** -22 * ref_lse.abs())
    assert ((lse[live].double() - ref_lse).abs() <= el).all()
    assert ((nll[live].double() - ref).abs() <= el).all()
    if dH is None and dW is None:
        return
    er = 3 * (el + 2.0 ** -15)[:, None]
    weight = torch.ones(len(live), device=DEV, dtype=torch.float64) if w is None else w[live].double()
    p = torch.softmax(z, 1)
    hot = torch.zeros_like(p).scatter_(1, t, 1.0)
    delta = p.scatter(1, t, torch.special.expm1(-ref)[:, None]) * weight[:, None]
    off = 2.0 ** -8 * delta.abs() + weight.abs()[:, None] * (p + hot) * er * (1 + 2.0 ** -8)
    if dH is not None:
        r = torch.mm(delta, W64)
        bound = torch.mm(off, W64.abs()) + (V + 64) * 2.0 ** -23 * torch.mm(delta.abs() + off, W64.abs())
        assert ((dH[live].double() - r).abs() <= bound + 2.0 ** -8 * (r.abs() + bound)).all()
    if dW is not None:
        r = torch.mm(delta.t().contiguous(), h)
        bound = torch.mm(off.t().contiguous(), h.abs()) + (len(live) + 64) * 2.0 ** -23 * torch.mm((delta.abs() + off).t().contiguous(), h.abs())
        assert ((dW.double() - r).abs() <= bound + 2.0 ** -8 * (r.abs() + bound)).all()


SIZES = [(1, 1, 1), (1, 64, 2), (1, 8, 1000), (2, 72, 257), (1, 4096, 300), (31, 100, 256), (32, 128, 2049), (33, 520, 255), (257, 129, 1000), (300, 64, 513),
         (300, 264, 3001), (513, 8, 700), (64, 1000, 5000), (200, 4104, 700), (513, 2056, 1000), (700, 72, 100), (150, 640, 9000)]


@pytest.mark.parametrize("T,D,V", SIZES)
@pytest.mark.parametrize("pads", [(0, 0), (8, 16), (3, 1)])
def test_loss_and_gradients(T, D, V, pads):
    _say("loss T=%d D=%d V=%d pads=%s" % (T, D, V, pads))
    H, W, y, w = _inputs(T, D, V, T + D + V, masked=0.0 if T == 1 else 0.3)
    h, _ = _inside(H, pads[0], 1 if pads[0] else 0)
    W_, _ = _inside(W, pads[1], 0)
    dH, wideH = _inside(torch.zeros_like(H), pads[1], 2)
    dW, wideW = _inside(torch.zeros_like(W), pads[0], 2)
    ws = torch.full((Q.token_loss_workspace(T, D, V, True, True),), 0xFF, dtype=torch.uint8, device=DEV)     # NaN wherever it is read unwritten
    got = Q.token_loss(h, W_, y, w, dH=dH, dW=dW, ws=ws)
    _check(H, W, y, w, got)
    for wide, left, n in ((wideH, pads[1], D), (wideW, pads[0], D)):         # what lies beside the rows stays
        assert (wide[:, :left] == 7).all() and (wide[:, left + n:] == 7).all()
    # each output alone (which outputs are asked for decides in what order a sum of exponentials is joined), and without weights
    for want in ((False, False), (True, False), (False, True)):
        alone = Q.token_loss(h, W_, y, w, want_dH=want[0], want_dW=want[1])
        _check(H, W, y, w, alone)
        for a, b in zip(alone, Q.token_loss(h, W_, y, w, want_dH=want[0], want_dW=want[1])):
            assert a is None or torch.equal(a, b)
    _check(H, W, y, None, Q.token_loss(h, W_, y))


@pytest.mark.parametrize("T,D,V", [(1, 8, 1), (1, 64, 7), (1, 2048, 5000), (1, 2056, 3001), (1, 4104, 1500), (1, 8192, 4097), (1, 8200, 600), (2, 200, 4000),
                                   (2, 4096, 2500), (2, 8192, 1025), (3, 1000, 9000), (4, 2048, 2049), (4, 4096, 1000), (4, 4104, 800), (4, 16, 200000)])
@pytest.mark.parametrize("pads", [(0, 0), (3, 8)])
def test_up_to_four_tokens(T, D, V, pads):
    _say("loss of few T=%d D=%d V=%d pads=%s" % (T, D, V, pads))
    H, W, y, w = _inputs(T, D, V, T + D + V, masked=0.0)
    h, _ = _inside(H, pads[0], 0)
    W_, _ = _inside(W, pads[1], 0)
    dH, wide = _inside(torch.zeros_like(H), pads[0], 2)
    ws = torch.full((Q.token_loss_workspace(T, D, V),), 0xFF, dtype=torch.uint8, device=DEV)
    got = Q.token_loss(h, W_, y, w, dH=dH, ws=ws)
    _check(H, W, y, w, got)
    assert (wide[:, :pads[0]] == 7).all() and (wide[:, pads[0] + D:] == 7).all()
    for t in range(T):                                # each left out once, its row not a number
        z = y.clone()
        z[t] = (-100, V, 1 << 40, -1)[t]
        g = H.clone()
        g[t] = float("nan")
        _check(H, W, z, None, Q.token_loss(g, W_, z))
    for v in (0, V - 1):                              # targets at the ends
        _check(H, W, torch.full_like(y, v), w, Q.token_loss(h, W_, torch.full_like(y, v), w))
    if T > 1:
        g = H.clone()
        g[1, 0] = float("inf")
        spoiled = Q.token_loss(g, W_, y, w)
        good = torch.arange(T, device=DEV) != 1
        for a, b in zip(got[:3], spoiled[:3]):
            assert torch.equal(a[good], b[good])
        assert not spoiled[0][1].isfinite() and not spoiled[2][1].isfinite().any()


@pytest.mark.parametrize("T,D,V", [(9000, 40, 30000), (8192, 64, 20000), (1, 4100, 20000), (30, 4100, 20000), (2000, 72, 70000), (700, 100, 150000)])
def test_pieces_of_the_vocabulary(T, D, V):
    """More vocabulary than a piece holds, read in place and packed."""
    _say("loss pieces T=%d D=%d V=%d" % (T, D, V))
    H, W, y, w = _inputs(T, D, V, V, masked=0.2 if T > 1 else 0.0)
    _check(H, W, y, w, Q.token_loss(H, W, y, w, want_dW=True))


@pytest.mark.parametrize("want_dW", [False, True])
def test_pieces_read_in_place(want_dW):
    """Several pieces of a vocabulary that needs no packing, for dH alone and with dW."""
    _say("loss pieces read in place dW=%s" % want_dW)
    H, W, y, w = _inputs(9000, 40, 100000, 11, masked=0.2)
    _check(H, W, y, w, Q.token_loss(H, W, y, w, want_dW=want_dW))


@pytest.mark.parametrize("T,D,V", [(3, 16, 5000000), (40, 8, 5000000), (20, 12, 4300000)])
def test_millions_of_entries(T, D, V):
    """Rows of delta longer than 32-bit offsets reach over a tile: several pieces, also for few tokens."""
    _say("loss of millions of entries T=%d D=%d V=%d" % (T, D, V))
    H, W, y, w = _inputs(T, D, V, 13, masked=0.0)
    y[0], y[1] = 0, V - 1
    _check(H, W, y, w, Q.token_loss(H, W, y, w, want_dW=True))
    _check(H, W, y, w, Q.token_loss(H, W, y, w))


@pytest.mark.parametrize("T,D,V", [(130, 256, 1000), (700, 128, 9000), (9000, 40, 100000)])
@pytest.mark.parametrize("rise", [-1.0, 1.0])
def test_logits_that_rise_over_the_vocabulary(T, D, V, rise):
    """The greatest logit so far changes from part to part, by more than the range of an exponent over the whole."""
    _say("loss with rising logits T=%d rise=%g" % (T, rise))
    H, W, y, w = _inputs(T, D, V, 12, masked=0.2)
    H[:, 0] = torch.linspace(0, 8, T, device=DEV).bfloat16()
    W[:, 0] = (rise * torch.linspace(-40, 40, V, device=DEV)).bfloat16()
    _check(H, W, y, w, Q.token_loss(H, W, y, w))


@pytest.mark.parametrize("scale", [0.0, 60.0, 3000.0])
@pytest.mark.parametrize("T", [50, 400])
def test_certain_and_hopeless_tokens_for_dH(T, scale):
    _say("loss scale %g T=%d, dH alone" % (scale, T))
    H, W, y, w = _inputs(T, 256, 1000, 6, masked=0.1, scale=scale)
    H[::3] = -H[::3]
    _check(H, W, y, w, Q.token_loss(H, W, y, w))
    y[:] = 999
    _check(H, W, y, w, Q.token_loss(H, W, y, w))


@pytest.mark.parametrize("T,D,V", [(1, 64, 100), (2, 2048, 32000), (4, 4096, 1000), (20, 100, 150000), (40, 200, 5000), (100, 8192, 4000), (300, 264, 3001),
                                   (700, 100, 150000), (2000, 72, 70000), (9000, 40, 100000)])
@pytest.mark.parametrize("want", [(False, False), (True, False), (False, True), (True, True)])
def test_the_workspace_ends_where_it_says(T, D, V, want):
    _say("loss workspace T=%d D=%d V=%d dH=%s dW=%s" % (T, D, V, *want))
    H, W, y, w = _inputs(T, D, V, 14, masked=0.0)
    W, _ = _inside(W, 1, 0) if T % 3 == 0 else (W, None)              # packed, or read in place
    need = Q.token_loss_workspace(T, D, V, *want)
    ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device=DEV)
    got = Q.token_loss(H, W, y, w, want_dH=want[0], want_dW=want[1], ws=ws[:need])
    assert (ws[need:] == 0xFF).all()
    for x in got:
        assert x is None or x.isfinite().all()


@pytest.mark.parametrize("T", [3, 100])
def test_no_target_at_all(T):
    _say("loss without targets T=%d" % T)
    H, W, y, w = _inputs(T, 72, 300, 4)
    got = Q.token_loss(torch.full_like(H, float("nan")), W, torch.full_like(y, -100), torch.full_like(w, float("nan")), want_dW=True)
    for x in got:
        assert not x.any()
    empty = Q.token_loss(H[:0], W, y[:0], w[:0], want_dW=True)
    assert empty[0].shape == (0,) and empty[2].shape == (0, 72) and not empty[3].any()


def test_left_out_rows_are_not_read_as_numbers():
    _say("loss with NaN in rows that are left out")
    H, W, y, w = _inputs(290, 136, 777, 5, masked=0.6)
    want = Q.token_loss(H, W, y, w, want_dW=True)
    out = (y < 0) | (y >= 777)
    H[out], w[out] = float("nan"), float("inf")
    for a, b in zip(want, Q.token_loss(H, W, y, w, want_dW=True)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("scale", [0.0, 60.0, 3000.0])
def test_certain_and_hopeless_tokens(scale):
    """Losses of nearly nothing keep their digits, losses of thousands do not overflow."""
    _say("loss scale %g" % scale)
    H, W, y, w = _inputs(130, 256, 1000, 6, masked=0.1, scale=scale)
    H[::3] = -H[::3]
    _check(H, W, y, w, Q.token_loss(H, W, y, w, want_dW=True))


@pytest.mark.parametrize("T", [20, 700])
def test_tokens_of_the_same_target(T):
    """All, and all but a few, tokens have one target; entries at the ends of the vocabulary."""
    _say("loss with one target T=%d" % T)
    H, W, _, w = _inputs(T, 320, 1025, T, masked=0.0)
    for v in (0, 63, 64, 1024):
        y = torch.full((T,), v, device=DEV)
        _check(H, W, y, w, Q.token_loss(H, W, y, w, want_dW=True))
        y[::5] = torch.arange(len(y[::5]), device=DEV) % 1025
        y[3] = -100
        _check(H, W, y, w, Q.token_loss(H, W, y, w, want_dW=True))


def test_one_bad_token():
    """A token whose hidden state is not finite spoils its own loss and row only (and dW)."""
    _say("loss with one token not finite")
    H, W, y, w = _inputs(70, 64, 500, 7, masked=0.0)
    want = Q.token_loss(H, W, y, w)
    H[13, 5] = float("nan")
    got = Q.token_loss(H, W, y, w)
    good = torch.arange(70, device=DEV) != 13
    for a, b in zip(want[:3], got[:3]):
        assert torch.equal(a[good], b[good]) and b[13].isnan().all()


def test_gradient_against_differences():
    """dH and dW against differences of the summed loss along a direction."""
    _say("loss differences")
    H, W, y, w = _inputs(40, 96, 400, 8)
    _, _, dH, dW = Q.token_loss(H, W, y, w, want_dW=True)

    def L(h, W_):
        nll, _, _, _ = Q.token_loss(h, W_, y, w, want_dH=False)
        live = (y >= 0) & (y < 400)
        return (nll.double() * torch.where(live, w, torch.zeros_like(w)).double()).sum()
    # a step of bfloat16 numbers: H and W moved to neighbours along their gradients' signs
    for X, G, f in ((H, dH, lambda x: L(x, W)), (W, dW, lambda x: L(H, x))):
        up, down = (X.float() + 0.02 * X.float().abs() * G.float().sign()).bfloat16(), (X.float() - 0.02 * X.float().abs() * G.float().sign()).bfloat16()
        first = ((up.double() - down.double()) * G.double()).sum()
        d = (f(up) - f(down)).double()
        # the third derivative of a softmax along a step of logits of size s is at most s^3; logits move by at most s here
        s = 0.03 * torch.mm(H.float().abs(), W.float().abs().t().contiguous()).amax(1).double()
        slack = (w.abs().double() * s ** 3).sum() + 2.0 ** -7 * ((up.double() - down.double()) * G.double()).abs().sum() + 1e-3
        assert (d - first).abs() <= slack


def test_replayed_in_a_graph():
    _say("loss in a graph")
    Q.init()
    H, W, y, w = _inputs(70, 200, 1500, 9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        Q.token_loss(H, W, y, w, want_dW=True)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = Q.token_loss(H, W, y, w, want_dW=True)
    for i in range(4):
        _say("loss replay %d" % i)
        a, b, c, d = _inputs(70, 200, 1500, 10 + i, masked=0.25 * i)
        H.copy_(a), W.copy_(b), y.copy_(c), w.copy_(d)
        graph.replay()
        torch.cuda.synchronize()
        kept = [x.clone() for x in held]
        for p, q in zip(kept, Q.token_loss(H, W, y, w, want_dW=True)):
            assert torch.equal(p, q)


def test_other_stream_and_shared_workspace():
    """Calls in a row on one workspace, on a stream of their own."""
    _say("loss on another stream")
    ws = torch.full((Q.token_loss_workspace(300, 264, 3001, True, True),), 0xFF, dtype=torch.uint8, device=DEV)
    s = torch.cuda.Stream()
    for T, D, V in ((300, 264, 3001), (5, 64, 100), (33, 72, 1000)):
        H, W, y, w = _inputs(T, D, V, T)
        want = Q.token_loss(H, W, y, w, want_dW=True)
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got = Q.token_loss(H, W, y, w, want_dW=True, ws=ws)
        s.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a, b)


@pytest.mark.parametrize("T,want_dW", [(2, False), (20, True), (70, False), (1100, False), (1100, True)])
def test_other_kernels_replayed(T, want_dW):
    _say("loss replayed T=%d dW=%s" % (T, want_dW))
    Q.init()
    held = _inputs(T, 200, 1500, 9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        Q.token_loss(*held, want_dW=want_dW)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = Q.token_loss(*held, want_dW=want_dW)
    for i in range(3):
        for a, b in zip(held, _inputs(T, 200, 1500, 10 + i, masked=0.25 * i)):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        kept = [None if x is None else x.clone() for x in out]
        for p, q in zip(kept, Q.token_loss(*held, want_dW=want_dW)):
            assert (p is None and q is None) or torch.equal(p, q)


def test_calls_on_two_streams_at_once():
    """Each with a workspace of its own; results as of calls one after another."""
    _say("loss and checkpoints on two streams")
    sets = [_inputs(T, 264, 5000, T) for T in (700, 40)]
    ends = [torch.tensor([0, 13, len(x[0])], device=DEV) for x in sets]

    def call(x, e):
        got = Q.token_loss(*x, want_dW=True)
        return got + (Q.checkpoint8_grad(got[2], *Q.checkpoint8(x[0]), e),)
    want = [call(x, e) for x, e in zip(sets, ends)]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        for x, e, s in zip(sets, ends, streams):
            with torch.cuda.stream(s):
                got.append(call(x, e))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        for a, b in zip(want[i % 2], g):
            assert torch.equal(a, b)


@pytest.mark.parametrize("T,D,V", [(1, 8, 1), (1, 64, 7), (1, 2048, 5000), (1, 4104, 1500), (1, 8192, 4097), (1, 8200, 600), (1, 16, 200000), (2, 200, 4000), (2, 4096, 1001), (3, 1000, 3000),
                                   (4, 2048, 2049), (4, 4096, 1000), (4, 16, 100000)])
def test_loss_alone_of_few_tokens(T, D, V):
    _say("loss alone T=%d D=%d V=%d" % (T, D, V))
    H, W, y, w = _inputs(T, D, V, T + D + V, masked=0.0)
    for z in (y, torch.zeros_like(y), torch.full_like(y, V - 1), torch.full_like(y, -100)):
        ws = torch.full((Q.token_loss_workspace(T, D, V, False),), 0xFF, dtype=torch.uint8, device=DEV)
        _check(H, W, z, w, Q.token_loss(H, W, z, w, want_dH=False, ws=ws))
