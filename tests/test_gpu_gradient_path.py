"""The operators that make gradient rows, together as a run uses them: the loss of a batch of ragged examples and its gradient with
respect to the last hidden states, an adapter's inputs kept in 8 bits from the forward pass, the adapter's weight gradients written
beside each other into rows, the rows projected and quantised into a datastore, and the datastore scored.

An adapter (A, B) of rank r adds B A x to the last hidden states: dU = dH B, dB = sum dH_t u_t^T, dA = sum dU_t x_t^T with u = A x.
The gradients' bounds are the sums of what each step may leave: of dH what a rounding of delta (2^-8), of the result (2^-8) and the
logits' sums of D terms may; of dU a rounding to bfloat16 more; of x and u half a step, and the fp32 additions of L terms."""
import numpy as np
import pytest
import torch

import oracle
from paper_2502_01703_amd import binding as Q

pytestmark = pytest.mark.gpu
DEV = "cuda"
D, V, R, K = 256, 1000, 16, 512


def _say(msg):
    print("[case] " + msg, flush=True)


def _batch(lengths, seed):
    """Examples' inputs, targets (a prompt of a third left out, the example at index 2 wholly) and their mean's weights."""
    g = torch.Generator().manual_seed(seed)
    ends = torch.tensor([0] + list(np.cumsum(lengths)))
    T = int(ends[-1])
    X = (torch.randn(T, D, generator=g) * torch.exp(torch.randn(1, D, generator=g))).bfloat16()
    y = torch.randint(0, V, (T,), generator=g)
    w = torch.zeros(T)
    for e, n in enumerate(lengths):
        a = int(ends[e])
        y[a:a + (n if e == 2 else n // 3)] = -100
        live = int((y[a:a + n] >= 0).sum())
        w[a:a + n] = 1.0 / max(live, 1)
    return X.to(DEV), y.to(DEV), w.to(DEV), ends.to(DEV)


def _model(seed):
    g = torch.Generator().manual_seed(seed)
    A, B = torch.randn(R, D, generator=g) / 16, torch.randn(D, R, generator=g) / 4
    base, head = torch.randn(D, D, generator=g) / 16, torch.randn(V, D, generator=g) / 8
    return [x.bfloat16().to(DEV) for x in (A, B, base, head)]


def _rows(model, X, y, w, ends):
    """Gradient rows [n, 2 R D] as bfloat16, dA beside dB, and what they were made of."""
    A, B, base, head = model
    n = len(ends) - 1
    U = torch.mm(X, A.t())
    H = torch.mm(X, base.t()) + torch.mm(U, B.t())
    xq, xs = Q.checkpoint8(X)
    uq, us = Q.checkpoint8(U)
    nll, _, dH, _ = Q.token_loss(H, head, y, w)
    dU = torch.mm(dH, B)
    G = torch.empty(n, 2 * R * D, dtype=torch.bfloat16, device=DEV)
    Q.checkpoint8_grad(dU, xq, xs, ends, out=G[:, :R * D])
    Q.checkpoint8_grad(dH, uq, us, ends, out=G[:, R * D:])
    return G, (nll, U, H, xs, us)


def _check_rows(model, X, y, w, ends, G, made):
    """The rows against the formulas in 64 bits, from the same H and U."""
    A, B, _, head = [x.double() for x in model]
    nll, U, H, xs, us = made
    x, u, h = X.double(), U.double(), H.double()
    live = y >= 0
    z = torch.mm(h, head.t().contiguous())
    at = y.clamp(min=0)[:, None]
    weight = torch.where(live, w, torch.zeros_like(w)).double()[:, None]
    p = torch.softmax(z, 1)
    ref = torch.logsumexp(z, 1) - z.gather(1, at)[:, 0]
    ez = (D + 64) * 2.0 ** -23 * torch.mm(h.abs(), head.abs().t().contiguous()).amax(1)
    el = 2 * (ez + 2.0 ** -15 + 2.0 ** -22 * torch.logsumexp(z, 1).abs())
    assert ((nll.double() - torch.where(live, ref, torch.zeros_like(ref))).abs() <= el).all()
    hot = torch.zeros_like(p).scatter_(1, at, 1.0)
    delta = p.scatter(1, at, torch.special.expm1(-ref)[:, None]) * weight
    off = 2.0 ** -8 * delta.abs() + weight * (p + hot) * 3 * (el + 2.0 ** -15)[:, None] * (1 + 2.0 ** -8)
    dH = torch.mm(delta, head)
    eH = torch.mm(off, head.abs()) + (V + 64) * 2.0 ** -23 * torch.mm(delta.abs() + off, head.abs())
    eH = eH + 2.0 ** -8 * (dH.abs() + eH)
    dU = torch.mm(dH, B)
    eU = torch.mm(eH, B.abs()) + (D + 64) * 2.0 ** -23 * torch.mm(dH.abs() + eH, B.abs())
    eU = eU + 2.0 ** -8 * (dU.abs() + eU)
    ex = xs.double().repeat_interleave(Q.CHECKPOINT_GROUP, 1)[:, :D] * 0.5 * (1 + 2.0 ** -20)
    eu = us.double().repeat_interleave(Q.CHECKPOINT_GROUP, 1)[:, :R] * 0.5 * (1 + 2.0 ** -20)
    for e in range(len(ends) - 1):
        a, b = int(ends[e]), int(ends[e + 1])
        for left, el_, right, er, got in ((dU, eU, x, ex, G[e, :R * D].view(R, D)), (dH, eH, u, eu, G[e, R * D:].view(D, R))):
            l, l_, r, r_ = left[a:b].t().contiguous(), el_[a:b].t().contiguous(), right[a:b], er[a:b]
            want, size = torch.mm(l, r), torch.mm(l.abs() + l_, r.abs() + r_)
            # a factor may be rounded to bfloat16 for bfloat16 rows: 2^-8 of every term
            bound = torch.mm(l_, r.abs() + r_) + torch.mm(l.abs(), r_) + (2.0 ** -8 + (b - a + 64) * 2.0 ** -23) * size
            assert ((got.double() - want).abs() <= bound + 2.0 ** -8 * (want.abs() + bound)).all(), "example %d" % e


@pytest.mark.parametrize("lengths", [[40, 1, 33, 0, 76, 5], [1], [300, 17, 64, 128]])
@pytest.mark.parametrize("bits", [8, 1])
def test_from_tokens_to_scores(lengths, bits):
    _say("gradient path lengths=%s bits=%d" % (lengths, bits))
    model = _model(1)
    stores = []
    for seed in (2, 3):                                   # training examples, and validation ones
        X, y, w, ends = _batch(lengths, seed)
        G, made = _rows(model, X, y, w, ends)
        _check_rows(model, X, y, w, ends, G, made)
        n = len(lengths)
        for e in range(n):
            if lengths[e] == 0 or e == 2:
                assert not G[e].any()
        P = torch.empty(n, K, dtype=torch.float32, device=DEV)
        Q.project_quantize_slice(G[:, :R * D], K, 0, P, True, False, bits=bits, seed=7)
        codes, S, rn = Q.project_quantize_slice(G[:, R * D:], K, R * D, P, False, True, bits=bits, seed=7)
        host = oracle.project(G.cpu(), K, seed=7)
        some = np.linalg.norm(host, axis=1) > 0
        err = np.linalg.norm(P.cpu().numpy()[some] - host[some], axis=1) / np.linalg.norm(host[some], axis=1)
        assert (err <= 1e-2).all() and not P.cpu().numpy()[~some].any()
        oc, oS, orn = oracle.quantize(P.cpu().numpy(), bits)
        np.testing.assert_array_equal(codes.cpu().numpy(), oc)
        np.testing.assert_array_equal(S.cpu().numpy(), oS)
        np.testing.assert_array_equal(rn.cpu().numpy(), orn)
        stores.append((codes, rn, oc, orn))
    (tc, tr, otc, otr), (vc, vr, ovc, ovr) = stores
    got = Q.score([tc], [tr], [vc], [vr], [1.0], K, bits)
    want = oracle.score([otc], [otr], [ovc], [ovr], [1.0], K, bits)
    np.testing.assert_array_equal(got.cpu().numpy().view(np.uint32), want.view(np.uint32))


def test_the_whole_path_in_a_graph():
    """Captured once, replayed over new batches: rows and codes equal those of separate calls."""
    _say("gradient path in a graph")
    Q.init()
    model = _model(1)
    lengths = [40, 1, 33, 0, 76, 5]
    held = list(_batch(lengths, 2))

    def run():
        G, made = _rows(model, *held)
        return (G, made[0]) + tuple(Q.project_quantize(G, K, 8, seed=7)[:3])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for seed in (3, 4, 5):
        _say("gradient path replay %d" % seed)
        for a, b in zip(held, _batch(lengths, seed)):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        kept = [x.clone() for x in out]
        for a, b in zip(kept, run()):
            assert torch.equal(a, b)
