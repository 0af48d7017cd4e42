"""8-bit activation checkpoints and the weight gradients that are taken from them, against their plain 64-bit forms.

Codes, steps and what they are read back as are whole or exactly defined: they have to be equal.  A gradient is a sum of L terms.
With fp32 results the terms are exact (bfloat16 dY) or off by 2^-24 of themselves (fp32 dY, in three bfloat16 parts), and the matrix
cores and the joins add them in fp32, each of at most L + 64 additions off by at most one step, 2^-23 of a partial sum that is at most
the sum S of the terms' absolute values: |error| <= (L + 64) 2^-23 S.  bfloat16 results add the rounding of a factor to bfloat16, 2^-8
of every term at most, and their own, 2^-8 of the result."""
import pytest
import torch

from paper_2502_01703_amd import binding as Q
import plain_gradients as plain

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _say(msg):
    print("[case] " + msg, flush=True)


def _inputs(T, D, seed, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    X = torch.randn(T, D, generator=g) * torch.exp(2 * torch.randn(1, D, generator=g)) * torch.exp(torch.randn(T, 1, generator=g))
    return X.to(dtype)


def _inside(X, left, right):
    """X as a view into a wider buffer on the GPU, rows `left` elements in, and that buffer."""
    T, D = X.shape
    wide = torch.full((T, left + D + right), 7, dtype=X.dtype, device=DEV)
    wide[:, left:left + D] = X.to(DEV)
    return wide[:, left:left + D], wide


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,D,left,right", [(1, 1, 0, 0), (1, 128, 0, 0), (3, 127, 0, 0), (5, 129, 1, 2), (2, 8, 0, 0), (7, 1000, 0, 24), (33, 1333, 3, 0),
                                            (130, 512, 0, 0), (1, 16384, 0, 0), (4099, 40, 0, 8)])
def test_written_and_read(T, D, left, right, dtype):
    _say("checkpoint T=%d D=%d left=%d right=%d %s" % (T, D, left, right, dtype))
    X = _inputs(T, D, T * 7 + D, dtype)
    codes, steps = plain.checkpoint(X)
    x, _ = _inside(X, left, right)
    q, cwide = _inside(torch.zeros(T, D, dtype=torch.int8), left, right)
    s, swide = _inside(torch.zeros(T, steps.shape[1]), right, left)
    Q.checkpoint8(x, q, s)
    assert torch.equal(q.cpu().long(), codes)
    assert torch.equal(s.cpu().double(), steps)
    for wide, a, n in ((cwide, left, D), (swide, right, steps.shape[1])):     # what lies beside the rows stays
        assert (wide[:, :a] == 7).all() and (wide[:, a + n:] == 7).all()
    for out in (torch.bfloat16, torch.float32):
        y, ywide = _inside(torch.zeros(T, D, dtype=out), right, left)
        Q.checkpoint8_read(q, s, out=y)
        assert torch.equal(y.cpu(), plain.values(codes, steps).to(out))
        assert (ywide[:, :right] == 7).all() and (ywide[:, right + D:] == 7).all()
        assert torch.equal(Q.checkpoint8_read(q, s, out), y)


def test_borders_of_the_rule():
    """Quotients at, just above and just below halves; largest values on and just above 127 steps; the least and largest numbers."""
    rows = []
    for s in (1.0, 1.0078125, 1.9921875, 2.0 ** -120, 2.0 ** 100):
        half = torch.arange(0.5, 127.0, 1.0) * s
        half = half.float()
        for step in (0, 1, -1):
            v = (half.view(torch.int32) + step).view(torch.float32)
            row = torch.zeros(128)
            row[:127] = v[:127]
            row[1::2] *= -1
            row[127] = 127.0 * s
            rows.append(row)
        for step in (1, 2, 255):
            row = torch.linspace(-1, 1, 128) * s
            row[5] = (torch.tensor(127.0 * s).view(torch.int32) + step).view(torch.float32)
            rows.append(row)
    tiny = torch.zeros(128)
    tiny[:4] = torch.tensor([1.4e-45, -1e-40, 3e-38, 1.2e-38])
    big = torch.full((128,), 3.4028234e38)
    rows += [tiny, tiny * 100, big, -big, torch.zeros(128)]
    X = torch.stack(rows)
    _say("checkpoint borders")
    codes, steps = plain.checkpoint(X)
    q, s = Q.checkpoint8(X.to(DEV))
    assert torch.equal(q.cpu().long(), codes) and torch.equal(s.cpu().double(), steps)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_groups_that_are_not_finite(dtype):
    X = _inputs(6, 300, 5, dtype)
    X[0, 3] = float("inf")
    X[1, 200] = float("nan")
    X[2, 299] = -float("inf")
    X[3, 127] = float("nan")
    _say("checkpoint not finite %s" % dtype)
    q, s = Q.checkpoint8(X.to(DEV))
    codes, steps = plain.checkpoint(X)
    bad = torch.zeros(6, 3, dtype=torch.bool)
    for t, g in ((0, 0), (1, 1), (2, 2), (3, 0)):
        bad[t, g] = True
    assert torch.equal(s.isnan().cpu(), bad) and torch.equal(q.cpu().long(), codes)
    assert torch.equal(s.cpu().double()[~bad], steps[~bad])
    back = Q.checkpoint8_read(q, s, torch.float32).cpu()
    assert torch.equal(back.isnan(), bad.repeat_interleave(128, 1)[:, :300])


def _bound(ends, size, ref, dtype):
    lengths = torch.tensor([b - a for a, b in zip(ends, ends[1:])], dtype=torch.float64)[:, None, None]
    bound = (lengths + 64) * 2.0 ** -23 * size
    if dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * size * (1 + 2.0 ** -8) + 2.0 ** -8 * ref.abs()
    return bound


CASES = [  # R, D, ends
    (16, 256, [0, 64, 128, 200]),
    (1, 1, [0, 1]),
    (1, 128, [0, 0, 1, 1, 2, 2]),
    (5, 130, [3, 10, 10, 75]),
    (17, 127, [0, 63, 64, 129]),
    (24, 1333, [0, 333]),
    (40, 260, [1, 5, 300]),
    (128, 384, [0, 100, 101, 257]),
    (200, 140, [0, 65, 190]),
    (16, 128, [0, 5000]),
    (8, 256, [0, 10, 4000, 4003]),
    (300, 129, [0, 2500]),
]
WHOLE = [  # R in eights, D in sixteens: rows of whole chunks
    (8, 16, [0, 1]),
    (16, 144, [0, 31, 32, 64, 129]),
    (24, 528, [2, 35, 35, 200]),
    (32, 512, [0, 100]),
    (40, 48, [0, 0, 33, 90]),
    (64, 1040, [0, 65, 70]),
    (72, 256, [5, 6, 134]),
    (128, 640, [0, 257, 300]),
    (136, 400, [0, 96, 97]),
    (16, 128, [0, 5000]),
    (8, 1024, [0, 10, 4000, 4003]),
    (256, 272, [0, 2500, 5000]),
    (520, 1040, [0, 200, 333]),
    (1032, 1995, [3, 200, 200, 455, 700]),               # tiles of expanded activations
    (4096, 2048, [0, 300]),
]


@pytest.mark.parametrize("dtY,dtG", [(torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32),
                                     (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("R,D,ends,pad", [(*c, 1) for c in CASES] + [(*c, 0) for c in WHOLE] + [(*c, 1) for c in WHOLE[1:9]])
def test_weight_gradients(R, D, ends, pad, dtY, dtG):
    _say("gradient R=%d D=%d ends=%s pad=%d %s %s" % (R, D, ends, pad, dtY, dtG))
    T = ends[-1] + 9                                  # tokens behind the last example
    codes, steps = plain.checkpoint(_inputs(T, D, R + D))
    g = torch.Generator().manual_seed(R * D)
    dY = (torch.randn(T, R, generator=g) * torch.exp(torch.randn(T, 1, generator=g)) * 1e-3).to(dtY)
    ref, size = plain.weight_gradients(dY, codes, steps, ends)
    for x in (dY, steps):                             # neither these nor the ones behind are read
        x[:ends[0]] = float("nan")
        x[ends[-1]:] = float("nan")
    y, _ = _inside(dY, pad, 2 * pad)
    q, _ = _inside(codes.to(torch.int8), 3 * pad, pad)
    s, _ = _inside(steps.float(), 0, pad)
    off = torch.tensor(ends, device=DEV)
    G = Q.checkpoint8_grad(y, q, s, off, dtype=dtG)
    assert G.shape == ref.shape and G.dtype == dtG
    bound = _bound(ends, size, ref, dtG)
    assert ((G.cpu().double() - ref).abs() <= bound).all()
    # again, into a slice of wider rows: the same bits, and nothing beside it
    out, wide = _inside(torch.zeros(len(ends) - 1, R * D, dtype=dtG), 5, 6)
    Q.checkpoint8_grad(y, q, s, off, out=out)
    assert torch.equal(out.reshape(ref.shape), G)
    assert (wide[:, :5] == 7).all() and (wide[:, 5 + R * D:] == 7).all()


@pytest.mark.parametrize("dtY,dtG", [(torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32)])
@pytest.mark.parametrize("R,D,ends", [(100, 1333, [0, 9000, 9001, 15100]), (6, 1344, [0, 40, 15000]), (70, 1344, [5, 8000, 15000]), (7, 1333, [0, 7000, 15100]),
                                      (4100, 2040, [0, 140])])
def test_rows_worth_packing(R, D, ends, dtY, dtG):
    """Rows that are no whole chunks, of tensors large enough (or products enough) to be packed first; the workspace ends where it says."""
    _say("gradient of packed rows R=%d D=%d %s %s" % (R, D, dtY, dtG))
    T, n = ends[-1] + 9, len(ends) - 1
    codes, steps = Q.checkpoint8(_inputs(T, D, R + D).to(DEV))
    g = torch.Generator().manual_seed(R * D)
    dY = (torch.randn(T, R, generator=g) * torch.exp(torch.randn(T, 1, generator=g)) * 1e-3).to(dtY).to(DEV)
    x, y = codes.double() * steps.double().repeat_interleave(Q.CHECKPOINT_GROUP, 1)[:, :D], dY.double()
    ref = torch.stack([torch.mm(y[a:b].t().contiguous(), x[a:b]) for a, b in zip(ends, ends[1:])])
    size = torch.stack([torch.mm(y[a:b].t().abs().contiguous(), x[a:b].abs()) for a, b in zip(ends, ends[1:])])
    for t in (dY, steps):
        t[:ends[0]] = float("nan")
        t[ends[-1]:] = float("nan")
    need = Q.checkpoint8_grad_workspace(T, n, R, D)
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device=DEV)
    G = Q.checkpoint8_grad(dY, codes, steps, torch.tensor(ends, device=DEV), dtype=dtG, ws=ws[:need])
    assert (ws[need:] == 0xFF).all()
    assert ((G.cpu().double() - ref.cpu()).abs() <= _bound(ends, size.cpu(), ref.cpu(), dtG)).all()


@pytest.mark.parametrize("n,R,D", [(4, 2048, 2048), (5, 2045, 1800), (32, 1024, 512), (22, 1536, 512), (65, 1024, 250), (33, 1100, 264), (9, 4096, 500)])
@pytest.mark.parametrize("how", ["ragged", "alike"])
def test_many_rows_of_many_examples(n, R, D, how):
    """Expanded activations and tiles of whole examples, ranked by length up to 64 of them; empty ones, and ones that end in a stage."""
    _say("gradient of many rows n=%d R=%d D=%d %s" % (n, R, D, how))
    g = torch.Generator().manual_seed(n)
    T = 130 * n
    ends = [130 * e for e in range(n + 1)]
    if how == "ragged":
        ends = [3] + torch.sort(torch.randint(3, T, (n - 3,), generator=g)).values.tolist() + [T, T, T + 1]
        T += 1
    codes, steps = Q.checkpoint8(_inputs(T, D, R + D).to(DEV))
    dY = (torch.randn(T, R, generator=g) * torch.exp(torch.randn(T, 1, generator=g)) * 1e-3).bfloat16().to(DEV)
    x, y = codes.double() * steps.double().repeat_interleave(Q.CHECKPOINT_GROUP, 1)[:, :D], dY.double()
    G = Q.checkpoint8_grad(dY, codes, steps, torch.tensor(ends, device=DEV), dtype=torch.bfloat16)
    for e, (a, b) in enumerate(zip(ends, ends[1:])):
        ref, size = torch.mm(y[a:b].t().contiguous(), x[a:b]), torch.mm(y[a:b].t().abs().contiguous(), x[a:b].abs())
        assert ((G[e].double() - ref).abs().cpu() <= _bound([a, b], size[None].cpu(), ref[None].cpu(), torch.bfloat16)[0]).all(), "example %d" % e


@pytest.mark.parametrize("n", [2, 63, 64, 65, 128, 255, 256, 257, 600])
@pytest.mark.parametrize("how", ["ragged", "alike", "one long"])
@pytest.mark.parametrize("dtY", [torch.bfloat16, torch.float32])
def test_many_examples(n, how, dtY):
    """Examples of any lengths, in parts or whole, none of them lost and none taken twice, whatever the order of the work."""
    _say("gradient of many examples n=%d %s %s" % (n, how, dtY))
    g = torch.Generator().manual_seed(n)
    if how == "ragged":
        T = 9 * n + 1500
        ends = [0] + torch.sort(torch.randint(0, T // 2, (n - 2,), generator=g)).values.tolist() + [T // 2, T]
    elif how == "alike":
        T = 7 * n
        ends = list(range(0, T + 1, 7))
    else:
        T = 3000
        ends = [0] * (n // 2 + 1) + [T] * (n - n // 2)
    codes, steps = plain.checkpoint(_inputs(T, 144, n))
    dY = (torch.randn(T, 8, generator=g) * 1e-3).to(dtY)
    ref, size = plain.weight_gradients(dY, codes, steps, ends)
    G = Q.checkpoint8_grad(dY.to(DEV), codes.to(torch.int8).to(DEV), steps.float().to(DEV), torch.tensor(ends, device=DEV))
    assert ((G.cpu().double() - ref).abs() <= _bound(ends, size, ref, torch.float32)).all()



def test_no_tokens_and_no_examples():
    _say("gradient of nothing")
    empty = (torch.empty(0, 4, device=DEV), torch.empty(0, 200, dtype=torch.int8, device=DEV), torch.empty(0, 2, device=DEV))
    G = Q.checkpoint8_grad(*empty, torch.zeros(4, dtype=torch.int64, device=DEV))
    assert G.shape == (3, 4, 200) and not G.any()
    assert Q.checkpoint8_grad(*empty, torch.zeros(1, dtype=torch.int64, device=DEV)).shape == (0, 4, 200)
    q, s = Q.checkpoint8(torch.empty(0, 200, device=DEV))
    assert q.shape == (0, 200) and Q.checkpoint8_read(q, s).shape == (0, 200)


def test_a_bad_token_stays_in_its_group():
    """A group that is not finite reaches its own example's columns and no others."""
    X = _inputs(100, 300, 9)
    X[40, 130] = float("nan")
    _say("gradient not finite")
    q, s = Q.checkpoint8(X.to(DEV))
    dY = torch.randn(100, 20, generator=torch.Generator().manual_seed(3)).to(DEV)
    G = Q.checkpoint8_grad(dY, q, s, torch.tensor([0, 30, 70, 100], device=DEV))
    bad = torch.zeros(3, 20, 300, dtype=torch.bool)
    bad[1, :, 128:256] = True
    assert torch.equal(G.isnan().cpu(), bad)


def test_captured():
    """Written, read and used inside a graph, replayed on new activations with eager work in between."""
    Q.init()
    T, D, R = 700, 520, 24
    X = torch.empty(T, D, dtype=torch.bfloat16, device=DEV)
    dY = torch.empty(T, R, dtype=torch.bfloat16, device=DEV)
    off = torch.tensor([0, 100, 100, 650], device=DEV)

    def step():
        q, s = Q.checkpoint8(X)
        return q, s, Q.checkpoint8_read(q, s), Q.checkpoint8_grad(dY, q, s, off)
    X.zero_(), dY.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        _say("checkpoint replay %d" % i)
        X.copy_(_inputs(T, D, i, torch.bfloat16))
        dY.copy_(torch.randn(T, R, generator=torch.Generator().manual_seed(i)))
        graph.replay()
        torch.cuda.synchronize()
        kept = [x.clone() for x in held]
        for a, b in zip(kept, step()):
            assert torch.equal(a, b)
