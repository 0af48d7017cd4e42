"""The operators that make a gradient row before the datastore projects it: the loss of a batch over the vocabulary with its
gradients, 8-bit activation checkpoints, and the per-example weight gradients that are taken from them.  Each case is a dict
of plain values; `prepare` makes what a program holds before the call, `run` is one pass (in plain torch operations, or
through the public entry points where `own` is true), `exact` the same numbers in 64 bits."""
import math

import torch

DEV = "cuda"
GROUP = 128          # columns that share a step

own = False


def listed():
    return [
        # One token's loss and its gradient at the last hidden state: the smallest call, a loop over single tokens.
        dict(name="loss_one_token", kind="loss", T=1, D=2048, V=32000, masked=0.0, dH=1, dW=0, pad=0),
        # Evaluation of a short odd batch under a tokenizer of odd size: the loss alone.
        dict(name="loss_eval_odd", kind="loss", T=301, D=1000, V=50257, masked=0.25, dH=0, dW=0, pad=0),
        # Gradient extraction of an instruction-tuning batch at the 7B-class width: 16 examples of 512 tokens, prompts masked, head frozen.
        dict(name="loss_batch_masked", kind="loss", T=8192, D=4096, V=32000, masked=0.6, dH=1, dW=0, pad=0),
        # The same with a vocabulary of 2^17 and no prompt.
        dict(name="loss_wide_vocab", kind="loss", T=4096, D=4096, V=131072, masked=0.0, dH=1, dW=0, pad=0),
        # A training step of a small model whose head learns too; rows of a wider buffer.
        dict(name="loss_train_head", kind="loss", T=2048, D=2048, V=50257, masked=0.1, dH=1, dW=1, pad=8),
        # One short example's activations written and read back: launches count.
        dict(name="trip_short", kind="trip", T=48, D=1024, dtype="bf16", pad=0),
        # A batch of a 7B-class layer's input, written in the forward pass and read in the backward pass.
        dict(name="trip_layer", kind="trip", T=32768, D=4096, dtype="bf16", pad=0),
        # fp32 activations of an odd width in a wider buffer.
        dict(name="trip_odd_fp32", kind="trip", T=5003, D=1333, dtype="fp32", pad=3),
        # Per-example gradients of one rank-16 adapter, 64 ragged examples, as rows to project.
        dict(name="grad_rank16", kind="grad", T=32768, n=64, R=16, D=4096, y="bf16", g="bf16"),
        # The 7B-class configuration's adapters of rank 128 on width 4096, fp32 gradients.
        dict(name="grad_rank128_fp32", kind="grad", T=16384, n=32, R=128, D=4096, y="bf16", g="fp32"),
        # One example at a time, odd sizes, fp32 throughout.
        dict(name="grad_one_odd", kind="grad", T=333, n=1, R=24, D=1333, y="fp32", g="fp32"),
        # The weight gradient of a whole linear layer over a batch.
        dict(name="grad_full_weight", kind="grad", T=8192, n=1, R=4096, D=4096, y="bf16", g="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["loss", "loss", "trip", "grad", "grad"])
    if kind == "loss":
        dH = rng.choice([0, 1, 1, 1])
        dW = dH and rng.choice([0, 0, 1])
        D = _log(rng, 64, 8192)
        if rng.random() < 0.6:
            D = max(64, D // 64 * 64)
        V = _log(rng, 1000, 150000)
        cap = 6e12 / (2.0 * D * V * (1 + dH + 2 * dW))
        T = _log(rng, 1, max(1, min(8192, cap, 5e8 / V)))
        return dict(kind=kind, T=T, D=D, V=V, masked=rng.choice([0.0, 0.0, 0.3, 0.7]), dH=dH, dW=dW, pad=rng.choice([0, 0, 8, 3]))
    if kind == "trip":
        D = _log(rng, 16, 16384)
        if rng.random() < 0.6:
            D = max(16, D // 16 * 16)
        T = _log(rng, 1, max(1, min(65536, 1.3e8 / D)))
        return dict(kind=kind, T=T, D=D, dtype=rng.choice(["bf16", "bf16", "fp32"]), pad=rng.choice([0, 0, 8, 3]))
    R = rng.choice([_log(rng, 1, 256), 1 << rng.randint(3, 7), _log(rng, 256, 4096)])
    D = _log(rng, 16, 8192)
    if rng.random() < 0.6:
        D = max(16, D // 16 * 16)
    n = _log(rng, 1, max(1, min(256, 6e7 / (R * D))))
    T = min(_log(rng, 1, 1024) * n, int(min(65536, 2.5e11 / (2.0 * R * D), 1.3e8 / max(R, D)))) + 1
    return dict(kind=kind, T=T, n=n, R=R, D=D, y=rng.choice(["bf16", "bf16", "fp32"]), g=rng.choice(["bf16", "fp32"]))


_DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
_EXAMPLE = 512       # tokens of an example in the loss cases


def _masked(case):
    """Host list of truth values: the leading part of every example is prompt."""
    skip = int(case["masked"] * min(_EXAMPLE, case["T"]))
    return [t % _EXAMPLE < skip for t in range(case["T"])]


def _activations(T, D, gen, dtype):
    """Activations of a transformer layer: some channels far larger than the rest, rows of different size."""
    x = torch.randn(T, D, generator=gen, device=DEV)
    x *= torch.exp(0.5 * torch.randn(1, D, generator=gen, device=DEV))
    x *= torch.exp(0.3 * torch.randn(T, 1, generator=gen, device=DEV))
    x *= 1.0 + 19.0 * (torch.rand(1, D, generator=gen, device=DEV) < 0.003)
    return x.to(dtype)


def _padded(x, pad):
    if not pad:
        return x
    wide = torch.zeros(x.shape[0], x.shape[1] + pad, dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = dict(case)
    if case["kind"] == "loss":
        T, D, V = case["T"], case["D"], case["V"]
        W = torch.empty(V, D, dtype=torch.bfloat16, device=DEV)
        for v in range(0, V, 16384):
            W[v:v + 16384] = torch.randn(min(16384, V - v), D, generator=gen, device=DEV) / math.sqrt(D)
        target = torch.randint(0, V, (T,), generator=gen, device=DEV)
        # tokens from unpredictable to certain: the target's logit stands 0 .. 16 above the others'
        H = 1.5 * torch.randn(T, D, generator=gen, device=DEV)
        H += 16.0 * torch.rand(T, 1, generator=gen, device=DEV) * W[target].float()
        mask = torch.tensor(_masked(case), device=DEV)
        s["target"] = torch.where(mask, torch.full_like(target, -100), target)
        s["H"] = _padded(H.to(torch.bfloat16), case["pad"])
        s["W"] = _padded(W, case["pad"])
        # the mean over each example's answer
        example = torch.arange(T, device=DEV) // _EXAMPLE
        count = torch.zeros(int((T + _EXAMPLE - 1) // _EXAMPLE), device=DEV).index_add_(0, example, (~mask).float())
        s["weight"] = 1.0 / count.clamp(min=1.0)[example]
    elif case["kind"] == "trip":
        s["X"] = _padded(_activations(case["T"], case["D"], gen, _DT[case["dtype"]]), case["pad"])
    else:
        T, n, R, D = case["T"], case["n"], case["R"], case["D"]
        X = _activations(T, D, gen, torch.float32)
        s["codes"], s["step"] = _write(X)
        s["dY"] = (torch.randn(T, R, generator=gen, device=DEV) * torch.exp(0.5 * torch.randn(T, 1, generator=gen, device=DEV)) / T).to(_DT[case["y"]])
        cut = torch.sort(torch.randint(0, T + 1, (n - 1,), generator=gen, device=DEV)).values
        edge = torch.tensor([0, T], device=DEV)
        s["offsets"] = torch.cat([edge[:1], cut, edge[1:]])
        s["ends"] = s["offsets"].tolist()
    return s


# ---- the plain forms

def _columns(step, D):
    """Each column's step."""
    return step.repeat_interleave(GROUP, dim=1)[:, :D]


def _write(X):
    """Codes and steps: the step of a row's group is the least number of 8 significant bits (at least 2^-126) of which 127 reach
    the group's largest value; a code is the nearest whole number of steps, ties to even."""
    T, D = X.shape
    G = (D + GROUP - 1) // GROUP
    x = torch.nn.functional.pad(X.float(), (0, G * GROUP - D)).view(T, G, GROUP)
    top = x.abs().amax(2)
    step = (((top / 127.0).view(torch.int32) + 0xFFFF) & ~0xFFFF).view(torch.float32)
    below, above = (step.view(torch.int32) - 0x10000).view(torch.float32), (step.view(torch.int32) + 0x10000).view(torch.float32)
    step = torch.where(below * 127.0 >= top, below, torch.where(step * 127.0 < top, above, step)).clamp(min=2.0 ** -126)
    step = torch.where(top == 0, torch.zeros_like(step), step)
    each = torch.where(step == 0, torch.ones_like(step), step)[..., None]
    q = torch.empty(T, G, GROUP, dtype=torch.int8, device=X.device)
    for t in range(0, T, 8192):          # quotients next to a half need 64 bits
        q[t:t + 8192] = (x[t:t + 8192].double() / each[t:t + 8192].double()).round().to(torch.int8)
    return q.view(T, G * GROUP)[:, :D].contiguous(), step


def _loss(s):
    H, W, target, weight, V = s["H"], s["W"], s["target"], s["weight"], s["V"]
    keep = (target >= 0) & (target < V)
    at = target.clamp(0, V - 1)[:, None]
    h = torch.where(keep[:, None], H, torch.zeros_like(H)).float()
    w = W.float()
    logits = h @ w.t()
    top = logits.amax(1, keepdim=True)
    lse = top + (logits - top).exp().sum(1, keepdim=True).log()
    zero = torch.zeros_like(lse[:, 0])
    out = {"nll": torch.where(keep, (lse - logits.gather(1, at))[:, 0], zero), "lse": torch.where(keep, lse[:, 0], zero)}
    if s["dH"] or s["dW"]:
        delta = (logits - lse).exp()
        delta.scatter_add_(1, at, torch.full_like(lse, -1.0))
        delta *= torch.where(keep, weight, zero)[:, None]
        if s["dH"]:
            out["dH"] = (delta @ w).to(H.dtype)
        if s["dW"]:
            out["dW"] = (delta.t() @ h).to(W.dtype)
    return out


def _grad(s):
    x = s["codes"].float() * _columns(s["step"], s["D"])
    y = s["dY"].float()
    G = torch.zeros(s["n"], s["R"], s["D"], device=x.device)
    for e in range(s["n"]):
        a, b = s["ends"][e], s["ends"][e + 1]
        if b > a:
            G[e] = y[a:b].t() @ x[a:b]
    return G.to(_DT[s["g"]])


def run(state):
    s = state
    if own:
        from paper_2502_01703_amd import binding as Q
        if s["kind"] == "loss":
            nll, lse, dH, dW = Q.token_loss(s["H"], s["W"], s["target"], s["weight"], want_dH=bool(s["dH"]), want_dW=bool(s["dW"]))
            out = {"nll": nll, "lse": lse}
            if s["dH"]:
                out["dH"] = dH
            if s["dW"]:
                out["dW"] = dW
            return out
        if s["kind"] == "trip":
            codes, step = Q.checkpoint8(s["X"])
            return {"X": Q.checkpoint8_read(codes, step, s["X"].dtype), "step": step}
        return Q.checkpoint8_grad(s["dY"], s["codes"], s["step"], s["offsets"], dtype=_DT[s["g"]])
    if s["kind"] == "loss":
        return _loss(s)
    if s["kind"] == "trip":
        codes, step = _write(s["X"])
        return {"X": (codes.float() * _columns(step, s["D"])).to(s["X"].dtype), "step": step}
    return _grad(s)


def work(case):
    """Matrix products and bytes of one pass: tokens that count, every input and output once."""
    if case["kind"] == "loss":
        T, D, V = case["T"], case["D"], case["V"]
        live = T - sum(_masked(case))
        parts = 1 + case["dH"] + case["dW"]
        bytes_ = 2 * V * D * (1 + case["dW"]) + 2 * live * D + (2 * T * D if case["dH"] else 0) + 20 * T
        return {"bytes": bytes_, "flops": 2 * live * D * V * parts}
    T, D = case["T"], case["D"]
    G = (D + GROUP - 1) // GROUP
    if case["kind"] == "trip":
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": T * (2 * D * size + 2 * D + 8 * G), "flops": 4 * T * D}
    ysize, gsize = (2 if case["y"] == "bf16" else 4), (2 if case["g"] == "bf16" else 4)
    R, n = case["R"], case["n"]
    return {"bytes": T * (R * ysize + D + 4 * G) + n * R * D * gsize + 8 * (n + 1), "flops": 2 * T * R * D}


def exact(case, seed):
    """From the definitions, in 64 bits."""
    s = prepare(case, seed)
    if case["kind"] == "loss":
        T, D, V = case["T"], case["D"], case["V"]
        target, weight = s["target"], s["weight"].double()
        live = [t for t, m in enumerate(_masked(case)) if not m]
        nll = torch.zeros(T, dtype=torch.float64, device=DEV)
        lse = torch.zeros(T, dtype=torch.float64, device=DEV)
        W = s["W"]
        dH = torch.zeros(T, D, dtype=torch.float64, device=DEV) if case["dH"] else None
        dW = torch.zeros(V, D, dtype=torch.float64, device=DEV) if case["dW"] else None
        for i in range(0, len(live), 1024):
            rows = torch.tensor(live[i:i + 1024], device=DEV)
            h, y = s["H"][rows].double(), target[rows]
            z = torch.empty(len(rows), V, dtype=torch.float64, device=DEV)
            for v in range(0, V, 32768):
                z[:, v:v + 32768] = torch.mm(h, W[v:v + 32768].double().t().contiguous())
            lse[rows] = torch.logsumexp(z, 1)
            nll[rows] = lse[rows] - z[torch.arange(len(rows), device=DEV), y]
            if dH is None and dW is None:
                continue
            p = torch.softmax(z, 1)
            p[torch.arange(len(rows), device=DEV), y] = torch.special.expm1(-nll[rows])
            p *= weight[rows][:, None]
            for v in range(0, V, 32768):
                part = p[:, v:v + 32768].contiguous()
                if dH is not None:
                    dH[rows] += torch.mm(part, W[v:v + 32768].double())
                if dW is not None:
                    dW[v:v + 32768] += torch.mm(part.t().contiguous(), h)
        out = {"nll": nll, "lse": lse}
        if dH is not None:
            out["dH"] = dH
        if dW is not None:
            out["dW"] = dW
        return out
    if case["kind"] == "trip":
        X = s["X"].double()
        T, D = X.shape
        back, steps = torch.empty_like(X), []
        for c in range(0, D, GROUP):
            x = X[:, c:c + GROUP]
            top = x.abs().max(1).values
            share = top / torch.full_like(top, 127.0)
            _, e = torch.frexp(share)                                  # share = m 2^e, 1/2 <= m < 1
            unit = ((e.long() - 8 + 1023) << 52).view(torch.float64)   # 2^(e - 8)
            step = torch.ceil(share / unit) * unit
            step = torch.where(top > 0, step.clamp(min=2.0 ** -126), torch.zeros_like(step))
            steps.append(step)
            back[:, c:c + GROUP] = torch.round(x / torch.where(step > 0, step, torch.ones_like(step))[:, None]) * step[:, None]
        return {"X": back, "step": torch.stack(steps, 1)}
    G = torch.zeros(case["n"], case["R"], case["D"], dtype=torch.float64, device=DEV)
    for e in range(case["n"]):
        for a in range(s["ends"][e], s["ends"][e + 1], 4096):
            b = min(a + 4096, s["ends"][e + 1])
            x = s["codes"][a:b].double()
            for c in range(0, case["D"], GROUP):
                x[:, c:c + GROUP] *= s["step"][a:b, c // GROUP, None].double()
            G[e] += torch.mm(s["dY"][a:b].double().t().contiguous(), x)
    return G
