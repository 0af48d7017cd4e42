"""Plain 64-bit forms, on the CPU, of the operators that make gradient rows, from their definitions."""
import math

import torch

GROUP = 128


def step_of(top):
    """The least number of eight significant bits, at least 2^-126, of which 127 reach `top` (a float); 0 for 0."""
    if top == 0:
        return 0.0
    if not math.isfinite(top):
        return float("nan")
    unit = 2.0 ** (math.frexp(top)[1] - 16)              # below every step in question; 127 k unit is exact
    while True:
        k = math.ceil(top / (127.0 * unit))
        while 127.0 * unit * (k - 1) >= top:
            k -= 1
        while 127.0 * unit * k < top:
            k += 1
        if k <= 256:
            return max(k * unit, 2.0 ** -126)
        unit *= 2.0


def checkpoint(X):
    """Codes (int64) and steps (float64) of X [T, D]: a code is the nearest whole number of steps, ties to even."""
    X = X.cpu().double()
    T, D = X.shape
    codes, steps = torch.zeros(T, D, dtype=torch.int64), torch.zeros(T, -(-D // GROUP), dtype=torch.float64)
    for g in range(steps.shape[1]):
        x = X[:, g * GROUP:(g + 1) * GROUP]
        steps[:, g] = torch.tensor([step_of(v) for v in x.abs().amax(1).tolist()], dtype=torch.float64)
        s = steps[:, g, None]
        codes[:, g * GROUP:(g + 1) * GROUP] = torch.where(s > 0, torch.round(x / s), torch.zeros_like(x)).long()
    return codes, steps


def values(codes, steps):
    """The activations that codes and steps stand for."""
    return codes.cpu().double() * steps.cpu().double().repeat_interleave(GROUP, dim=1)[:, :codes.shape[1]]


def weight_gradients(dY, codes, steps, ends):
    """(G [n, R, D], the sums of the terms' absolute values)."""
    y, x = dY.cpu().double(), values(codes, steps)
    G = torch.zeros(len(ends) - 1, y.shape[1], x.shape[1], dtype=torch.float64)
    size = torch.zeros_like(G)
    for e in range(len(ends) - 1):
        a, b = ends[e], ends[e + 1]
        G[e] = y[a:b].t() @ x[a:b]
        size[e] = y[a:b].abs().t() @ x[a:b].abs()
    return G, size
