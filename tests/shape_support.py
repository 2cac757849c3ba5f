"""Plain 64-bit implementations of scores with a shape, received attention weight and token choice."""
from __future__ import annotations

import math

import torch

from tests import context_support as S


class Shape:
    """What the calls do to scores, as plain values: slopes [heads], first [rows], prefix [sequences] on the CPU."""

    def __init__(self, cap=0.0, slopes=None, window=0, first=None, prefix=None):
        self.cap, self.slopes, self.window, self.first, self.prefix = cap, slopes, window, first, prefix

    def make(self, P, device):
        on = lambda x, dt: None if x is None else torch.tensor(x, dtype=dt, device=device)  # noqa: E731
        return P.make_shape(self.cap, on(self.slopes, torch.float32), self.window, on(self.prefix, torch.int32),
                            on(self.first, torch.int32))

    def visible(self, s, rows, pos, kv):
        """[rows][keys]: which keys of sequence s tokens `rows` at positions pos see."""
        j = torch.arange(kv)
        lo = torch.zeros_like(pos)
        if self.window:
            lo = torch.maximum(lo, pos - self.window + 1)
        if self.first is not None:
            lo = torch.maximum(lo, torch.tensor([self.first[r] for r in rows.tolist()], dtype=torch.long))
        hi = pos + 1
        if self.prefix is not None:
            hi = torch.maximum(hi, torch.tensor(self.prefix[s]))
        return (j >= lo[:, None]) & (j < hi[:, None]) & (pos >= 0)[:, None]

    def scores(self, q, k, pos, head):
        """q [rows][128], k [keys][128] in 64 bits, positions and heads of the rows: scores, and the largest magnitude that
        went into a row's: S.check_state's bound of a plain score's error is `mag` * 2^-16.  A cap's error is at most
        cap * 2^-20 on top (reciprocal 2^-22, exponential 2^-24, sums and products 2^-23 each, of the cap), a bias's 2^-22 of
        the bias (its slope's two roundings and the sum's)."""
        z = (q @ k.T.contiguous()) * S.SCALE
        mag = ((q.abs() @ k.abs().T.contiguous()) * S.SCALE).amax(-1) if k.shape[0] else torch.zeros_like(z.sum(-1))
        if self.cap:
            cap = float(torch.tensor(self.cap, dtype=torch.float32))
            z = cap * torch.tanh(z / cap)
            mag = mag + cap / 16
        if self.slopes is not None:
            slope = torch.tensor(self.slopes, dtype=torch.float32).double().to(z.device)[head]
            bias = slope[:, None] * (pos[:, None] - torch.arange(k.shape[0], device=z.device)).abs()
            z = z - bias
            mag = mag + (bias.abs().amax(-1) if k.shape[0] else 0.0)
        return z, mag

    def attend(self, q, k, v, pos, head, visible):
        """As S.attend64."""
        z, mag = self.scores(q, k, pos, head)
        if k.shape[0] == 0:
            zero = torch.zeros(q.shape[0], S.D, dtype=torch.float64, device=q.device)
            return zero, zero[:, 0] - math.inf, zero[:, 0].clone(), zero.clone(), mag
        z = z.masked_fill(~visible, -math.inf)
        m = z.amax(-1)
        p = torch.exp(z - torch.where(m.isinf(), 0.0, m)[:, None])
        l = p.sum(-1)
        w = p / torch.where(l == 0, 1.0, l)[:, None]
        return w @ v, m, l, w @ v.abs(), mag


def slopes_of(heads):
    return [2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)]


def keep_of(mass, budget, sink, recent):
    """Positions kept of one sequence and KV head (a list of numbers)."""
    n = len(mass)
    count = min(budget, n)
    if count == n:
        return list(range(n))
    value = [-math.inf if x != x else x for x in mass]
    nan = [x != x for x in mass]
    always = [p < sink or p >= n - recent for p in range(n)]
    order = sorted(range(n), key=lambda p: (not always[p], nan[p], -value[p], p))
    return sorted(order[:count])
