"""Plain 64-bit implementations of rotary cache writes, attention over a paged cache and e4m3 rows, and
the batches that their tests share."""
from __future__ import annotations

import math
import zlib

import torch

D = 128
SCALE = 1.0 / math.sqrt(D)


def half_step(dtype):
    """Largest relative error of one rounding to the type."""
    return torch.finfo(dtype).eps / 2


class Batch:
    """Sequences over one pool of pages: new tokens and cached tokens of each, a shuffled page table."""

    def __init__(self, new, kv, page, pad=0, paged=True, device="cpu", spare=3, seed=0, single=False):
        self.new, self.kv, self.page = list(new), list(kv), page
        n = len(new)
        per = [-(-k // page) for k in kv]
        self.width = max(1, max(per))
        self.pool = max(1, sum(per)) + spare
        g = torch.Generator().manual_seed(seed)
        ids = torch.randperm(self.pool, generator=g) if paged else torch.arange(self.pool)
        # entries behind a sequence's last page must not be read: out of range on purpose
        self.table = torch.full((n, self.width), -7, dtype=torch.int32)
        at = 0
        for i, p in enumerate(per):
            self.table[i, :p] = ids[at:at + p].to(torch.int32)
            at += p
        self.paged = paged
        cu = [0]
        for x in new:
            cu.append(cu[-1] + x)
        self.cu, self.total = cu, cu[-1] + pad
        self.single = single  # one new token per sequence, no cu_q
        self.device = device
        self.d_cu = torch.tensor(cu, dtype=torch.int32, device=device)
        self.d_kv = torch.tensor(kv, dtype=torch.int32, device=device)
        self.d_table = self.table.to(device)

    def make(self, P, **over):
        a = dict(n_seqs=len(self.new), total_q=self.total, max_q=max(1, max(self.new)) if self.single else max(self.new),
                 max_kv=max(self.kv), cu_q=None if self.single else self.d_cu, kv_len=self.d_kv,
                 page_table=self.d_table if self.paged else None, table_stride=self.width)
        a.update(over)
        return P.make_batch(**a)

    def slots(self, s, first, last):
        """Pool slots (page * page_size + offset) of positions [first, last) of sequence s."""
        pos = torch.arange(first, last)
        return self.table[s].long()[pos // self.page] * self.page + pos % self.page

    def sequences(self):
        """(sequence, rows, positions) of the new tokens."""
        for s, n in enumerate(self.new):
            rows = torch.arange(self.cu[s], self.cu[s] + n)
            yield s, rows, self.kv[s] - n + torch.arange(n)


def seed_of(*parts):
    return zlib.crc32(repr(parts).encode())


# ------------------------------------------------------------------------------- e4m3

def quantise64(x, dtype):
    """(values of the codes, powers of two, e + 127) of rows of x, from the definition in 64 bits."""
    limit = 0.9375 * (2.0 ** 16 if dtype == torch.float16 else 2.0 ** 128)
    x = x.double().clamp(-limit, limit)
    top = x.abs().amax(-1)
    e = torch.full_like(top, -126.0)
    some = top > 448.0 * 2.0 ** -126
    e[some] = torch.ceil(torch.log2(top[some] / 448.0))
    e = torch.where(top > 448.0 * torch.exp2(e), e + 1, e)
    e = torch.where((top <= 448.0 * torch.exp2(e - 1)) & (e > -126), e - 1, e)
    y = x * torch.exp2(-e)[..., None]
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step, torch.exp2(e), (e + 127).to(torch.uint8)


def codes_of(values):
    """e4m3 codes of exactly representable values."""
    return values.float().to(torch.float8_e4m3fn)


# ------------------------------------------------------------------------------- rotation

def rotate64(x, pos, freqs, rot, interleaved, scale):
    """x [rows][heads][128] rotated at pos, in 64 bits; and the sum of magnitudes that went into each channel."""
    y = x.double().clone()
    mag = y.abs() * 0
    if rot:
        ang = pos.double()[:, None] * freqs.double()
        c, s = torch.cos(ang)[:, None] * scale, torch.sin(ang)[:, None] * scale
        if interleaved:
            ia, ib = torch.arange(0, rot, 2), torch.arange(1, rot, 2)
        else:
            ia, ib = torch.arange(0, rot // 2), torch.arange(rot // 2, rot)
        a, b = x[..., ia].double(), x[..., ib].double()
        y[..., ia], y[..., ib] = a * c - b * s, a * s + b * c
        mag[..., ia] = mag[..., ib] = (a.abs() + b.abs()) * abs(scale)
    return y, mag


# ------------------------------------------------------------------------------- attention

def attend64(q, k, v, visible=None):
    """q [rows][128], k, v [keys][128] in 64 bits, visible [rows][keys] or None: o, m, l, and the bounds'
    ingredients: weights times |v|, and the largest sum of |q_i k_i| / sqrt(128)."""
    rows, keys = q.shape[0], k.shape[0]
    if keys == 0:
        z = torch.zeros(rows, D, dtype=torch.float64, device=q.device)
        return z, z[:, 0] - math.inf, z[:, 0].clone(), z.clone(), z[:, 0].clone()
    s = (q @ k.T.contiguous()) * SCALE
    if visible is not None:
        s = s.masked_fill(~visible, -math.inf)
    m = s.amax(-1)
    p = torch.exp(s - torch.where(m.isinf(), 0.0, m)[:, None])
    l = p.sum(-1)
    w = p / torch.where(l == 0, 1.0, l)[:, None]
    return w @ v, m, l, w @ v.abs(), ((q.abs() @ k.abs().T.contiguous()) * SCALE).amax(-1)


def check_state(got_o, got_m, got_l, o, m, l, a, mag, weight_err, out_err, keys, floor=0.0, what=""):
    """A softmax state against the 64-bit one.

    A float32 product of 128 terms is off by at most 128 * 2^-24 of the sum of the terms' magnitudes: `mag` *
    2^-17 for a scaled logit.  The exponent's scaled argument and exp2 add 2^-22 of the logit (< mag) and
    2^-23: dm = mag * 2^-16 + 2^-22 bounds both.  A weight is off by 2 dm relative (its logit's and the maximum's),
    a sum of `keys` weights by keys * 2^-24 more.  The output's weights carry weight_err (their rounding) on top,
    `floor` is their absolute error (subnormal terms); one final rounding is out_err of the result."""
    dm = mag * 2.0 ** -16 + 2.0 ** -22
    seen = l > 0
    assert torch.equal(got_m.isinf(), ~seen), what
    assert torch.all(got_l[~seen] == 0) and torch.all(got_o[~seen] == 0), what
    if not seen.any():
        return
    e = (got_m - m).abs()[seen]
    assert torch.all(e <= dm[seen]), (what, "m", (e / dm[seen]).max())
    tl = 2 * dm + keys * 2.0 ** -24 + 2.0 ** -20
    e = ((got_l - l).abs() / torch.where(seen, l, 1.0))[seen]
    assert torch.all(e <= tl[seen]), (what, "l", (e / tl[seen]).max())
    to = out_err * o.abs() + (weight_err + 2 * tl)[:, None] * a * (1 + out_err) + floor
    e = (got_o - o).abs()[seen]
    assert torch.all(e <= to[seen]), (what, "o", (e / to[seen]).max())
