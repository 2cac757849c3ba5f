"""Caps on both sides of where their forms change, held tightly: scores that are one product each, so that nothing but the
cap and the softmax rounds."""
import math

import pytest
import torch

from tests import context_support as S
from tests.shape_support import Shape

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f16": torch.float16}
CAPS = [50.0, 2.0 ** 10, 2.0 ** 11, 2.0 ** 14, 2.0 ** 20]
# of the cap: around 1/64, around 0.6, far above
PLACES = [0.010, 0.0157, 0.025, 0.1, 0.5, 0.58, 0.62, 0.9, 3.0]


def products(cap, place, n, dt, seed):
    """A number x and n numbers y of the type, x y / sqrt(128) about `place` of the cap and a few steps of the type apart."""
    s = place * cap * math.sqrt(128.0)
    x = 2.0 ** round(math.log2(math.sqrt(s)))
    step = torch.finfo(DT[dt]).eps / 2
    pick = torch.randint(-6, 7, (n,), generator=torch.Generator().manual_seed(seed))
    return x, (s / x * (1.0 + 2 * step * pick)).to(DT[dt])


def capped(x, y, cap):
    """z in 64 bits, and how far a float32 cap may be off.

    The product x y is exact.  The polynomial (below 0.6 of the cap) is off by 2^-22.4 relative, the cap and the scale by two
    roundings each, their products by three: 2^-22.4 + 7 * 2^-24 < 2^-20.8 of z.  Above it, an exponential of one unit in the last
    place (2^-23) and of an argument off by 2^-23 relative (2 s / cap >= 1.2, where x e^-x <= 0.37), a sum's rounding
    2^-24, a reciprocal 2^-23: all below 2^-21 together of 2 / (1 + e) <= 0.47, and the last sum: less than 2^-21 of the cap
    on top."""
    raw = x * y.double() / math.sqrt(128.0)
    z = cap * torch.tanh(raw / cap)
    return z, z.abs() * 2.0 ** -20.8 + torch.where(raw.abs() > 0.599 * cap, cap * 2.0 ** -21, 0.0)


def inputs(cap, place, n, dt, sign=1.0):
    """Queries x in channel 0, keys sign * y there and noise in the other channels, values; z and its bound."""
    x, y = products(cap, place, n, dt, S.seed_of(cap, place, n, dt))
    g = torch.Generator(device=DEV).manual_seed(n)
    page = -(-n // 16)
    k, v = (torch.randn(1, page * 16, S.D, generator=g, device=DEV).to(DT[dt]) for _ in range(2))
    y = sign * y
    k[0, :n, 0] = y.to(DEV)
    q = torch.zeros(n, 1, S.D, dtype=DT[dt], device=DEV)
    q[..., 0] = x
    z, tol = capped(x, y, cap)
    return q, k.view(1, page, 16, S.D), v.view(1, page, 16, S.D), z.to(DEV), tol.to(DEV)


def shapes(cap):
    """The instances that cap: alone, with masks, with slopes."""
    return [Shape(cap=cap), Shape(cap=cap, window=2 ** 30), Shape(cap=cap, slopes=[0.0])]


def check(o, m, l, z, tol, v, visible, out_err, what):
    """o, m, l of rows over keys with scores z (known up to tol): the maximum to its score's bound, a weight to twice that."""
    z = z.expand(len(visible), -1).masked_fill(~visible, -math.inf)
    dm = torch.where(visible, tol, 0.0).amax(-1) + 2.0 ** -22
    m64 = z.amax(-1)
    p = torch.exp(z - m64[:, None])
    l64 = p.sum(-1)
    w = p / l64[:, None]
    assert torch.all((m - m64).abs() <= dm), (what, "m", ((m - m64).abs() / dm).max())
    # (a weight's exponent: its score's error, the maximum's, and the exponent's own roundings, 2^-22 of its two terms)
    tl = 2 * dm + m64.abs() * 2.0 ** -22 + z.shape[1] * 2.0 ** -24 + 2.0 ** -20
    assert torch.all((l - l64).abs() <= torch.expm1(tl) * l64), (what, "l", ((l - l64).abs() / l64 / tl).max())
    v = v.double()
    to = out_err * (w @ v).abs() + (out_err + 2 * torch.expm1(tl))[:, None] * (w @ v.abs()) + 2.0 ** -14 * out_err * v.abs().max()
    assert torch.all((o - w @ v).abs() <= to), (what, "o", ((o - w @ v).abs() / to).max())


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("cap", CAPS)
def test_prompt_caps_at_their_borders(cap, dt):
    import paper_2606_30389_amd as P
    n = 150
    for place in PLACES:
        for sign in (1.0, -1.0):
            q, k, v, z, tol = inputs(cap, place, n, dt, sign)
            dims = P.make_dims(1, 1, 16, k.shape[1], P.PRR_BF16 if dt == "bf16" else P.PRR_F16)
            lens = [torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([0, n], [n])]
            batch = P.make_batch(1, n, n, n, lens[0], lens[1])
            pos = torch.arange(n, device=DEV)
            for i, shape in enumerate([*shapes(cap), Shape(cap=cap, window=1)]):
                sh = shape.make(P, DEV)
                out, m, l = torch.zeros_like(q), torch.zeros(n, 1, device=DEV), torch.zeros(n, 1, device=DEV)
                nbytes = P.prr_prompt_shaped_workspace_size(dims, batch, sh)
                ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=DEV)
                P.prr_prompt_attn_shaped(dims, batch, sh, q, k, v, out, m, l, ws, nbytes)
                torch.cuda.synchronize()
                visible = (pos[None] <= pos[:, None]) & (pos[None] > pos[:, None] - (shape.window or n))
                check(out[:, 0].double(), m[:, 0].double(), l[:, 0].double(), z, tol, v.flatten(0, 2)[:n], visible,
                      S.half_step(DT[dt]), (cap, place, sign, i))


@pytest.mark.gpu
@pytest.mark.parametrize("cap", [50.0, 2.0 ** 14])
def test_prompt_caps_of_eight_waves(cap):
    """As many key tiles as take the workgroups of eight waves."""
    import paper_2606_30389_amd as P
    n = 4500
    q, k, v, z, tol = inputs(cap, 0.025, n, "bf16")
    dims = P.make_dims(1, 1, 16, k.shape[1], P.PRR_BF16)
    lens = [torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([0, n], [n])]
    batch, sh = P.make_batch(1, n, n, n, lens[0], lens[1]), Shape(cap=cap).make(P, DEV)
    out, m, l = torch.zeros_like(q), torch.zeros(n, 1, device=DEV), torch.zeros(n, 1, device=DEV)
    nbytes = P.prr_prompt_shaped_workspace_size(dims, batch, sh)
    ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=DEV)
    P.prr_prompt_attn_shaped(dims, batch, sh, q, k, v, out, m, l, ws, nbytes)
    torch.cuda.synchronize()
    pos = torch.arange(n, device=DEV)
    check(out[:, 0].double(), m[:, 0].double(), l[:, 0].double(), z, tol, v.flatten(0, 2)[:n], pos[None] <= pos[:, None],
          S.half_step(torch.bfloat16), cap)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("cap", CAPS)
def test_decode_caps_at_their_borders(cap, dt):
    import paper_2606_30389_amd as P
    n = 150
    for place in PLACES:
        for sign in (1.0, -1.0):
            q, k, v, z, tol = inputs(cap, place, n, dt, sign)
            dims = P.make_dims(1, 1, 16, k.shape[1], P.PRR_BF16 if dt == "bf16" else P.PRR_F16)
            batch = P.make_batch(1, 1, 1, n, None, torch.tensor([n], dtype=torch.int32, device=DEV))
            for i, shape in enumerate(shapes(cap)):
                sh = shape.make(P, DEV)
                out, m, l = torch.zeros(1, 1, S.D, device=DEV), torch.zeros(1, 1, device=DEV), torch.zeros(1, 1, device=DEV)
                nbytes = P.prr_decode_shaped_workspace_size(dims, batch, sh, 0)
                ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=DEV)
                P.prr_decode_attn_shaped(dims, batch, sh, q[:1], 0, k, v, None, None, None, None, 0, out, None, m, l, ws, nbytes)
                torch.cuda.synchronize()
                check(out[0].double(), m[0].double(), l[0].double(), z, tol, v.flatten(0, 2)[:n],
                      torch.ones(1, n, dtype=torch.bool, device=DEV), S.half_step(DT[dt]), (cap, place, sign, i))


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("cap", CAPS)
def test_mass_caps_at_their_borders(cap, dt):
    """Weights of one token and of 150, relative to the largest score in 64 bits."""
    import paper_2606_30389_amd as P
    n = 150
    for place in PLACES:
        for sign in (1.0, -1.0):
            q, k, _, z, tol = inputs(cap, place, n, dt, sign)
            dims = P.make_dims(1, 1, 16, k.shape[1], P.PRR_BF16 if dt == "bf16" else P.PRR_F16)
            kv = torch.tensor([n], dtype=torch.int32, device=DEV)
            cu = torch.tensor([0, n], dtype=torch.int32, device=DEV)
            top = z.max().float()
            for new in (1, n):
                m, l = torch.full((new, 1), top.item(), device=DEV), torch.ones(new, 1, device=DEV)
                batch = P.make_batch(1, new, new, n, cu if new > 1 else None, kv)
                seen = torch.arange(n, 0, -1, device=DEV) if new > 1 else 1
                for i, shape in enumerate(shapes(cap)):
                    sh = shape.make(P, DEV)
                    mass = torch.zeros(1, k.shape[1], 16, device=DEV)
                    assert P.prr_mass_workspace_size(dims, batch, sh, 0) == 0
                    P.prr_key_mass(dims, batch, sh, q[:new], 0, k, None, m, l, 0, None, None, 0, None, 0.0, mass, None, 0)
                    torch.cuda.synchronize()
                    # (the exponent's two terms are rounded: 2^-22 of each; its sum over rows: 2^-16; each of the rows'
                    # weights below 2^-126 is 0, so `new` of them lose less than new * 2^-126)
                    want = seen * torch.exp(z - top.double())
                    off = torch.expm1(tol + (z.abs() + top.abs()) * 2.0 ** -22 + 2.0 ** -20) + 2.0 ** -16
                    e = (mass.flatten()[:n].double() - want).abs()
                    assert torch.all(e <= off * want + new * 2.0 ** -126), ((cap, place, sign, new, i), (e / (off * want)).max())
