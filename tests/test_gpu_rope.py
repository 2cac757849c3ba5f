"""prr_rope_append and prr_cache_read against 64 bits: layouts, parts of the head, far positions, packed and
ragged batches, strides, both kinds of cache; what must be left alone is."""
import math

import numpy as np
import pytest
import torch

from tests import context_support as S

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f16": torch.float16}


def lib():
    import paper_2606_30389_amd as P
    return P


def dims_of(P, hq, hkv, page, pool, dt):
    return P.make_dims(hq, hkv, page, pool, P.PRR_BF16 if dt == "bf16" else P.PRR_F16)


BATCHES = {
    "first": dict(new=[1], kv=[1], paged=False),
    "prompt": dict(new=[300], kv=[300], paged=False),
    "far": dict(new=[2], kv=[40000], paged=True),
    "tokens": dict(new=[1] * 70, kv=[1 + 37 * i % 500 for i in range(70)], single=True),
    "packed": dict(new=[0, 17, 1, 0, 130, 5, 0], kv=[9, 17, 400, 0, 200, 2, 33], pad=4),
    "one_of_many": dict(new=[0] * 200 + [3] + [0] * 100, kv=[1] * 200 + [50] + [1] * 100, pad=1),
}


def tolerance(exact, mag, dt):
    """One rounding to the type, and a float32 rotation: the fraction of a turn is off by at most 2^-25, cos and
    sin by 2 pi 2^-25 + 2^-23 < 2^-21.6, products and sum by 3 * 2^-24 more: under 2^-20 of |a| + |b|, scaled."""
    return S.half_step(DT[dt]) * (exact.abs() + mag * 2.0 ** -20) + mag * 2.0 ** -20 + (2.0 ** -25 if dt == "f16" else 0.0)


def run_case(batch, hq, hkv, dt, page, rot, layout, kv, scale=1.0, positions=None, parts="qkv", in_place=False):
    P = lib()
    b = S.Batch(page=page, device=DEV, seed=3, **batch)
    g = torch.Generator().manual_seed(S.seed_of(hq, hkv, dt, page, rot, layout, kv, b.total))
    qkv = torch.randn(b.total, hq + 2 * hkv, S.D, generator=g).to(DT[dt]).to(DEV)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    if in_place:
        q = q.contiguous()
    x64 = [t.cpu().clone() for t in (q, k, v)]
    freqs = torch.from_numpy(P.prr_rope_freqs(P.PRR_ROPE_PLAIN, max(2, rot), 10000.0)[0]).to(DEV)
    shape = (hkv, b.pool, page, S.D)
    if kv == "e4m3":
        caches = [torch.full(shape, 0x31, dtype=torch.uint8, device=DEV) for _ in range(2)]
        scales = [torch.full(shape[:3], 90, dtype=torch.uint8, device=DEV) for _ in range(2)]
    else:
        caches = [torch.full(shape, 3.0, dtype=DT[dt], device=DEV) for _ in range(2)]
        scales = [None, None]
    q_out = q if in_place else torch.full((b.total, hq, S.D), 5.0, dtype=DT[dt], device=DEV)
    before = q_out.cpu().clone()
    pos_t = None if positions is None else torch.tensor(positions, dtype=torch.int32, device=DEV)
    has_q, has_kv = "q" in parts, "kv" in parts
    P.prr_rope_append(dims_of(P, hq, hkv, page, b.pool, dt), b.make(P), q if has_q else None, k if has_kv else None,
                      v if has_kv else None, pos_t, freqs if rot else None, rot,
                      P.PRR_ROPE_INTERLEAVED if layout == "interleaved" else P.PRR_ROPE_HALF, scale,
                      q_out if has_q else None, P.PRR_KV_E4M3 if kv == "e4m3" else P.PRR_KV_16, caches[0] if has_kv else None,
                      caches[1] if has_kv else None, *(scales if has_kv else [None, None]))
    torch.cuda.synchronize()
    want_q = before.double()
    tol_q = torch.zeros_like(want_q)
    kept = [torch.full((hkv, b.pool * page), True) for _ in range(2)]
    got = [c.cpu().flatten(1, 2) for c in caches]
    got_s = [None if s is None else s.cpu().flatten(1, 2) for s in scales]
    for s, rows, pos in b.sequences():
        if not len(rows):
            continue
        rpos = pos if positions is None else torch.tensor(positions)[rows]
        y, mag = S.rotate64(x64[0][rows], rpos, freqs.cpu(), rot, layout == "interleaved", scale)
        want_q[rows], tol_q[rows] = y, tolerance(y, mag, dt)
        tol_q[rows] *= (mag > 0) | (torch.arange(S.D) < rot)  # plain channels are copied
        stored = pos >= 0
        if not stored.any() or not has_kv:
            continue
        slot = b.slots(s, int(pos[stored][0]), b.kv[s])
        for i, x in enumerate(x64[1:]):
            y, mag = S.rotate64(x[rows][stored], rpos[stored], freqs.cpu(), rot if i == 0 else 0, layout == "interleaved", scale)
            y, mag = y.transpose(0, 1), mag.transpose(0, 1)
            kept[i][:, slot] = False
            if kv == "e4m3":
                code, power, byte = S.quantise64(y, DT[dt])
                assert torch.equal(got_s[i][:, slot], byte)
                value = got[i][:, slot].view(torch.float8_e4m3fn).double() * power[..., None]
                # one rounding to e4m3 (subnormal: half of 2^-9 units) of a value that is off by the rotation's error
                tol = 2.0 ** -4 * (y.abs() + mag * 2.0 ** -20) + mag * 2.0 ** -20 + 2.0 ** -10 * power[..., None]
                assert torch.all((value - y).abs() <= tol)
                same = got[i][:, slot] == S.codes_of(code).view(torch.uint8)
                assert same.float().mean() > 0.9999  # (ties aside: a value within 2^-20 of one)
            else:
                tol = tolerance(y, mag, dt) * ((mag > 0) | (torch.arange(S.D) < (rot if i == 0 else 0)))
                assert torch.all((got[i][:, slot].double() - y).abs() <= tol)
    if has_q:
        assert torch.all((q_out.cpu().double() - want_q).abs() <= tol_q)
    else:
        assert torch.equal(q_out.cpu(), before)
    for i in range(2):  # everything else is left as it was
        assert torch.all(got[i][kept[i]] == (0x31 if kv == "e4m3" else 3.0))
        if kv == "e4m3":
            assert torch.all(got_s[i][kept[i]] == 90)


@pytest.mark.gpu
@pytest.mark.parametrize("kv", ["16", "e4m3"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("batch", list(BATCHES))
def test_rope_append_batches(batch, layout, kv):
    run_case(BATCHES[batch], 8, 2, "bf16", 16, 128, layout, kv)


@pytest.mark.gpu
@pytest.mark.parametrize("kv", ["16", "e4m3"])
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hkv,page,rot,layout,scale", [
    (1, 1, 16, 0, "half", 1.0), (32, 2, 16, 64, "interleaved", 1.0), (28, 4, 64, 96, "half", 1.25), (8, 8, 256, 8, "half", 1.0),
    (16, 1, 32, 24, "interleaved", 0.5), (5, 5, 128, 120, "half", 1.0), (64, 8, 16, 128, "half", 1.2079)])
def test_rope_append_shapes(hq, hkv, page, rot, layout, scale, dt, kv):
    run_case(BATCHES["packed"], hq, hkv, dt, page, rot, layout, kv, scale)


@pytest.mark.gpu
def test_rope_append_positions_parts_and_in_place():
    new = BATCHES["packed"]["new"]
    total = sum(new) + 4
    far = [(7919 * i) % 1000003 for i in range(total)]
    run_case(BATCHES["packed"], 4, 2, "bf16", 16, 128, "half", "16", positions=far)
    run_case(BATCHES["packed"], 4, 2, "f16", 16, 64, "interleaved", "e4m3", positions=[-x for x in far])
    run_case(BATCHES["packed"], 4, 2, "bf16", 16, 128, "half", "16", parts="q")
    run_case(BATCHES["packed"], 4, 2, "bf16", 16, 128, "half", "e4m3", parts="kv")
    run_case(BATCHES["prompt"], 4, 2, "bf16", 16, 128, "half", "16", in_place=True)
    run_case(BATCHES["tokens"], 4, 2, "f16", 16, 128, "interleaved", "16", in_place=True)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_rope_append_e4m3_extremes(dt):
    """Rows of zeros, the type's smallest and largest numbers, infinities and NaN, and rows whose largest value is
    448 * 2^k or just above it."""
    P = lib()
    big = torch.finfo(DT[dt]).max
    tiny = torch.finfo(DT[dt]).smallest_normal
    rows = torch.zeros(12, 1, S.D)
    rows[1, 0, 5] = tiny / 4
    rows[2, 0, :] = big
    rows[3, 0, 7] = math.inf
    rows[4, 0, 7], rows[4, 0, 8] = math.nan, 3.0
    rows[5, 0, 3] = 448.0 * 2 ** -6
    rows[6, 0, 3] = 448.0 * 2 ** -6 * (1 + 2.0 ** -7)
    rows[7, 0, 3], rows[7, 0, 4] = -1.0, tiny
    rows[8, 0, :] = torch.linspace(-3, 3, S.D)
    rows[9, 0, 0] = -0.0
    rows[10, 0, ::2] = 61440.0
    rows[11, 0, :] = -math.inf
    x = rows.to(DT[dt]).to(DEV)
    b = S.Batch([12], [12], 16, paged=False, device=DEV, spare=0)
    codes = [torch.zeros(1, 1, 16, S.D, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = [torch.zeros(1, 1, 16, dtype=torch.uint8, device=DEV) for _ in range(2)]
    d = dims_of(P, 1, 1, 16, 1, dt)
    P.prr_rope_append(d, b.make(P), None, x, x, None, None, 0, P.PRR_ROPE_HALF, 1.0, None, P.PRR_KV_E4M3, *codes, *scales)
    back = [torch.full((1, 1, 16, S.D), 7.0, dtype=DT[dt], device=DEV) for _ in range(2)]
    P.prr_cache_read(d, *codes, *scales, None, 12, 0, 1, *back)
    torch.cuda.synchronize()
    assert torch.equal(codes[0], codes[1]) and torch.equal(scales[0], scales[1])
    clean = torch.nan_to_num(x.cpu().float(), nan=0.0, posinf=math.inf, neginf=-math.inf)
    code, power, byte = S.quantise64(clean[:, 0], DT[dt])
    assert torch.equal(scales[0].cpu()[0, 0, :12], byte)
    want = (code * power[:, None]).to(DT[dt])
    got = back[0].cpu()[0, 0]
    nan = x.cpu()[:, 0].isnan()
    assert torch.equal(got[:12].isnan(), nan) and torch.all(got[:12][~nan].isfinite())
    assert torch.equal(got[:12][~nan], want[~nan])
    assert torch.all(got[12:] == 7.0) and torch.equal(back[0][0, 0, :12].isnan(), back[1][0, 0, :12].isnan())


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("hkv,page,tokens,first,last,paged", [(1, 16, 1, 0, 1, False), (2, 16, 1000, 0, 63, True),
                                                              (8, 64, 777, 5, 13, True), (3, 256, 1024, 1, 4, False),
                                                              (2, 32, 100, 2, 2, True), (1, 128, 129, 0, 2, True)])
def test_cache_read(hkv, page, tokens, first, last, paged, dt):
    P = lib()
    b = S.Batch([1], [tokens], page, paged=paged, device=DEV, seed=5)
    g = torch.Generator().manual_seed(tokens)
    shape = (hkv, b.pool, page, S.D)
    codes = [torch.randint(0, 256, shape, generator=g, dtype=torch.uint8) for _ in range(2)]
    for c in codes:
        c[(c & 127) == 127] = 0x38
    lo, hi = (1, 246) if dt == "bf16" else (90, 134)  # every number stays below the type's largest
    scales = [torch.randint(lo, hi, shape[:3], generator=g, dtype=torch.uint8) for _ in range(2)]
    out = [torch.full((hkv, max(1, last - first), page, S.D), 7.0, dtype=DT[dt], device=DEV) for _ in range(2)]
    P.prr_cache_read(dims_of(P, hkv, hkv, page, b.pool, dt), *[c.to(DEV) for c in codes], *[s.to(DEV) for s in scales],
                     b.d_table if paged else None, tokens, first, last, *out)
    torch.cuda.synchronize()
    n = min(tokens, last * page) - first * page
    for c, s, o in zip(codes, scales, out):
        got = o.cpu().flatten(1, 2)
        if n > 0:
            slot = b.slots(0, first * page, first * page + n)
            want = c.view(torch.float8_e4m3fn).double().flatten(1, 2)[:, slot] * torch.exp2(s.double() - 127).flatten(1, 2)[:, slot, None]
            assert torch.equal(got[:, :n], want.to(DT[dt]))
        assert torch.all(got[:, max(0, n):] == 7.0)


@pytest.mark.gpu
def test_bad_pages_are_left_out():
    """Page-table entries out of range: nothing is stored or read there, everything else is served."""
    P = lib()
    b = S.Batch([40], [40], 16, device=DEV, seed=1)
    b.table[0, 1] = 1 << 30
    b.d_table = b.table.to(DEV)
    x = torch.randn(40, 2, S.D, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    d = dims_of(P, 2, 2, 16, b.pool, "bf16")
    caches = [torch.full((2, b.pool, 16, S.D), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    P.prr_rope_append(d, b.make(P), None, x, x, None, None, 0, P.PRR_ROPE_HALF, 1.0, None, P.PRR_KV_16, *caches)
    torch.cuda.synchronize()
    good = torch.cat([b.slots(0, 0, 16), b.slots(0, 32, 40)])
    got = caches[0].cpu().flatten(1, 2)
    assert torch.equal(got[:, good], x.cpu()[torch.cat([torch.arange(16), torch.arange(32, 40)])].transpose(0, 1))
    rest = torch.ones(b.pool * 16, dtype=torch.bool)
    rest[good] = False
    assert torch.all(got[:, rest] == 3.0)
    codes = [torch.full((2, b.pool, 16, S.D), 0x38, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = [torch.full((2, b.pool, 16), 127, dtype=torch.uint8, device=DEV) for _ in range(2)]
    out = [torch.full((2, 3, 16, S.D), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    P.prr_cache_read(d, *codes, *scales, b.d_table, 40, 0, 3, *out)
    torch.cuda.synchronize()
    for o in out:
        assert torch.all(o[:, 0] == 1.0) and torch.all(o[:, 1] == 7.0)
        assert torch.all(o[:, 2, :8] == 1.0) and torch.all(o[:, 2, 8:] == 7.0)
