"""Attention over caches whose values lie far apart: rows that one channel or a scale makes large, keys that outweigh all
others, infinities.  Every channel is held to its own bound: what is large in one channel excuses nothing in
another."""
import math

import pytest
import torch

from tests import context_support as S

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f16": torch.float16}


def decode(cache, scale, q, kv, dt):
    """prr_decode_attn of one sequence of kv tokens over an identity table: o32, o, m, l."""
    import paper_2606_30389_amd as P
    hq, hkv, pool, page = q.shape[1], *cache[0].shape[:3]
    dims = P.make_dims(hq, hkv, page, pool, P.PRR_BF16 if dt == "bf16" else P.PRR_F16)
    kind = P.PRR_KV_16 if scale[0] is None else P.PRR_KV_E4M3
    lens = torch.tensor([kv], dtype=torch.int32, device=DEV)
    batch = P.make_batch(1, 1, 1, kv, None, lens)
    nbytes = P.prr_decode_workspace_size(dims, batch, kind)
    ws = torch.full((max(nbytes, 256),), 0xff, dtype=torch.uint8, device=DEV)
    out = [torch.empty(1, hq, S.D, device=DEV), torch.empty(1, hq, S.D, dtype=DT[dt], device=DEV), torch.empty(1, hq, device=DEV),
           torch.empty(1, hq, device=DEV)]
    P.prr_decode_attn(dims, batch, q, kind, *cache, *scale, None, None, 0, *out, ws, nbytes)
    torch.cuda.synchronize()
    return out


def check(out, q, k, v, weight_err, floor=0.0, dt="bf16", what=""):
    """k, v [Hkv][kv][128] in 64 bits; floor [Hq][128] or a number."""
    hkv = k.shape[0]
    G = q.shape[1] // hkv
    for h in range(hkv):
        heads = slice(h * G, (h + 1) * G)
        o, m, l, a, mag = S.attend64(q[0, heads].double(), k[h], v[h])
        fl = floor[heads] if torch.is_tensor(floor) else floor
        got = [x[0, heads].double() for x in out]
        S.check_state(got[0], got[2], got[3], o, m, l, a, mag, weight_err, 2.0 ** -22, k.shape[1], fl, (what, h))
        eps = S.half_step(DT[dt])
        # (beyond the 16-bit type's largest number and half a step more, rounding gives infinity)
        far = o.abs() > torch.finfo(DT[dt]).max * (1 + eps)
        assert torch.equal(got[1][far], o[far].sign() * math.inf), what
        o, got[1] = o.masked_fill(far, 0.0), got[1].masked_fill(far, 0.0)
        S.check_state(got[1], got[2], got[3], o, m, l, a, mag, weight_err + eps, eps, k.shape[1],
                      fl + (2.0 ** -25 if dt == "f16" else 0.0), (what, h))


def e4m3_rows(code, scale, kv):
    """The numbers of an e4m3 cache's first kv rows (identity table)."""
    p = torch.exp2(scale.flatten(1, 2)[:, :kv].double() - 127)
    return code.view(torch.float8_e4m3fn).flatten(1, 2)[:, :kv].double() * p[..., None]


@pytest.mark.gpu
@pytest.mark.parametrize("dt,outlier", [("bf16", 1e4), ("bf16", 1e6), ("bf16", 3e38), ("bf16", math.inf), ("f16", 6e4), ("f16", -math.inf)])
@pytest.mark.parametrize("kv,at", [(16, 5), (700, 0), (700, 699), (4096, 2000), (20011, 3)])
def test_e4m3_row_with_one_large_channel(kv, at, dt, outlier):
    """One row's value is far larger in channel 0 than anything else: the other channels keep their accuracy.
    Weights are three bfloat16 terms."""
    from paper_2606_30389_amd import runtime as R
    pc = R.PathConfig(num_q_heads=8, num_kv_heads=2, page_size=16, num_tokens=kv, k_select=1, dtype=dt)
    cache = R.PagedCache(pc, DEV, kind="e4m3")
    g = torch.Generator(device=DEV).manual_seed(kv + at)
    k, v = (torch.randn(kv, 2, S.D, generator=g, device=DEV).to(DT[dt]) for _ in range(2))
    v[at, :, 0] = outlier
    q = (1.5 * torch.randn(1, 8, S.D, generator=g, device=DEV)).to(DT[dt])
    cache.append(R.Batch(DEV, [kv], [kv]), None, k, v)
    codes, scales = (cache.k.view(torch.uint8), cache.v.view(torch.uint8)), (cache.k_scale, cache.v_scale)
    out = decode(codes, scales, q, kv, dt)
    check(out, q, e4m3_rows(codes[0], scales[0], kv), e4m3_rows(codes[1], scales[1], kv), 2.0 ** -24, 2.0 ** -126, dt, outlier)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("large,small", [(254, 120), (200, 20), (150, 149), (60, 1), (1, 1)])
@pytest.mark.parametrize("kv", [16, 1000])
def test_e4m3_scales_of_rows_that_are_empty_where_it_matters(kv, large, small, dt):
    """Rows with a large scale byte hold zeros (every third row) or one number in channel 0 (one row): the other rows
    decide every other channel."""
    g = torch.Generator(device=DEV).manual_seed(kv + large)
    pages = -(-kv // 16)
    codes = [(40 * torch.randn(2, pages, 16, S.D, generator=g, device=DEV)).to(torch.float8_e4m3fn).view(torch.uint8) for _ in range(2)]
    scales = [torch.full((2, pages, 16), b, dtype=torch.uint8, device=DEV) for b in (120, small)]
    v, s = codes[1].flatten(1, 2), scales[1].flatten(1, 2)
    v[:, 1::3] = 0
    s[:, 1::3] = large
    v[:, 4, 0] = 0x38  # 1.0
    q = torch.randn(1, 8, S.D, generator=g, device=DEV).to(DT[dt])
    out = decode(codes, scales, q, kv, dt)
    # (numbers below 2^-126 are of no account)
    check(out, q, e4m3_rows(codes[0], scales[0], kv), e4m3_rows(codes[1], scales[1], kv), 2.0 ** -24, 2.0 ** -125, dt, (large, small))


def one_key_above(kv, at, nats, hkv, dt):
    """Caches in which one key lies `nats` above all others, which are alike, and its value is 0."""
    g = torch.Generator(device=DEV).manual_seed(kv + at)
    pages = -(-kv // 16)
    k, v = torch.zeros(hkv, pages, 16, S.D, device=DEV), 0.5 + torch.randn(hkv, pages, 16, S.D, generator=g, device=DEV)
    k.flatten(1, 2)[:, at] = nats / math.sqrt(S.D)
    v.flatten(1, 2)[:, at] = 0.0
    return k.to(DT[dt]), v.to(DT[dt])


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("nats", [10.0, 17.0, 20.0, 25.0])
@pytest.mark.parametrize("kv,at", [(1000, 999), (131072, 7)])
def test_decode_keys_far_below_one(kv, at, nats, dt):
    """Two float16 terms of a weight are off by 2^-22, or by 2^-39 of the largest weight among the 16 tokens of a tile
    (subnormal terms): that much of the largest |v| of the channel, for each token."""
    k, v = one_key_above(kv, at, nats, 2, dt)
    q = torch.ones(1, 8, S.D, device=DEV, dtype=DT[dt])
    out = decode((k, v), (None, None), q, kv, dt)
    k64, v64 = (x.flatten(1, 2)[:, :kv].double() for x in (k, v))
    werr, floor = 2.0 ** -24, 0.0
    if dt == "f16":
        tops = 1.0 + kv / 16 * math.exp(-nats * 0.999)  # (sum over tiles of their largest weights; l > 1)
        werr, floor = 2.0 ** -22, (2.0 ** -39 * 16 * tops * v64.abs().amax(1)).repeat_interleave(4, 0)
    check(out, q, k64, v64, werr, floor, dt, nats)


@pytest.mark.gpu
@pytest.mark.parametrize("nats", [10.0, 15.0, 17.0, 20.0])
@pytest.mark.parametrize("kv,new,at", [(1000, 40, 7), (20000, 300, 19000), (1500, 1500, 3)])
def test_prompt_keys_far_below_one(kv, new, at, nats):
    """float16 weights of a prompt are off by 2^-11, or by 2^-36 of the row's largest (subnormal)."""
    import paper_2606_30389_amd as P
    from paper_2606_30389_amd import runtime as R
    k, v = one_key_above(kv, at, nats, 2, "f16")
    pc = R.PathConfig(num_q_heads=4, num_kv_heads=2, page_size=16, num_tokens=kv, k_select=1, dtype="f16")
    cache = R.PagedCache(pc, DEV, k=k, v=v)
    q = torch.ones(new, 4, S.D, device=DEV, dtype=torch.float16)
    got = cache.prompt(R.Batch(DEV, [new], [kv]), q)
    torch.cuda.synchronize()
    assert P.PRR_KV_16 == cache.kind
    pos = torch.arange(kv - new, kv, device=DEV)
    eps = S.half_step(torch.float16)
    for h in range(4):
        k64, v64 = (x.flatten(1, 2)[h // 2, :kv].double() for x in (k, v))
        seen = torch.arange(kv, device=DEV) <= pos[:, None]
        o, m, l, a, mag = S.attend64(q[:, h].double(), k64, v64, seen)
        floor = 2.0 ** -36 * kv * v64.abs().amax(0) / l[:, None] + 2.0 ** -25
        S.check_state(got[0][:, h].double(), got[1][:, h].double(), got[2][:, h].double(), o, m, l, a, mag, eps, eps, kv, floor, (h, nats))


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("kv,at", [(1, 0), (40, 39), (700, 3), (9000, 8123)])
def test_decode_infinite_values(kv, at, dt):
    """A value of infinity makes its channel that infinity, two of both signs or a NaN make it NaN; the other channels do
    not change."""
    g = torch.Generator(device=DEV).manual_seed(kv)
    pages = -(-kv // 16)
    k, v = (torch.randn(2, pages, 16, S.D, generator=g, device=DEV).to(DT[dt]) for _ in range(2))
    q = torch.randn(1, 8, S.D, generator=g, device=DEV).to(DT[dt])
    clean = decode((k, v), (None, None), q, kv, dt)
    dirty = v.clone()
    rows = dirty.flatten(1, 2)
    rows[0, at, 5], rows[0, at, 127], rows[0, at, 64] = math.inf, -math.inf, math.nan
    rows[1, at, 0] = math.inf
    if kv > 1:
        rows[0, at - 1, 5], rows[1, at - 1, 0] = math.inf, -math.inf
    out = decode((k, dirty), (None, None), q, kv, dt)
    for o in (x[0].float() for x in out[:2]):
        assert torch.all(o[:4, 5] == math.inf) and torch.all(o[:4, 127] == -math.inf) and torch.all(o[:4, 64].isnan())
        assert torch.all(o[4:, 0].isnan() if kv > 1 else o[4:, 0] == math.inf)
    same = torch.ones(8, S.D, dtype=torch.bool, device=DEV)
    same[:4, [5, 64, 127]] = False
    same[4:, 0] = False
    assert all(torch.equal(x[0][same], y[0][same]) for x, y in zip(out[:2], clean[:2]))
    assert torch.equal(out[2], clean[2]) and torch.equal(out[3], clean[3])
