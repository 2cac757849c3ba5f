"""prr_key_mass, prr_keep_tokens and prr_cache_compact against plain implementations, alone and one after the other."""
import math

import pytest
import torch

from tests import context_support as S
from tests.shape_support import Shape, keep_of, slopes_of

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f16": torch.float16}


# ------------------------------------------------------------------------------- received weight

def mass_case(new, kv, hq, hkv, dt="bf16", page=16, kind="16", pad=0, paged=True, shape=None, last=0, decay=None, lists=None,
              spread=1.5, single=False, edit=None, alias=False):
    import paper_2606_30389_amd as P
    b = S.Batch(new, kv, page, pad=pad, paged=paged, device=DEV, seed=3, single=single)
    G = hq // hkv
    g = torch.Generator(device=DEV).manual_seed(S.seed_of(new, kv, hq, hkv, dt, page, kind, last))
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    q = (spread * rand(b.total, hq, S.D)).to(DT[dt])
    sizes = (hkv, b.pool, page, S.D)
    used = torch.zeros(b.pool * page, dtype=torch.bool)
    for s, n in enumerate(kv):
        used[b.slots(s, 0, n)] = True
    unused = ~used.to(DEV)
    scale = None
    if kind == "e4m3":
        k = (40 * rand(*sizes)).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        scale = torch.randint(120, 124, sizes[:3], generator=g, device=DEV, dtype=torch.uint8)
        k.flatten(1, 2)[:, unused] = 0x7f
        scale.flatten(1, 2)[:, unused] = 255
        keys = k.view(torch.float8_e4m3fn).double() * torch.exp2(scale.double() - 127)[..., None]
    else:
        k = rand(*sizes).to(DT[dt])
        k.flatten(1, 2)[:, unused] = math.nan
        keys = k.double()
    shape = Shape() if shape is None else shape
    if shape.first is not None:
        shape.first = list(shape.first) + [10 ** 9] * pad
    before = None if decay is None else torch.rand(sizes[:3], generator=g, device=DEV)
    if edit:
        edit(b, q, keys, before)
    # statistics of the attention in 64 bits, rounded; NaN for rows that no sequence has
    m, l = torch.full((b.total, hq), math.nan, device=DEV), torch.full((b.total, hq), math.nan, device=DEV)
    want = torch.full(sizes[:3], math.nan, dtype=torch.float64, device=DEV).flatten(1, 2)
    tol = torch.zeros_like(want)
    written = torch.zeros(hkv, b.pool * page, dtype=torch.bool, device=DEV)
    for s, rows, pos in b.sequences():
        n = kv[s]
        if n == 0:
            for x in (m, l):
                x[rows.to(DEV)] = 0.0
            continue
        vis = shape.visible(s, rows, pos, n).to(DEV).repeat_interleave(G, 0)
        rows, pos = rows.to(DEV), pos.to(DEV).repeat_interleave(G, 0)
        counted = torch.arange(len(rows), device=DEV) >= len(rows) - (min(last, len(rows)) if last else len(rows))
        counted = counted.repeat_interleave(G, 0)
        slot = b.slots(s, 0, n).to(DEV)
        for h in range(hkv):
            kk = keys[h].flatten(0, 1)[slot]
            heads = slice(h * G, (h + 1) * G)
            head = (h * G + torch.arange(G, device=DEV)).repeat(len(rows))
            z, mag = shape.scores(q[rows, heads].double().reshape(-1, S.D), kk, pos, head)
            z = z.masked_fill(~vis, -math.inf)
            m64 = z.amax(-1)
            l64 = torch.exp(z - torch.where(m64.isinf(), 0.0, m64)[:, None]).sum(-1)
            if len(rows):
                m[rows, heads], l[rows, heads] = m64.float().view(-1, G), l64.float().view(-1, G)
            mf, lf = m64.float().double(), l64.float().double()
            w = torch.exp(z - torch.where(mf.isinf(), 0.0, mf)[:, None]) / torch.where(lf == 0, 1.0, lf)[:, None]
            w = torch.where(counted[:, None], w, 0.0)
            # a weight: its score's error (S.check_state's dm), the reference exponent's |m| + ln l and the exponential
            # below 2^-16 together; a sum of up to 2^18 of them in a fixed order 2^-16 (128 + n / 2048 additions of 2^-24, and
            # the lanes' and parts'); weights below 2^-126 are 0
            t = (w * (mag[:, None] * 2.0 ** -16 + 2.0 ** -15)).sum(0) + len(w) * 2.0 ** -120
            total = w.sum(0)
            if before is not None:
                was = decay * before[h].flatten()[slot].double()
                t = t + (was.abs() + total) * 2.0 ** -23
                total = total + was
            on = torch.ones(n, dtype=torch.bool, device=DEV)
            if lists is not None:
                on = torch.isin(torch.arange(n, device=DEV) // page, torch.tensor(lists[s], dtype=torch.long, device=DEV))
            want[h, slot[on]], tol[h, slot[on]] = total[on], t[on]
            written[h, slot[on]] = True
    dims = P.make_dims(hq, hkv, page, b.pool, P.PRR_BF16 if dt == "bf16" else P.PRR_F16)
    batch, sh = b.make(P), shape.make(P, DEV)
    pages = count = None
    if lists is not None:
        pages = torch.full((len(kv), hkv, max(1, max(len(x) for x in lists))), -3, dtype=torch.int32)
        for s, x in enumerate(lists):
            pages[s, :, :len(x)] = torch.tensor(x, dtype=torch.int32)
        pages, count = pages.to(DEV), torch.tensor([[len(x)] * hkv for x in lists], dtype=torch.int32, device=DEV)
    code, cap = P.PRR_KV_E4M3 if kind == "e4m3" else P.PRR_KV_16, 0 if pages is None else pages.shape[-1]
    nbytes = P.prr_mass_workspace_size(dims, batch, sh, code, last, cap)
    ws = torch.full((max(nbytes, 256),), 0xff, dtype=torch.uint8, device=DEV)

    def call(out, src=before):
        P.prr_key_mass(dims, batch, sh, q, code, k, scale, m, l, last, pages, count, cap, src, 0.0 if decay is None else decay, out,
                       ws, nbytes)
        torch.cuda.synchronize()
        return out

    got = call(torch.full(sizes[:3], 5.0, device=DEV))
    flat = got.flatten(1, 2).double()
    assert torch.all(flat[~written] == 5.0)
    e = (flat - want).abs()[written]
    assert torch.all(e <= tol[written]), ((e / tol[written]).max(), (new, kv))
    assert torch.equal(call(torch.full(sizes[:3], 5.0, device=DEV)), got)  # the same bits
    if alias:
        x = before.clone()
        call(x, x)
        assert torch.equal(x.flatten(1, 2)[written], got.flatten(1, 2)[written])
        assert torch.equal(x.flatten(1, 2)[~written], before.flatten(1, 2)[~written])
    return P, dims, batch, sh, q, k, m, l, got, call, nbytes


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["16", "e4m3"])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 65, 130, 257, 700])
def test_mass_lengths(n, kind):
    mass_case([n], [n], 16, 1, kind=kind)
    mass_case([n], [n + 41], 4, 4, dt="f16", kind=kind, paged=False, decay=0.9, alias=True)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["16", "e4m3"])
@pytest.mark.parametrize("hq,hkv,page,dt", [(1, 1, 16, "bf16"), (32, 2, 16, "f16"), (28, 4, 64, "bf16"), (5, 1, 32, "f16"),
                                            (8, 8, 256, "bf16"), (36, 3, 128, "f16")])
def test_mass_heads_and_pages(hq, hkv, page, dt, kind):
    mass_case([300, 0, 1, 45], [300, 7, 500, 111], hq, hkv, dt, page, kind, pad=3, decay=1.0)


def shapes(new, kv, hq):
    rows = [(n, k, i) for n, k in zip(new, kv) for i in range(n)]
    size = max(1, max(kv) // 3)
    return {"cap": Shape(cap=3.0), "slopes": Shape(slopes=slopes_of(hq)), "window": Shape(window=max(1, max(kv) // 4)),
            "docs": Shape(first=[max(0, k - n + i) // size * size for n, k, i in rows]),
            "prefix": Shape(prefix=[(7 * k) // 9 for k in kv]),
            "all": Shape(cap=5.0, slopes=slopes_of(hq), window=max(1, max(kv) // 2), first=[max(0, k - n + i) // size * size for n, k, i in rows],
                         prefix=[(7 * k) // 9 for k in kv])}


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["cap", "slopes", "window", "docs", "prefix", "all"])
@pytest.mark.parametrize("new,kv,hq,hkv", [([200], [200], 16, 1), ([333, 20, 1], [400, 900, 77], 8, 2), ([1500], [1700], 2, 2)])
def test_mass_shapes(new, kv, hq, hkv, which):
    mass_case(new, kv, hq, hkv, shape=shapes(new, kv, hq)[which], pad=1)
    mass_case(new, kv, hq, hkv, dt="f16", kind="e4m3", shape=shapes(new, kv, hq)[which], last=130)


@pytest.mark.gpu
@pytest.mark.parametrize("last", [1, 7, 32, 1000])
def test_mass_of_the_last_tokens(last):
    mass_case([100, 3, 40], [3000, 3, 90], 16, 2, last=last)
    mass_case([500], [500], 4, 1, last=last, paged=False, dt="f16")


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["16", "e4m3"])
@pytest.mark.parametrize("kv", [[1], [5000], [1, 0, 700, 16, 5000, 33], [20011], [3] * 70])
def test_mass_single_tokens(kv, kind):
    mass_case([1] * len(kv), kv, 16, 2, kind=kind, single=True, decay=0.5, pad=2, alias=True)
    mass_case([1] * len(kv), kv, 3, 3, dt="f16", kind=kind, single=True, shape=Shape(window=100, cap=2.0))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["16", "e4m3"])
def test_mass_listed_pages(kind):
    """The statistics are those of the whole cache here; only listed tokens are written."""
    lists = [[5, 0, 61, 30, 31], [2, -7, 2 ** 30], [], [0, 1, 2, 3], [3]]
    for page in (16, 64):
        mass_case([1] * 5, [1000, 40, 500, 60, 50], 8, 2, page=page, kind=kind, single=True, lists=lists, decay=1.0, alias=True)
    mass_case([1], [9999], 16, 1, kind=kind, single=True, lists=[list(range(624, 0, -3))], shape=Shape(window=4000, slopes=slopes_of(16)))


@pytest.mark.gpu
def test_mass_rows_split():
    """Few keys and many rows: the rows are split over workgroups and joined."""
    *_, nbytes = mass_case([3000], [3000], 16, 1)
    assert nbytes > 0
    *_, nbytes = mass_case([1100, 1, 900], [1100, 50, 901], 8, 1, decay=0.25, dt="f16", kind="e4m3", pad=3, shape=Shape(window=999), alias=True)
    assert nbytes > 0


@pytest.mark.gpu
def test_mass_many_sequences():
    new = [(37 * i) % 23 for i in range(150)]
    kv = [n + (53 * i) % 91 * (i % 3 > 0) for i, n in enumerate(new)]
    mass_case(new, kv, 8, 2, pad=2, decay=1.0)


@pytest.mark.gpu
def test_mass_tokens_without_a_place():
    mass_case([10, 70, 4], [3, 0, 4], 8, 2, pad=2, decay=1.0)
    mass_case([300], [130], 16, 1, dt="f16", shape=Shape(prefix=[100]))


@pytest.mark.gpu
@pytest.mark.parametrize("spread,cap", [(0.0, 0.0), (12.0, 0.0), (40.0, 30.0)])
def test_mass_flat_and_sharp(spread, cap):
    mass_case([200], [260], 8, 2, spread=spread, shape=Shape(cap=cap))


@pytest.mark.gpu
def test_mass_weights_sum_to_the_rows():
    """Without a shape every counted token spreads a weight of one per head."""
    P, dims, batch, sh, q, k, m, l, got, call, _ = mass_case([400], [900], 8, 2)
    assert abs(got[got != 5.0].double().sum().item() / (400 * 8) - 1) < 2 ** -12


@pytest.mark.gpu
def test_mass_nan_and_empty_rows():
    """A row with l = 0 gives nothing; one of NaN gives NaN to the tokens that it sees and to no other."""
    P, dims, batch, sh, q, k, m, l, got, call, _ = mass_case([50], [120], 4, 1, paged=False)
    l[20] = 0.0
    m[20] = -math.inf
    x = call(torch.full_like(got, 5.0))
    flat, was = x.flatten(), got.flatten()
    assert torch.all(flat[:91] <= was[:91]) and torch.all(flat[:91] >= 0) and torch.equal(flat[91:], was[91:])
    l[20] = 3.0
    m[20] = math.nan
    x = call(torch.full_like(got, 5.0)).flatten()
    assert torch.all(x[:91].isnan()) and torch.equal(x[91:], was[91:])
    q[49] = math.nan
    m[20] = 0.0
    x = call(torch.full_like(got, 5.0)).flatten()
    assert torch.all(x[:120].isnan()) and torch.all(x[120:] == 5.0)


@pytest.mark.gpu
def test_mass_bad_pages_are_skipped():
    import paper_2606_30389_amd as P
    table = torch.tensor([[0, -1, 5, 2 ** 30, 2]], dtype=torch.int32, device=DEV)
    q = torch.randn(1, 4, S.D, device=DEV).to(torch.bfloat16)
    k = torch.randn(2, 5, 16, S.D, device=DEV).to(torch.bfloat16)
    batch = P.make_batch(1, 1, 1, 80, None, torch.tensor([80], dtype=torch.int32, device=DEV), table, 5)
    out, one = torch.full((2, 5, 16), 7.0, device=DEV), torch.ones(1, 4, device=DEV)
    P.prr_key_mass(P.make_dims(4, 2, 16, 5, P.PRR_BF16), batch, None, q, 0, k, None, one, one, 0, None, None, 0, None, 0.0, out, None, 0)
    torch.cuda.synchronize()
    assert torch.all(out[:, [1, 3, 4]] == 7.0) and torch.all(out[:, [0, 2]] != 7.0)


# ------------------------------------------------------------------------------- choice

def keep_case(kv, budget, sink=0, recent=0, hkv=2, page=16, paged=True, values="random", seed=0):
    import paper_2606_30389_amd as P
    b = S.Batch([1] * len(kv), kv, page, paged=paged, device=DEV, seed=seed, single=True)
    g = torch.Generator(device=DEV).manual_seed(S.seed_of(kv, budget, values))
    shape = (hkv, b.pool, page)
    mass = torch.exp(2 * torch.randn(shape, generator=g, device=DEV))
    if values == "ties":
        mass = torch.randint(0, 4, shape, generator=g, device=DEV).float()
    elif values == "equal":
        mass = torch.full(shape, 0.25, device=DEV)
    elif values == "signs":
        mass = torch.randn(shape, generator=g, device=DEV)
        mass[mass.abs() < 0.1] = 0.0
        mass[(mass > 0.5) & (mass < 0.6)] = -0.0
    elif values == "odd":
        pick = torch.randint(0, 8, shape, generator=g, device=DEV)
        for i, x in enumerate((math.nan, math.inf, -math.inf, 1e-45, -1e-45, 3.4e38)):
            mass[pick == i] = x
        mass[mass.isnan() & (torch.rand(shape, generator=g, device=DEV) < 0.5)] = -math.nan
    elif values == "close":  # the last bits decide
        mass = (torch.randint(0, 5000, shape, generator=g, device=DEV, dtype=torch.int32) + 0x3f800000).view(torch.float32)
    dims, batch = P.make_dims(hkv, hkv, page, b.pool, P.PRR_BF16), b.make(P)
    nbytes = P.prr_keep_workspace_size(dims, batch, budget)
    ws = torch.full((max(nbytes, 256),), 0xff, dtype=torch.uint8, device=DEV)
    keep = torch.full((len(kv), hkv, budget), -9, dtype=torch.int32, device=DEV)
    kept = torch.full((len(kv),), -9, dtype=torch.int32, device=DEV)
    P.prr_keep_tokens(dims, batch, mass, budget, sink, recent, keep, kept, ws, nbytes)
    torch.cuda.synchronize()
    assert kept.tolist() == [min(budget, n) for n in kv]
    flat = mass.flatten(1, 2).cpu()
    for s, n in enumerate(kv):
        for h in range(hkv):
            want = keep_of(flat[h, b.slots(s, 0, n)].tolist(), budget, sink, recent)
            assert keep[s, h, :len(want)].tolist() == want, (s, h, n)
            assert torch.all(keep[s, h, len(want):] == -9)
    return P, dims, batch, mass, keep, kept, ws, nbytes


@pytest.mark.gpu
@pytest.mark.parametrize("values", ["random", "ties", "equal", "signs", "odd", "close"])
@pytest.mark.parametrize("n,budget", [(1, 1), (5, 3), (64, 63), (100, 1), (1000, 300), (4096, 4095), (4097, 100), (9001, 2000), (20000, 7)])
def test_keep_lengths(n, budget, values):
    keep_case([n], budget, values=values)
    keep_case([n], budget, sink=min(4, budget), recent=min(9, budget - min(4, budget)), values=values, paged=False, hkv=1)


@pytest.mark.gpu
@pytest.mark.parametrize("values", ["random", "ties", "equal", "odd", "close"])
@pytest.mark.parametrize("n,budget", [(32769, 5000), (70001, 70000), (131072, 40), (100003, 30000)])
def test_keep_long(n, budget, values):
    """More than one workgroup's tokens: chunks."""
    P, dims, batch, *_ , nbytes = keep_case([n], budget, sink=3, recent=30, values=values, page=64)
    assert nbytes > 0


@pytest.mark.gpu
@pytest.mark.parametrize("values", ["random", "ties"])
def test_keep_ragged(values):
    keep_case([0, 1, 16, 17, 500, 2049, 33], 100, sink=4, recent=16, values=values, hkv=3)
    keep_case([0, 40000, 1, 8192, 8193, 100, 16384, 33000], 8000, sink=4, recent=100, values=values, page=128)


@pytest.mark.gpu
@pytest.mark.parametrize("sink,recent", [(0, 0), (10, 0), (0, 10), (4, 6), (10, 40), (0, 50)])
def test_keep_sinks_and_recent(sink, recent):
    keep_case([50, 51, 60, 200], 50, sink, recent)
    keep_case([40000, 51], 50, sink, recent)


@pytest.mark.gpu
def test_keep_one_chunk_boundary():
    """Always kept tokens that cross the chunks' borders."""
    keep_case([40000], 30000, sink=9000, recent=20000)
    keep_case([40000], 30000, sink=0, recent=30000, values="ties")
    keep_case([40000], 30000, sink=30000, recent=0, values="ties")


@pytest.mark.gpu
def test_keep_bad_pages_have_no_mass():
    import paper_2606_30389_amd as P
    table = torch.tensor([[0, -1, 2, 2 ** 30, 1]], dtype=torch.int32, device=DEV)
    mass = torch.rand(1, 3, 16, device=DEV)
    batch = P.make_batch(1, 1, 1, 80, None, torch.tensor([80], dtype=torch.int32, device=DEV), table, 5)
    keep, kept = torch.zeros(1, 1, 50, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    P.prr_keep_tokens(P.make_dims(1, 1, 16, 3, P.PRR_BF16), batch, mass, 50, 0, 0, keep, kept, None, 0)
    torch.cuda.synchronize()
    assert keep[0, 0].tolist() == [*range(16), 16, 17, *range(32, 48), *range(64, 80)]


# ------------------------------------------------------------------------------- moves

def compact_case(kv, budget, hkv=2, page=16, kind="16", in_place=True, paged=True, mass=True, dt="bf16", order="kept"):
    import paper_2606_30389_amd as P
    b = S.Batch([1] * len(kv), kv, page, paged=paged, device=DEV, seed=5, single=True, spare=0 if in_place else sum(-(-min(n, budget) // page) for n in kv) + 2)
    g = torch.Generator(device=DEV).manual_seed(S.seed_of(kv, budget, kind))
    sizes = (hkv, b.pool, page, S.D)
    if kind == "e4m3":
        cache = [torch.randint(0, 256, sizes, generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
        scale = [torch.randint(0, 256, sizes[:3], generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
    else:
        cache = [torch.randint(-2 ** 15, 2 ** 15, sizes, generator=g, device=DEV, dtype=torch.int16).view(DT[dt]) for _ in range(2)]
        scale = []
    held = torch.rand(sizes[:3], generator=g, device=DEV) if mass else None
    kept = [min(budget, n) for n in kv]
    keep = torch.full((len(kv), hkv, budget), 2 ** 30, dtype=torch.int32)
    for s, n in enumerate(kv):
        for h in range(hkv):
            x = torch.randperm(n)[:kept[s]]
            keep[s, h, :kept[s]] = (x.sort().values if order == "kept" else x).to(torch.int32)
    table = None
    if not in_place:
        free = [p for p in range(b.pool) if p not in set(b.table.flatten().tolist())]
        table = torch.full((len(kv), -(-max(1, max(kept)) // page)), -3, dtype=torch.int32)
        at = 0
        for s, n in enumerate(kept):
            per = -(-n // page)
            table[s, :per] = torch.tensor(free[at:at + per], dtype=torch.int32)
            at += per
    all_ = [x for x in (*cache, *scale, held) if x is not None]
    bits = [x.view(torch.int16) if x.dtype in DT.values() else x for x in all_]
    want = [x.clone() for x in bits]
    for s, n in enumerate(kv):
        to = torch.arange(kept[s])
        to = ((b.table if in_place else table)[s].long()[to // page] * page + to % page).to(DEV)
        for h in range(hkv):
            frm = keep[s, h, :kept[s]].long()
            frm = (b.table[s].long()[frm // page] * page + frm % page).to(DEV)
            for x, y in zip(bits, want):
                y[h].flatten(0, 1)[to] = x[h].flatten(0, 1)[frm]
    dims, batch = P.make_dims(hkv, hkv, page, b.pool, P.PRR_BF16 if dt == "bf16" else P.PRR_F16), b.make(P)
    code = P.PRR_KV_E4M3 if kind == "e4m3" else P.PRR_KV_16
    nbytes = P.prr_compact_workspace_size(dims, batch, code, budget, in_place)
    assert (nbytes > 0) == in_place
    ws = torch.full((nbytes,), 0xff, dtype=torch.uint8, device=DEV) if nbytes else None
    table = None if table is None else table.to(DEV)
    P.prr_cache_compact(dims, batch, keep.to(DEV), torch.tensor(kept, dtype=torch.int32, device=DEV), budget, code, *cache,
                        *(scale or (None, None)), held, table, 0 if table is None else table.shape[-1], ws, nbytes)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(bits, want))


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("kind", ["16", "e4m3"])
@pytest.mark.parametrize("kv,budget", [([1], 1), ([5], 3), ([64], 63), ([100], 1), ([1000], 300), ([4097], 4000), ([0, 1, 16, 17, 500, 2049, 33], 100)])
def test_compact(kv, budget, kind, in_place):
    compact_case(kv, budget, kind=kind, in_place=in_place)
    compact_case(kv, budget, kind=kind, in_place=in_place, hkv=5, page=64, mass=False, dt="f16")
    if in_place and len(kv) == 1:
        compact_case(kv, budget, kind=kind, paged=False, hkv=1)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["16", "e4m3"])
def test_compact_budget_beyond_the_tokens(kind):
    compact_case([100, 7], 5000, kind=kind)
    compact_case([100, 7], 5000, kind=kind, in_place=False)


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [True, False])
def test_compact_any_order(in_place):
    compact_case([3000, 200], 1500, order="random", in_place=in_place)
    compact_case([3000, 200], 1500, order="random", in_place=in_place, kind="e4m3", page=256)


@pytest.mark.gpu
def test_compact_skips_what_is_out_of_range():
    import paper_2606_30389_amd as P
    table = torch.tensor([[0, -1, 2, 1]], dtype=torch.int32, device=DEV)
    dst = torch.tensor([[3, 2 ** 30, 4]], dtype=torch.int32, device=DEV)
    k = torch.arange(5 * 16 * S.D, device=DEV, dtype=torch.int32).to(torch.int16).view(1, 5, 16, S.D).view(torch.bfloat16)
    v = k.clone()
    keep = torch.tensor([[[5, -1, 17, 64, 63, 2 ** 31 - 1, *range(6, 40)]]], dtype=torch.int32, device=DEV)
    batch = P.make_batch(1, 1, 1, 64, None, torch.tensor([60], dtype=torch.int32, device=DEV), table, 4)
    was = k.view(torch.int16).clone()
    P.prr_cache_compact(P.make_dims(1, 1, 16, 5, P.PRR_BF16), batch, keep, torch.tensor([40], dtype=torch.int32, device=DEV), 40, 0, k, v,
                        None, None, None, dst, 3)
    torch.cuda.synchronize()
    got, rows = k.view(torch.int16).flatten(1, 2)[0], was.flatten(1, 2)[0].clone()
    for i, p in enumerate(keep[0, 0].tolist()):
        src, to = (table[0, p // 16].item() if 0 <= p < 60 else -1), dst[0, i // 16].item()
        if src >= 0 and to < 5:
            rows[to * 16 + i % 16] = was.flatten(1, 2)[0, src * 16 + p % 16]
    assert torch.equal(got, rows) and torch.equal(v.view(torch.int16), k.view(torch.int16))
    # more kept tokens than the sequence has are cut to it
    P.prr_cache_compact(P.make_dims(1, 1, 16, 5, P.PRR_BF16), batch, keep, torch.tensor([2 ** 31 - 1], dtype=torch.int32, device=DEV), 40, 0,
                        k, v, None, None, None, dst, 3)
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------- one after the other

def rand(*shape, seed=0, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["16", "e4m3"])
@pytest.mark.parametrize("to_other_pages", [False, True])
def test_a_session_that_evicts(kind, to_other_pages):
    """Tokens into a cache, attention with a shape, their weight, a smaller cache, and attention over it with the next token:
    as attention over the kept tokens' rows alone."""
    from paper_2606_30389_amd import runtime as R
    kv, budget, hq, hkv = [300, 77], 90, 8, 2
    cfg = R.PathConfig(num_q_heads=hq, num_kv_heads=hkv, page_size=16, num_tokens=640, k_select=1)
    cache, rope = R.PagedCache(cfg, DEV, kind=kind), R.Rope(DEV, rot_dim=64)
    table = torch.randperm(40, generator=torch.Generator().manual_seed(1))[:38].view(2, 19).to(torch.int32).to(DEV)
    b = R.Batch(DEV, kv, kv, table)
    n = sum(kv)
    q = cache.append(b, rand(n, hq, S.D), rand(n, hkv, S.D, seed=1), rand(n, hkv, S.D, seed=2), rope)
    # (the last tokens attend one by one, which an e4m3 cache's tokens do)
    ends = torch.tensor([kv[0] - 1, n - 1], device=DEV)
    one = R.Batch(DEV, [1, 1], kv, table)
    shape = R.Shape(cap=20.0, slopes=torch.tensor([0.01 * h for h in range(hq)], device=DEV), window=250)
    _, o, m, l = cache.attend(one, q[ends], shape=shape)
    mass = cache.weigh(one, q[ends], m, l, shape=shape)
    again = cache.weigh(one, q[ends], m, l, before=mass, decay=0.5, shape=shape)
    torch.cuda.synchronize()
    assert torch.allclose(again, 1.5 * mass, rtol=1e-6)
    keep, kept = cache.keep(one, mass, budget, sink=3, recent=20)
    rows = lambda x, s, h, p, t: x.view(torch.uint8)[h, t[s].long()[p // 16], p % 16]  # noqa: E731
    want = [[[rows(x, s, h, keep[s, h, :kept[s]].long(), table).clone() for x in (cache.k, cache.v)] for h in range(hkv)] for s in range(2)]
    weights = [[rows(mass.view(hkv, -1, 16, 1), s, h, keep[s, h, :kept[s]].long(), table).clone() for h in range(hkv)] for s in range(2)]
    dst = None
    if to_other_pages:
        # (pages of the first batch are taken: a pool of its own half)
        cache2 = R.PagedCache(R.PathConfig(num_q_heads=hq, num_kv_heads=hkv, page_size=16, num_tokens=1024, k_select=1), DEV, kind=kind)
        for name in ("k", "v", "k_scale", "v_scale"):
            if getattr(cache, name) is not None:
                getattr(cache2, name).view(torch.uint8)[:, :40] = getattr(cache, name).view(torch.uint8)
        big = torch.zeros(hkv, 64, 16, device=DEV)
        big[:, :40] = mass
        mass, cache = big, cache2
        dst = torch.arange(41, 41 + 2 * 7, dtype=torch.int32, device=DEV).view(2, 7)
    got = cache.evict(one, mass, budget, sink=3, recent=20, dst_table=dst)
    torch.cuda.synchronize()
    assert got.tolist() == kept.tolist() == [90, 77]
    small = table if dst is None else dst
    for s in range(2):
        for h in range(hkv):
            p = torch.arange(int(kept[s]), device=DEV)
            assert all(torch.equal(rows(x, s, h, p, small), y) for x, y in zip((cache.k, cache.v), want[s][h]))
            assert torch.equal(rows(mass.view(hkv, -1, 16, 1), s, h, p, small), weights[s][h])
    # the next token of each, rotated at its true position
    nxt = R.Batch(DEV, [1, 1], [91, 78], small)
    true = torch.tensor([300, 77], dtype=torch.int32, device=DEV)
    q1 = cache.append(nxt, rand(2, hq, S.D, seed=5), rand(2, hkv, S.D, seed=6), rand(2, hkv, S.D, seed=7), rope, positions=true)
    o32, o, m, l = cache.attend(nxt, q1)
    torch.cuda.synchronize()
    for s, c in enumerate((91, 78)):
        p = torch.arange(c, device=DEV)
        for h in range(hkv):
            vals = []
            for x, sc in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
                y = x.view(torch.uint8)[h, small[s].long()[p // 16], p % 16].view(x.dtype).double()
                vals.append(y if sc is None else y * torch.exp2(sc[h, small[s].long()[p // 16], p % 16].double() - 127)[:, None])
            o64, m64, l64, a, mag = S.attend64(q1[s, 4 * h:4 * h + 4].double(), *vals)
            S.check_state(o32[s, 4 * h:4 * h + 4].double(), m[s, 4 * h:4 * h + 4].double(), l[s, 4 * h:4 * h + 4].double(), o64, m64, l64, a,
                          mag, 2.0 ** -22, 2.0 ** -22, c, 0.0 if kind == "16" else 2.0 ** -25 * c * float(vals[1].abs().max()))


@pytest.mark.gpu
def test_a_layer_that_evicts_and_decodes():
    """prefill, evict, a token, selection and repair over the smaller cache: the selected pages' attention."""
    import numpy as np
    import oracle as O
    from paper_2606_30389_amd import runtime as R
    n, budget = 2000, 500
    cfg = R.PathConfig(num_q_heads=8, num_kv_heads=2, page_size=16, num_tokens=n, k_select=8)
    st = R.LayerState(cfg, DEV)
    stack = R.DecodeStack([st], [torch.zeros(8, S.D, dtype=torch.bfloat16, device=DEV)], DEV)
    rope = R.Rope(DEV)
    q_rot = torch.zeros(n, 8, S.D, dtype=torch.bfloat16, device=DEV)
    o, m, l = st.prefill(rand(n, 8, S.D), rand(n, 2, S.D, seed=1), rand(n, 2, S.D, seed=2), rope, q_out=q_rot)
    st.init_bits.fill_(-1)
    st.pred_count[0].fill_(3)
    kept = st.evict(q_rot, m, l, budget, sink=4, recent=64, last=32)
    assert kept == budget and not st.init_bits.any() and not st.pred_count[0].any()
    stack.set_tokens(kept + 1)
    q1 = st.append(rand(1, 8, S.D, seed=3), rand(1, 2, S.D, seed=4), rand(1, 2, S.D, seed=5), rope,
                   positions=torch.tensor([n], dtype=torch.int32, device=DEV))
    st.select(q1[0])
    st.repair(q1[0], serial=True)
    torch.cuda.synchronize()
    k64, v64 = (x[:, :32].double().cpu().numpy() for x in (st.k, st.v))
    _, sel, (o64, m64, l64) = O.serial_step(q1[0].double().cpu().numpy(), k64, v64, 16, kept + 1, 8)
    assert np.array_equal(np.sort(st.sel.cpu().numpy()[0, :int(st.sel_count[0])]), sel[0])
    assert np.abs(st.out_o32.cpu().numpy() - o64).max() < 1e-4
    # what the token gave to the selected pages, on top
    mass = torch.zeros(2, st.k.shape[1], 16, device=DEV)
    batch = R.Batch(DEV, [1], [kept + 1])
    st.cache().weigh(batch, q1, st.out_m[None], st.out_l[None], before=mass, pages=st.sel[None], counts=st.sel_count[None], out=mass)
    torch.cuda.synchronize()
    assert torch.allclose(mass.sum((1, 2)), torch.full((2,), 4.0, device=DEV), atol=1e-4)  # (4 heads of weight one)


@pytest.mark.gpu
@pytest.mark.parametrize("lists", [False, True])
def test_tokens_outside_a_call_keep_their_mass(lists):
    """A call for one sequence, or with lists, on top of the mass of a pool: the others' is in the result as it was."""
    from paper_2606_30389_amd import runtime as R
    cfg = R.PathConfig(num_q_heads=8, num_kv_heads=2, page_size=16, num_tokens=128, k_select=1)
    cache = R.PagedCache(cfg, DEV, k=rand(2, 8, 16, S.D), v=rand(2, 8, 16, S.D, seed=1))
    table = torch.tensor([[5, 2, 7, 0]], dtype=torch.int32, device=DEV)
    q, batch = rand(1, 8, S.D, seed=2), R.Batch(DEV, [1], [50], table)
    given = dict(pages=torch.tensor([[[1, 0], [3, 2]]], dtype=torch.int32, device=DEV),
                 counts=torch.tensor([[1, 2]], dtype=torch.int32, device=DEV)) if lists else {}
    _, _, m, l = cache.attend(batch, q, **given)
    before = torch.rand(2, 8, 16, device=DEV)
    was = before.clone()
    got = cache.weigh(batch, q, m, l, before=before, decay=0.5, **given)
    torch.cuda.synchronize()
    written = torch.zeros(2, 8, 16, dtype=torch.bool)
    for h, logical in enumerate([[1], [3, 2]] if lists else [range(4)] * 2):
        for lp in logical:
            written[h, int(table[0, lp]), :min(16, 50 - 16 * lp)] = True
    got, was = got.cpu(), was.cpu()
    assert torch.equal(before.cpu(), was) and torch.equal(got[~written], was[~written])
    assert abs(float((got[written] - 0.5 * was[written]).sum()) - 8.0) < 1e-3  # (8 heads of weight one)


@pytest.mark.gpu
def test_eviction_on_other_streams_and_in_graphs():
    """weigh, keep and compact on a stream of their own, and captured: the results of the eager calls."""
    from paper_2606_30389_amd import runtime as R
    n, budget = 40000, 3000
    cfg = R.PathConfig(num_q_heads=8, num_kv_heads=2, page_size=16, num_tokens=n, k_select=1)
    src = [rand(2, 2500, 16, S.D, seed=i) for i in (1, 2)]
    q, batch = rand(40, 8, S.D, seed=3), R.Batch(DEV, [40], [n])

    def run(cache, stream=None):
        _, m, l = cache.prompt(batch, q, stream=stream)
        mass = cache.weigh(batch, q, m, l, last=16, stream=stream)
        kept = cache.evict(batch, mass, budget, sink=4, recent=100, stream=stream)
        return mass, kept

    def fresh():
        return R.PagedCache(cfg, DEV, k=src[0].clone(), v=src[1].clone())

    ref = fresh()
    want = run(ref)
    torch.cuda.synchronize()
    cache, stream = fresh(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = run(cache, stream)
    junk = [torch.full((2, 2500, 16), 3.0, device=DEV) for _ in range(8)]
    torch.cuda.synchronize()
    assert torch.equal(cache.k, ref.k) and torch.equal(cache.v, ref.v) and all(torch.equal(x, y) for x, y in zip(got, want))
    del junk
    cache = fresh()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(cache)
    for _ in range(4):
        cache.k.copy_(src[0])
        cache.v.copy_(src[1])
        other = run(fresh())  # eager work between the replays
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(cache.k, ref.k) and torch.equal(cache.v, ref.v) and all(torch.equal(x, y) for x, y in zip(got, want))
        assert all(torch.equal(x, y) for x, y in zip(other, want))
