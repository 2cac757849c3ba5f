"""prr_prompt_attn_shaped and prr_decode_attn_shaped against 64 bits: caps, slopes, windows, documents, prefixes and
all of them together; rows that see nothing; infinities and NaN in hidden places; splits, graphs, page tables."""
import math

import pytest
import torch

from tests import context_support as S
from tests.shape_support import Shape, slopes_of

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f16": torch.float16}


def starts(new, kv, size):
    """Where each new token's document begins, documents of `size` tokens."""
    return [max(0, k - n + i) // size * size for n, k in zip(new, kv) for i in range(n)]


def prompt_case(new, kv, hq, hkv, shape, dt="bf16", page=16, pad=0, paged=True, spread=1.5, edit=None, hide=None, single=False):
    import paper_2606_30389_amd as P
    b = S.Batch(new, kv, page, pad=pad, paged=paged, device=DEV, seed=9, single=single)
    G = hq // hkv
    g = torch.Generator(device=DEV).manual_seed(S.seed_of(new, kv, hq, hkv, dt, page))
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    q = (spread * rand(b.total, hq, S.D)).to(DT[dt])
    cache = [rand(hkv, b.pool, page, S.D).to(DT[dt]) for _ in range(2)]
    if edit:
        edit(b, q, cache)
    if shape.first is not None:
        shape.first = list(shape.first) + [10 ** 9] * pad
    # what no row sees must not matter: NaN, and no page in the table where a whole page is hidden
    seen = torch.zeros(b.pool * page, dtype=torch.bool)
    for s, rows, pos in b.sequences():
        if len(rows):
            vis = shape.visible(s, rows, pos, kv[s]).any(0)
            seen[b.slots(s, 0, kv[s])[vis]] = True
            if hide is not None:
                for p in range(-(-kv[s] // page)):
                    if not vis[p * page:(p + 1) * page].any():
                        b.d_table[s, p] = hide
    for c in cache:
        c.flatten(1, 2)[:, ~seen.to(DEV)] = math.nan
    out = torch.full((b.total, hq, S.D), 5.0, dtype=DT[dt], device=DEV)
    m, l = (torch.full((b.total, hq), 5.0, device=DEV) for _ in range(2))
    dims = P.make_dims(hq, hkv, page, b.pool, P.PRR_BF16 if dt == "bf16" else P.PRR_F16)
    batch, sh = b.make(P), shape.make(P, DEV)
    nbytes = P.prr_prompt_shaped_workspace_size(dims, batch, sh)
    ws = torch.full((max(nbytes, 256),), 0xff, dtype=torch.uint8, device=DEV) if nbytes else None
    P.prr_prompt_attn_shaped(dims, batch, sh, q, *cache, out, m, l, ws, nbytes)
    torch.cuda.synchronize()
    eps = S.half_step(DT[dt])
    floor = 2.0 ** -24 if dt == "f16" else 0.0
    for s, rows, pos in b.sequences():
        if not len(rows):
            continue
        slot = b.slots(s, 0, kv[s]).to(DEV)
        visible = shape.visible(s, rows, pos, kv[s])
        # (a row's error bound is that of the scores that it sees)
        any_seen = visible.any(0)
        k0, k1 = (int(any_seen.nonzero().min()), int(any_seen.nonzero().max()) + 1) if any_seen.any() else (0, 0)
        visible = visible[:, k0:k1].to(DEV).repeat_interleave(G, 0)
        rows, pos = rows.to(DEV), pos.to(DEV).repeat_interleave(G, 0)
        for h in range(hkv):
            k, v = (c[h].flatten(0, 1)[slot[k0:k1]].double() for c in cache)
            k, v = k.nan_to_num(0.0), v.nan_to_num(0.0)
            qq = q[rows, h * G:(h + 1) * G].double().reshape(-1, S.D)
            head = (h * G + torch.arange(G, device=DEV)).repeat(len(rows))
            o64, m64, l64, a, mag = shape.attend(qq, k, v, pos - k0, head, visible)
            vmax = v.abs().max() if k1 > k0 else 0.0
            got = [x[rows, h * G:(h + 1) * G].double().reshape(-1, *x.shape[2:]) for x in (out, m, l)]
            S.check_state(*got, o64, m64, l64, a, mag, eps, eps, k1 - k0, floor * (1 + (k1 - k0) * vmax), what=(s, h))
    for x in (out, m, l):
        assert torch.all(x[b.cu[-1]:] == 5.0)
    return P, dims, batch, sh, q, cache, out, m, l, ws, nbytes


def shapes(new, kv, hq):
    """Every part of a shape alone, and all of them."""
    long = max(kv)
    prefix = [(7 * k) // 9 for k in kv]
    return {
        "cap": Shape(cap=3.0), "slopes": Shape(slopes=slopes_of(hq)), "window": Shape(window=max(1, long // 3)),
        "docs": Shape(first=starts(new, kv, max(1, long // 4))), "prefix": Shape(prefix=prefix),
        "all": Shape(cap=5.0, slopes=slopes_of(hq), window=max(1, 2 * long // 3), first=starts(new, kv, max(1, long // 2)), prefix=prefix),
    }


KINDS = ["cap", "slopes", "window", "docs", "prefix", "all"]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 2, 16, 63, 65, 130, 257, 700])
def test_prompt_lengths(n, kind):
    prompt_case([n], [n], 16, 1, shapes([n], [n], 16)[kind])
    prompt_case([n], [n + 37], 4, 4, shapes([n], [n + 37], 4)[kind], dt="f16", paged=False)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hkv,page,dt", [(1, 1, 16, "bf16"), (28, 4, 64, "f16"), (8, 8, 256, "bf16"), (36, 3, 16, "f16"), (10, 2, 128, "bf16")])
def test_prompt_heads_and_pages(hq, hkv, page, dt, kind):
    new, kv = [300, 0, 1, 45], [300, 7, 500, 111]
    prompt_case(new, kv, hq, hkv, shapes(new, kv, hq)[kind], dt, page, pad=3)


@pytest.mark.gpu
@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 200])
@pytest.mark.parametrize("hq,hkv", [(16, 1), (2, 2)])
def test_prompt_windows(window, hq, hkv):
    """Long (eight waves), short, and pages that no window reaches gone from the table."""
    prompt_case([1500], [1500], hq, hkv, Shape(window=window))
    prompt_case([130], [900], hq, hkv, Shape(window=window, cap=2.0), dt="f16", hide=-1)
    prompt_case([40, 300], [2000, 300], hq, hkv, Shape(window=window), hide=2 ** 30)


@pytest.mark.gpu
def test_prompt_many_sequences():
    new = [(37 * i) % 23 for i in range(150)]
    kv = [n + (53 * i) % 91 * (i % 3 > 0) for i, n in enumerate(new)]
    sh = Shape(cap=4.0, slopes=slopes_of(8), window=40, first=[(7 * i) % 50 for i in range(sum(new))], prefix=[(11 * i) % 60 for i in range(150)])
    prompt_case(new, kv, 8, 2, sh, pad=2)


@pytest.mark.gpu
@pytest.mark.parametrize("new,kv", [([3], [5000]), ([1, 2], [3000, 4097]), ([130], [2000])])
@pytest.mark.parametrize("kind", KINDS)
def test_prompt_few_rows_many_keys(new, kv, kind):
    """Few rows: the keys are split over workgroups and joined, parts of them hidden."""
    prompt_case(new, kv, 16, 1, shapes(new, kv, 16)[kind], pad=1)


@pytest.mark.gpu
@pytest.mark.parametrize("paged", [False, True])
def test_prompt_split_window(paged):
    """Few rows with a window of many tiles at the end of a long cache: parts of the window."""
    P, dims, batch, sh, *_ = prompt_case([5], [9000], 16, 1, Shape(window=4001), paged=paged, hide=-1 if paged else None)
    assert P.prr_prompt_shaped_workspace_size(dims, batch, sh) > 0
    # the window bounds the parts, unless a prefix may reach beyond it
    assert P.prr_prompt_shaped_workspace_size(dims, batch, sh) < P.prr_prompt_workspace_size(dims, batch)


@pytest.mark.gpu
@pytest.mark.parametrize("n,past", [(40, 0), (300, 0), (300, 1200)])
def test_prompt_rows_that_see_nothing(n, past):
    """`first` behind the token itself, and device values that are no positions at all."""
    first = [[past + i + 1, 0, -5, 2 ** 31 - 1, past + i, -2 ** 31][i % 6] for i in range(n)]
    prompt_case([n], [past + n], 8, 2, Shape(first=first))
    prompt_case([n], [past + n], 8, 2, Shape(first=first, prefix=[2 ** 31 - 1], cap=2.0), dt="f16")
    prompt_case([n], [past + n], 8, 2, Shape(prefix=[-2 ** 31], window=2 ** 30))
    # nothing for anyone
    prompt_case([n], [past + n], 8, 2, Shape(first=[past + n] * n))


@pytest.mark.gpu
def test_prompt_tokens_without_a_place():
    prompt_case([10, 70, 4], [3, 0, 4], 8, 2, Shape(prefix=[2, 5, 4], window=3), pad=2)
    prompt_case([300], [130], 16, 1, Shape(prefix=[130], slopes=slopes_of(16)), dt="f16")


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("cap,spread", [(50.0, 4.0), (2.0 ** -10, 1.5), (0.5, 0.01), (30.0, 40.0), (2.0 ** 20, 1.5), (1.0, 12.0)])
def test_prompt_caps(cap, spread, dt):
    """Logits far below the cap, around half of it (where the form changes), and far above."""
    prompt_case([200], [260], 8, 2, Shape(cap=cap), dt, spread=spread)


@pytest.mark.gpu
@pytest.mark.parametrize("slopes", [[0.0] * 8, [1.0, -1.0, 0.5, -0.01, 3.0, 0.0, 100.0, 1e-4]])
def test_prompt_slopes_of_any_sign(slopes):
    prompt_case([200], [460], 8, 2, Shape(slopes=slopes))
    prompt_case([200], [460], 8, 2, Shape(slopes=slopes, prefix=[400], window=250), dt="f16")


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_prompt_non_finite_tokens_reach_only_who_sees_them(dt):
    """An infinity or NaN in a token's key or value changes nothing for the tokens whose window or document leaves it out."""
    import paper_2606_30389_amd as P
    n, past, window = 400, 100, 90
    b = S.Batch([n], [past + n], 16, device=DEV, seed=2)
    g = torch.Generator(device=DEV).manual_seed(n)
    q = torch.randn(n, 4, S.D, generator=g, device=DEV).to(DT[dt])
    cache = [torch.randn(2, b.pool, 16, S.D, generator=g, device=DEV).to(DT[dt]) for _ in range(2)]
    dims = P.make_dims(4, 2, 16, b.pool, P.PRR_BF16 if dt == "bf16" else P.PRR_F16)
    batch = b.make(P)
    for shape in (Shape(window=window), Shape(first=starts([n], [past + n], 130)), Shape(prefix=[250], window=120, cap=9.0)):
        sh = shape.make(P, DEV)
        nbytes = P.prr_prompt_shaped_workspace_size(dims, batch, sh)
        ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=DEV)
        visible = shape.visible(0, torch.arange(n), past + torch.arange(n), past + n).to(DEV)

        def run(c):
            out = torch.zeros(n, 4, S.D, dtype=DT[dt], device=DEV)
            P.prr_prompt_attn_shaped(dims, batch, sh, q, *c, out, None, None, ws, nbytes)
            torch.cuda.synchronize()
            return out

        clean = run(cache)
        for at in (0, past + 3, 230, past + n // 2, past + n - 1):
            for i, x in ((0, math.inf), (0, math.nan), (1, math.inf), (1, -math.inf), (1, math.nan)):
                dirty = [c.clone() for c in cache]
                dirty[i].flatten(1, 2)[:, b.slots(0, at, at + 1).to(DEV), 5] = x
                got = run(dirty)
                sees = visible[:, at]
                assert torch.equal(got[~sees], clean[~sees])
                if i == 1 and sees.any():
                    want = got[sees][:, :, 5].float()
                    assert torch.all(want.isnan()) if math.isnan(x) else torch.all(want.isnan() | (want == x))
                    keep = [c for c in range(S.D) if c != 5]
                    assert torch.equal(got[sees][..., keep], clean[sees][..., keep])


@pytest.mark.gpu
def test_infinite_logits_are_capped():
    """A key whose logit is infinite counts as one at the cap."""
    import paper_2606_30389_amd as P
    n = 70
    b = S.Batch([n], [n], 16, device=DEV, seed=1)
    q = torch.ones(n, 2, S.D, device=DEV, dtype=torch.bfloat16)
    cache = [torch.randn(1, b.pool, 16, S.D, device=DEV).to(torch.bfloat16) for _ in range(2)]
    dims, batch, sh = P.make_dims(2, 1, 16, b.pool, P.PRR_BF16), b.make(P), Shape(cap=4.0).make(P, DEV)
    outs = []
    for x in (math.inf, 1e30):
        k = cache[0].clone()
        k.flatten(1, 2)[:, b.slots(0, 10, 11).to(DEV), 3] = x
        k.flatten(1, 2)[:, b.slots(0, 20, 21).to(DEV), 3] = -x
        out, m, l = torch.zeros_like(q), torch.zeros(n, 2, device=DEV), torch.zeros(n, 2, device=DEV)
        P.prr_prompt_attn_shaped(dims, batch, sh, q, k, cache[1], out, m, l, None, 0)
        o32 = torch.zeros(1, 2, S.D, device=DEV)
        tok = P.make_batch(1, 1, 1, n, None, b.d_kv, b.d_table, b.width)
        nbytes = P.prr_decode_shaped_workspace_size(dims, tok, sh, 0)
        ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=DEV)
        P.prr_decode_attn_shaped(dims, tok, sh, q[:1], 0, k, cache[1], None, None, None, None, 0, o32, None,
                                 torch.zeros(1, 2, device=DEV), torch.zeros(1, 2, device=DEV), ws, nbytes)
        torch.cuda.synchronize()
        assert out.isfinite().all() and l.isfinite().all() and o32.isfinite().all()
        # (the cap in the units of q.k, 1 / sqrt(128) and their product are rounded: 3 * 2^-24 of it)
        assert torch.all((m[10:] - 4.0).abs() <= 4.0 * 2.0 ** -22)
        outs.append((out, m, l, o32))
    assert all(torch.equal(x, y) for x, y in zip(*outs))


@pytest.mark.gpu
def test_no_shape_is_the_plain_call():
    """NULL and a shape with nothing set give the plain call's bits; so does a shape that hides nothing."""
    import paper_2606_30389_amd as P
    b = S.Batch([300, 20], [500, 20], 16, device=DEV, seed=1)
    g = torch.Generator(device=DEV).manual_seed(3)
    q = torch.randn(b.total, 8, S.D, generator=g, device=DEV).to(torch.bfloat16)
    cache = [torch.randn(2, b.pool, 16, S.D, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2)]
    dims, batch = P.make_dims(8, 2, 16, b.pool, P.PRR_BF16), b.make(P)

    def run(call):
        out, m, l = torch.zeros_like(q), torch.zeros(b.total, 8, device=DEV), torch.zeros(b.total, 8, device=DEV)
        nbytes = P.prr_prompt_workspace_size(dims, batch)
        call(out, m, l, torch.empty(max(nbytes, 256), dtype=torch.uint8, device=DEV), nbytes)
        torch.cuda.synchronize()
        return out, m, l

    want = run(lambda *o: P.prr_prompt_attn(dims, batch, q, *cache, *o))
    for sh in (None, P.make_shape(), Shape(window=2 ** 30).make(P, DEV), Shape(prefix=[0, 0]).make(P, DEV)):
        got = run(lambda *o: P.prr_prompt_attn_shaped(dims, batch, sh, q, *cache, *o))
        assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.gpu
def test_prompt_replayed_in_a_graph():
    """One capture, replayed with other lengths, documents, prefixes and slopes in the same buffers."""
    new, kv = [60, 20], [900, 700]
    shape = Shape(cap=6.0, slopes=slopes_of(8), window=650, first=starts(new, kv, 300), prefix=[100, 695])
    P, dims, batch, sh, q, cache, out, m, l, ws, nbytes = prompt_case(new, kv, 8, 2, shape)
    for c in cache:
        c.nan_to_num_(0.5)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        P.prr_prompt_attn_shaped(dims, batch, sh, q, *cache, out, m, l, ws, nbytes)
    slopes, first, prefix = sh.tensors
    for i in range(4):
        torch.manual_seed(i)
        q.copy_(torch.randn_like(q))
        batch.tensors[1].copy_(torch.tensor([900 - 13 * i, 700 - 40 * i], dtype=torch.int32))
        batch.tensors[0].copy_(torch.tensor([0, 60 - i, 80 - 2 * i], dtype=torch.int32))
        first.add_(7 * i)
        prefix.sub_(30)
        slopes.mul_(0.7)
        want = [torch.full_like(x, 2.0) for x in (out, m, l)]
        P.prr_prompt_attn_shaped(dims, batch, sh, q, *cache, *want, ws, nbytes)
        for x in (out, m, l):
            x.fill_(2.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((out, m, l), want))


# ------------------------------------------------------------------------------- single tokens

def decode_case(kv, hq, hkv, shape, dt="bf16", page=16, kind="16", paged=True, lists=None, spread=1.5, pad=0, hide=None):
    import paper_2606_30389_amd as P
    b = S.Batch([1] * len(kv), kv, page, pad=pad, paged=paged, device=DEV, seed=4, single=True)
    G = hq // hkv
    g = torch.Generator(device=DEV).manual_seed(S.seed_of(kv, hq, hkv, dt, page, kind))
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    q = (spread * rand(b.total, hq, S.D)).to(DT[dt])
    sizes = (hkv, b.pool, page, S.D)
    seen = torch.zeros(b.pool * page, dtype=torch.bool)
    vis = []
    for s, n in enumerate(kv):
        vis.append(shape.visible(s, torch.tensor([s]), torch.tensor([n - 1]), n)[0] if n else torch.zeros(0, dtype=torch.bool))
        seen[b.slots(s, 0, n)[vis[s]]] = True
        if hide is not None:
            for p in range(-(-n // page)):
                if not vis[s][p * page:(p + 1) * page].any():
                    b.d_table[s, p] = hide
    unseen = ~seen.to(DEV)
    if kind == "e4m3":
        cache = [(40 * rand(*sizes)).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for _ in range(2)]
        scale = [torch.randint(120, 124, sizes[:3], generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
        for c, x in zip(cache, scale):
            c.flatten(1, 2)[:, unseen] = 0x7f  # NaN
            x.flatten(1, 2)[:, unseen] = 255
    else:
        cache, scale = [rand(*sizes).to(DT[dt]) for _ in range(2)], [None, None]
        for c in cache:
            c.flatten(1, 2)[:, unseen] = math.nan
    dims = P.make_dims(hq, hkv, page, b.pool, P.PRR_BF16 if dt == "bf16" else P.PRR_F16)
    pages = count = None
    if lists is not None:
        pages = torch.full((len(kv), hkv, max(1, max(len(x) for x in lists))), -3, dtype=torch.int32)
        for s, x in enumerate(lists):
            pages[s, :, :len(x)] = torch.tensor(x, dtype=torch.int32)
        pages, count = pages.to(DEV), torch.tensor([[len(x)] * hkv for x in lists], dtype=torch.int32, device=DEV)
    batch, sh = b.make(P), shape.make(P, DEV)
    code, cap = P.PRR_KV_E4M3 if kind == "e4m3" else P.PRR_KV_16, 0 if pages is None else pages.shape[-1]
    nbytes = P.prr_decode_shaped_workspace_size(dims, batch, sh, code, cap)
    ws = torch.full((max(nbytes, 256),), 0xff, dtype=torch.uint8, device=DEV)
    out = [torch.full((b.total, hq, S.D), 5.0, device=DEV), torch.full((b.total, hq, S.D), 5.0, dtype=DT[dt], device=DEV),
           torch.full((b.total, hq), 5.0, device=DEV), torch.full((b.total, hq), 5.0, device=DEV)]
    call = lambda o: P.prr_decode_attn_shaped(dims, batch, sh, q, code, *cache, *scale, pages, count, cap, *o, ws, nbytes)  # noqa: E731
    call(out)
    torch.cuda.synchronize()
    eps = S.half_step(DT[dt])
    two = torch.float16 if kind == "e4m3" else DT[dt]
    werr, floor = (S.half_step(two) ** 2, 2.0 ** -25) if two == torch.float16 else (S.half_step(two) ** 3, 0.0)
    for s, n in enumerate(kv):
        pos = torch.arange(n)[vis[s]]
        if lists is not None:
            pos = pos[torch.isin(pos // page, torch.tensor(lists[s], dtype=torch.long))]
        slot = (b.table[s].long()[pos // page] * page + pos % page).to(DEV)
        for h in range(hkv):
            def rows(i):
                x = cache[i][h].flatten(0, 1)[slot]
                if kind == "e4m3":
                    return x.view(torch.float8_e4m3fn).double() * torch.exp2(scale[i][h].flatten()[slot].double() - 127)[:, None]
                return x.double()
            heads = slice(h * G, (h + 1) * G)
            k, v = rows(0), rows(1)
            # (positions are given as distances from the token, whose own is n - 1)
            keys = pos.to(DEV)
            sub = Shape(cap=shape.cap)
            z, mag = sub.scores(q[s, heads].double(), k, None, None)
            if shape.slopes is not None and len(pos):
                bias = torch.tensor(shape.slopes[h * G:(h + 1) * G], dtype=torch.float32).double().to(DEV)[:, None] * (n - 1 - keys)
                z, mag = z - bias, mag + bias.abs().amax(-1)
            if len(pos):
                m64 = z.amax(-1)
                p = torch.exp(z - m64[:, None])
                l64 = p.sum(-1)
                w = p / l64[:, None]
                o64, a = w @ v, w @ v.abs()
            else:
                o64 = a = torch.zeros(G, S.D, dtype=torch.float64, device=DEV)
                m64, l64 = o64[:, 0] - math.inf, o64[:, 0]
                mag = l64
            m, l = out[2][s, heads].double(), out[3][s, heads].double()
            fl = floor * len(pos) * float(v.abs().max()) if len(pos) else 0.0
            S.check_state(out[0][s, heads].double(), m, l, o64, m64, l64, a, mag, werr, 2.0 ** -22, len(pos), fl, (s, h))
            S.check_state(out[1][s, heads].double(), m, l, o64, m64, l64, a, mag, werr + eps, eps, len(pos),
                          fl + (2.0 ** -25 if dt == "f16" else 0.0), (s, h))
    for x in out:
        assert torch.all(x[len(kv):] == 5.0)
    return call, out, batch, sh


def decode_shapes(kv, hq):
    return {"cap": Shape(cap=2.0), "slopes": Shape(slopes=slopes_of(hq)), "window": Shape(window=max(1, max(kv) // 3)),
            "docs": Shape(first=[k // 3 for k in kv]), "prefix": Shape(prefix=[k // 2 for k in kv]),
            "all": Shape(cap=5.0, slopes=slopes_of(hq), window=max(1, max(kv) // 2), first=[k // 3 for k in kv], prefix=[3] * len(kv))}


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["16", "e4m3"])
@pytest.mark.parametrize("which", KINDS)
@pytest.mark.parametrize("kv", [0, 1, 15, 17, 128, 1000, 20011])
def test_decode_lengths(kv, which, kind):
    decode_case([kv], 16, 1, decode_shapes([kv], 16)[which], kind=kind)
    decode_case([kv], 4, 4, decode_shapes([kv], 4)[which], dt="f16", kind=kind, paged=False)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["16", "e4m3"])
@pytest.mark.parametrize("which", KINDS)
def test_decode_ragged(which, kind):
    kv = [1, 0, 700, 16, 5000, 33, 1200]
    for hq, hkv, page, dt in ((28, 4, 64, "bf16"), (8, 8, 16, "f16"), (10, 2, 256, "bf16")):
        decode_case(kv, hq, hkv, decode_shapes(kv, hq)[which], dt, page, kind, pad=2, hide=-1)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["16", "e4m3"])
@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 100, 4096])
def test_decode_windows(window, kind):
    decode_case([1, 16, 17, 100, 4100, 9000], 8, 2, Shape(window=window), kind=kind, hide=2 ** 30)
    decode_case([9000], 8, 2, Shape(window=window, cap=1.0, slopes=slopes_of(8)), dt="f16", kind=kind, paged=False)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["16", "e4m3"])
def test_decode_lists(kind):
    """Listed pages, some of them partly or wholly before the window, in any order, entries out of range skipped."""
    lists = [[5, 0, 61, 30, 31], [2], [], [0, 1, 2, 3]]
    kv = [1000, 40, 500, 60]
    for sh in (Shape(window=510), Shape(first=[490, 37, 0, 60], cap=2.0), Shape(slopes=slopes_of(8))):
        decode_case(kv, 8, 2, sh, lists=lists, kind=kind)
    decode_case([1000], 8, 2, Shape(first=[1000]), lists=[[62, 61]], kind=kind)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["16", "e4m3"])
@pytest.mark.parametrize("cap,spread", [(50.0, 4.0), (2.0 ** -10, 1.5), (0.5, 0.01), (1.0, 12.0)])
def test_decode_caps(cap, spread, kind):
    decode_case([777], 8, 2, Shape(cap=cap), kind=kind, spread=spread)
    decode_case([777], 8, 2, Shape(cap=cap, window=300), dt="f16", kind=kind, spread=spread)


@pytest.mark.gpu
def test_decode_infinite_values():
    """An infinite value of a visible key gives infinity, one of a hidden key nothing."""
    import paper_2606_30389_amd as P
    n, window = 3000, 1000
    for dt in DT.values():
        cache = [torch.randn(1, 188, 16, S.D, device=DEV).to(dt) for _ in range(2)]
        dims = P.make_dims(4, 1, 16, 188, P.PRR_BF16 if dt == torch.bfloat16 else P.PRR_F16)
        batch, sh = P.make_batch(1, 1, 1, n, None, torch.tensor([n], dtype=torch.int32, device=DEV)), Shape(window=window).make(P, DEV)
        q = torch.randn(1, 4, S.D, device=DEV).to(dt)
        nbytes = P.prr_decode_shaped_workspace_size(dims, batch, sh, 0)
        ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=DEV)
        got = []
        for at in (None, n - window - 1, n - window, n - 1):
            v = cache[1].clone()
            if at is not None:
                v.flatten(1, 2)[0, at, 7] = -math.inf
            out = torch.zeros(1, 4, S.D, device=DEV)
            P.prr_decode_attn_shaped(dims, batch, sh, q, 0, cache[0], v, None, None, None, None, 0, out, None,
                                     torch.zeros(1, 4, device=DEV), torch.zeros(1, 4, device=DEV), ws, nbytes)
            torch.cuda.synchronize()
            got.append(out)
        keep = [c for c in range(S.D) if c != 7]
        assert torch.equal(got[0], got[1])
        for x in got[2:]:
            assert torch.all(x[..., 7] == -math.inf) and torch.equal(x[..., keep], got[0][..., keep])


@pytest.mark.gpu
def test_decode_replayed_in_a_graph():
    kv = [3000, 50, 999]
    call, out, batch, sh = decode_case(kv, 8, 2, Shape(cap=3.0, slopes=slopes_of(8), window=700, first=[10, 20, 500]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        call(out)
    for i in range(4):
        batch.tensors[1].copy_(torch.tensor([3000 - 5 * i, 50 - 3 * i, 999 - 7 * i], dtype=torch.int32))
        sh.tensors[1].copy_(torch.tensor([2500 - i, 30, 990 + 20 * i], dtype=torch.int32))
        want = [torch.full_like(x, 2.0) for x in out]
        call(want)
        for x in out:
            x.fill_(2.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        # (NaN: keys that the first call hid are NaN)
        assert all(torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0)) for x, y in zip(out, want))
