"""Mass that goes on after an eviction, and in a buffer of one's own."""
import pytest
import torch

from tests import context_support as S
from tests.shape_support import keep_of

DEV = "cuda:0"


def rand(*shape, seed=0, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["16", "e4m3"])
@pytest.mark.parametrize("to_other_pages", [False, True])
@pytest.mark.parametrize("apart", [False, True])
def test_tokens_after_an_eviction_begin_without_mass(kind, to_other_pages, apart):
    """Evict, append token by token with their mass added up, evict again: mass and choice as the weights in 64 bits give them.
    apart: keep and compact by themselves."""
    from paper_2606_30389_amd import runtime as R
    kv, budget, hq, hkv, G = [300, 77, 64, 5], 90, 8, 2, 4
    n = len(kv)
    cfg = R.PathConfig(num_q_heads=hq, num_kv_heads=hkv, page_size=16, num_tokens=16 * 120, k_select=1)
    cache = R.PagedCache(cfg, DEV, kind=kind)
    ids = torch.randperm(120, generator=torch.Generator().manual_seed(1)).to(torch.int32)
    table = ids[:76].view(n, 19).contiguous().to(DEV)
    dst = ids[76:76 + 4 * 9].view(n, 9).contiguous().to(DEV) if to_other_pages else None
    rope = R.Rope(DEV, rot_dim=64)
    b = R.Batch(DEV, kv, kv, table)
    cache.append(b, None, rand(sum(kv), hkv, S.D, seed=1), rand(sum(kv), hkv, S.D, seed=2), rope)
    # what the tokens received so far; pages that hold none of them have what other sequences left there, but those that the
    # sequences will grow into, which their owner clears
    one = R.Batch(DEV, [1] * n, kv, table)
    mass = 3.0 + torch.rand(hkv, 120, 16, device=DEV, generator=torch.Generator(device=DEV).manual_seed(3))
    small = table if dst is None else dst
    left = [min(budget, x) for x in kv]
    for s in range(n):
        mass[:, small[s].long()[-(-(kv[s] if dst is None else left[s]) // 16):]] = 0.0
    gave = mass.clone()
    held = [[gave[h].double().flatten()[(table[s].long()[torch.arange(x, device=DEV) // 16] * 16 + torch.arange(x, device=DEV) % 16)]
             for h in range(hkv)] for s, x in enumerate(kv)]

    def evict(batch, lengths, dst):
        keep, kept = cache.keep(batch, mass, budget, sink=2, recent=10)
        if apart:
            cache.compact(batch, keep, kept, mass, dst)
        else:
            kept = cache.evict(batch, mass, budget, sink=2, recent=10, dst_table=dst)
        torch.cuda.synchronize()
        assert kept.tolist() == [min(budget, x) for x in lengths]
        for s in range(n):
            for h in range(hkv):
                want = keep_of(held[s][h].tolist(), budget, 2, 10)
                assert keep[s, h, :len(want)].tolist() == want
                held[s][h] = held[s][h][torch.tensor(want, device=DEV)]

    evict(one, kv, dst)
    steps, lens = 50, left
    nxt = R.Batch(DEV, [1] * n, [x + 1 for x in lens], small, max_kv=max(lens) + steps)
    for i in range(steps):
        if i:
            nxt.advance()
        lens = [x + 1 for x in lens]
        true = torch.tensor([x + i for x in kv], dtype=torch.int32, device=DEV)
        q = cache.append(nxt, rand(n, hq, S.D, seed=10 + i), rand(n, hkv, S.D, seed=100 + i), rand(n, hkv, S.D, seed=200 + i), rope,
                         positions=true)
        _, _, m, l = cache.attend(nxt, q)
        cache.weigh(nxt, q, m, l, before=mass, out=mass)
        torch.cuda.synchronize()
        for s in range(n):
            p = torch.arange(lens[s], device=DEV)
            page, off = small[s].long()[p // 16], p % 16
            for h in range(hkv):
                k = cache.k.view(torch.uint8)[h, page, off].view(cache.k.dtype).double()
                if kind == "e4m3":
                    k = k * torch.exp2(cache.k_scale[h, page, off].double() - 127)[:, None]
                heads = slice(h * G, (h + 1) * G)
                z = (q[s, heads].double() @ k.T.contiguous()) * S.SCALE
                w = torch.softmax(z, -1).sum(0)
                held[s][h] = torch.cat([held[s][h], held[s][h].new_zeros(1)]) + w
                # a weight is off by its score's, the maximum's and twice the sum's error, mag * 2^-16 each (mag < 14 here), and
                # 2^-15 for its exponent; a sum of 50 by 50 * 2^-24 more
                e = (mass[h, page, off].double() - held[s][h]).abs()
                assert torch.all(e <= held[s][h] * 2.0 ** -10), (s, h, i, e.max())
    evict(nxt, lens, None)


@pytest.mark.gpu
def test_mass_of_vacated_places_is_cleared():
    """What compact writes of the mass: the kept tokens', and 0 where no token is any more; the other pages' as it was."""
    from paper_2606_30389_amd import runtime as R
    cfg = R.PathConfig(num_q_heads=2, num_kv_heads=2, page_size=16, num_tokens=16 * 40, k_select=1)
    for kv in ([100, 33, 0, 16, 48], [128] * 5):
        for budget in (1, 20, 48, 200):
            for to_other_pages in (False, True):
                cache = R.PagedCache(cfg, DEV, k=rand(2, 40, 16, S.D), v=rand(2, 40, 16, S.D, seed=1))
                if to_other_pages and sum(kv) > 300:
                    continue  # (no pages left)
                ids, at, dst = torch.randperm(40, generator=torch.Generator().manual_seed(budget)).to(torch.int32), 0, None
                table = torch.full((5, 8), -1, dtype=torch.int32)
                for s, x in enumerate(kv):
                    per = -(-x // 16)
                    table[s, :per] = ids[at:at + per]
                    at += per
                if to_other_pages:
                    dst = torch.full((5, 8), 10 ** 6, dtype=torch.int32)
                    for s, x in enumerate(kv):
                        per = -(-min(budget, x) // 16)
                        dst[s, :per] = ids[at:at + per]
                        at += per
                batch = R.Batch(DEV, [1] * 5, kv, table.to(DEV))
                mass = 1.0 + torch.rand(2, 40, 16, device=DEV)
                keep, kept = cache.keep(batch, mass, budget)
                want = mass.clone()
                for s, x in enumerate(kv):
                    count = min(budget, x)
                    to = (table if dst is None else dst)[s].long()
                    end = -(-(x if dst is None else count) // 16) * 16
                    for h in range(2):
                        frm = keep[s, h, :count].long().cpu()
                        row = torch.cat([mass[h, table[s].long()[frm // 16].to(DEV), (frm % 16).to(DEV)], torch.zeros(end - count, device=DEV)])
                        p = torch.arange(end)
                        want[h, to[p // 16].to(DEV), (p % 16).to(DEV)] = row
                cache.compact(batch, keep, kept, mass, None if dst is None else dst.to(DEV))
                torch.cuda.synchronize()
                assert torch.equal(mass, want), (kv, budget, to_other_pages)


@pytest.mark.gpu
@pytest.mark.parametrize("page", [16, 256])
def test_mass_clear_at_its_borders(page):
    """Lengths behind and before the sequence, entries out of range, sequences without tokens, a long one; a captured call."""
    import paper_2606_30389_amd as P
    kv, start = [1, 0, 5 * page, 3 * page + 1, 70001, 2 * page], [0, 5, -2 ** 31, 2 ** 31 - 1, 1234, 2 * page]
    b = S.Batch([1] * 6, kv, page, device=DEV, seed=3, single=True)
    b.d_table[2, 1], b.d_table[2, 3] = -1, 2 ** 30
    dims, batch = P.make_dims(3, 3, page, b.pool, P.PRR_F16), b.make(P)
    from_len = torch.tensor(start, dtype=torch.int32, device=DEV)
    was = 1.0 + torch.rand(3, b.pool, page, device=DEV)
    want = was.clone()
    for s, n in enumerate(kv):
        for p in range(-(-n // page)):
            first = min(max(start[s] - p * page, 0), page) if start[s] < n else min(max(n - p * page, 0), page)
            if 0 <= int(b.d_table[s, p]) < b.pool:
                want[:, int(b.d_table[s, p]), first:] = 0.0
    mass = was.clone()
    P.prr_mass_clear(dims, batch, from_len, mass)
    torch.cuda.synchronize()
    assert torch.equal(mass, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        P.prr_mass_clear(dims, batch, from_len, mass)
    for _ in range(3):
        mass.copy_(was)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(mass, want)
    # the batch's own length: the rest of the last pages
    mass.copy_(was)
    P.prr_mass_clear(dims, batch, batch.tensors[1], mass)
    torch.cuda.synchronize()
    for s, n in enumerate(kv):
        if n % page:
            was[:, int(b.d_table[s, n // page]), n % page:] = 0.0
    assert torch.equal(mass, was)


@pytest.mark.gpu
@pytest.mark.parametrize("lists", [False, True])
def test_mass_in_a_buffer_of_ones_own(lists):
    """A given out that is not `before`: the call's tokens on top of `before`, all else as it was in out."""
    from paper_2606_30389_amd import runtime as R
    cfg = R.PathConfig(num_q_heads=8, num_kv_heads=2, page_size=16, num_tokens=128, k_select=1)
    cache = R.PagedCache(cfg, DEV, k=rand(2, 8, 16, S.D), v=rand(2, 8, 16, S.D, seed=1))
    table = torch.tensor([[5, 2, 7, 0]], dtype=torch.int32, device=DEV)
    q, batch = rand(1, 8, S.D, seed=2), R.Batch(DEV, [1], [50], table)
    given = dict(pages=torch.tensor([[[1, 0], [3, 2]]], dtype=torch.int32, device=DEV),
                 counts=torch.tensor([[1, 2]], dtype=torch.int32, device=DEV)) if lists else {}
    _, _, m, l = cache.attend(batch, q, **given)
    before, out = torch.rand(2, 8, 16, device=DEV), 9.0 + torch.rand(2, 8, 16, device=DEV)
    want, was = cache.weigh(batch, q, m, l, before=before, decay=0.5, **given), out.clone()
    got = cache.weigh(batch, q, m, l, before=before, decay=0.5, out=out, **given)
    torch.cuda.synchronize()
    written = torch.zeros(2, 8, 16, dtype=torch.bool, device=DEV)
    for h, logical in enumerate([[1], [3, 2]] if lists else [range(4)] * 2):
        for lp in logical:
            written[h, int(table[0, lp]), :min(16, 50 - 16 * lp)] = True
    assert got is out and torch.equal(got[written], want[written]) and torch.equal(got[~written], was[~written])
