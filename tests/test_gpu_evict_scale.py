"""Shaped attention and eviction in large pools, with very many sequences, and several calls at once."""
import pytest
import torch

from tests import context_support as S
from tests.shape_support import Shape, keep_of, slopes_of

DEV = "cuda:0"


def rand(*shape, seed=0, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


@pytest.mark.gpu
def test_rows_behind_four_gigabytes():
    """A sequence in the last pages of a pool whose last head's rows lie more than 2^32 bytes behind its beginning: the
    bits of the same sequence in a small pool."""
    import paper_2606_30389_amd as P
    hkv, hq, page, n, big = 16, 16, 16, 700, 131072
    per = -(-n // page)
    small_k, small_v = rand(hkv, per, page, S.D, seed=1), rand(hkv, per, page, S.D, seed=2)
    q = rand(20, hq, S.D, seed=3)
    kv = torch.tensor([n], dtype=torch.int32, device=DEV)
    cu = torch.tensor([0, 20], dtype=torch.int32, device=DEV)
    keep = torch.stack([torch.randperm(n, generator=torch.Generator().manual_seed(h))[:300].sort().values for h in range(hkv)])
    keep, kept = keep.to(torch.int32)[None].to(DEV), torch.tensor([300], dtype=torch.int32, device=DEV)
    results = []
    for pool in (per, big):
        k, v = (x.clone() if pool == per else torch.zeros(hkv, pool, page, S.D, dtype=x.dtype, device=DEV) for x in (small_k, small_v))
        if pool == big:
            k[:, -per:], v[:, -per:] = small_k, small_v
            assert k[-1, -per].data_ptr() - k.data_ptr() > 1 << 32
        table = torch.arange(pool - per, pool, dtype=torch.int32, device=DEV)[None]
        dims = P.make_dims(hq, hkv, page, pool, P.PRR_BF16)
        b = P.make_batch(1, 20, 20, n, cu, kv, table, per)
        one = P.make_batch(1, 1, 1, n, None, kv, table, per)
        sh = Shape(cap=9.0, slopes=slopes_of(hq), window=400).make(P, DEV)
        out, m, l = torch.zeros_like(q), torch.zeros(20, hq, device=DEV), torch.zeros(20, hq, device=DEV)
        ws = torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
        P.prr_prompt_attn_shaped(dims, b, sh, q, k, v, out, m, l, ws, 1 << 24)
        o32 = torch.zeros(1, hq, S.D, device=DEV)
        m1, l1 = torch.zeros(1, hq, device=DEV), torch.zeros(1, hq, device=DEV)
        P.prr_decode_attn_shaped(dims, one, sh, q[:1], 0, k, v, None, None, None, None, 0, o32, None, m1, l1, ws, 1 << 24)
        mass = torch.zeros(hkv, pool, page, device=DEV)
        P.prr_key_mass(dims, b, sh, q, 0, k, None, m, l, 0, None, None, 0, None, 0.0, mass, ws, 1 << 24)
        before = mass[:, -per:].clone()
        P.prr_cache_compact(dims, one, keep, kept, 300, 0, k, v, None, None, mass, None, 0, ws, 1 << 24)
        torch.cuda.synchronize()
        results.append([out, m, l, o32, m1, l1, before, mass[:, -per:].clone(), k[:, -per:].clone(), v[:, -per:].clone()])
        if pool == big:
            assert not k[:, :-per].any() and not mass[:, :-per].any()
    assert all(torch.equal(x, y) for x, y in zip(*results))
    assert results[0][6].any()


@pytest.mark.gpu
def test_as_many_sequences_as_there_may_be():
    """4096 sequences of 0 to 40 tokens, 0 to 3 of them new."""
    import paper_2606_30389_amd as P
    n, hq, hkv, budget = 4096, 4, 2, 9
    new = [(5 * i) % 4 for i in range(n)]
    kv = [max(a, (11 * i) % 41) for i, a in enumerate(new)]
    b = S.Batch(new, kv, 16, device=DEV, seed=8, pad=2)
    dims, batch = P.make_dims(hq, hkv, 16, b.pool, P.PRR_BF16), b.make(P)
    q, k, v = rand(b.total, hq, S.D, seed=1), rand(hkv, b.pool, 16, S.D, seed=2), rand(hkv, b.pool, 16, S.D, seed=3)
    sh = Shape(cap=5.0, window=20).make(P, DEV)
    out, m, l = torch.zeros_like(q), torch.zeros(b.total, hq, device=DEV), torch.zeros(b.total, hq, device=DEV)
    ws = torch.empty(1 << 26, dtype=torch.uint8, device=DEV)
    assert P.prr_mass_workspace_size(dims, batch, sh, 0) <= 1 << 26 and P.prr_compact_workspace_size(dims, batch, 0, budget) <= 1 << 26
    P.prr_prompt_attn_shaped(dims, batch, sh, q, k, v, out, m, l, ws, 1 << 26)
    mass = torch.full((hkv, b.pool, 16), 5.0, device=DEV)
    P.prr_key_mass(dims, batch, sh, q, 0, k, None, m, l, 0, None, None, 0, None, 0.0, mass, ws, 1 << 26)
    flat = mass.flatten(1, 2).clone()
    used = torch.cat([b.slots(s, 0, x) for s, x in enumerate(kv)]).to(DEV)
    rest = torch.ones(b.pool * 16, dtype=torch.bool, device=DEV)
    rest[used] = False
    assert torch.all(flat[:, rest] == 5.0)
    # every token with a place spreads a weight of one per head
    assert abs(flat[:, used].double().sum().item() / (sum(new) * hq) - 1) < 2 ** -12
    keep = torch.zeros(n, hkv, budget, dtype=torch.int32, device=DEV)
    kept = torch.zeros(n, dtype=torch.int32, device=DEV)
    P.prr_keep_tokens(dims, batch, mass, budget, 1, 2, keep, kept, None, 0)
    was = k.clone()
    P.prr_cache_compact(dims, batch, keep, kept, budget, 0, k, v, None, None, mass, None, 0, ws, 1 << 26)
    torch.cuda.synchronize()
    assert kept.tolist() == [min(budget, x) for x in kv]
    flat, keep_cpu = flat.cpu(), keep.cpu()
    for s in list(range(0, n, 97)) + [n - 1]:
        for h in range(hkv):
            slot = b.slots(s, 0, kv[s])
            want = keep_of(flat[h, slot].tolist(), budget, 1, 2)
            assert keep_cpu[s, h, :len(want)].tolist() == want
            assert torch.equal(k[h].flatten(0, 1)[slot[:len(want)].to(DEV)], was[h].flatten(0, 1)[slot[want].to(DEV)])


@pytest.mark.gpu
def test_keep_of_a_million_tokens():
    import paper_2606_30389_amd as P
    n, budget = 1 << 20, 50000
    mass = torch.rand(1, n // 256, 256, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    mass[0, ::7] = 0.75  # (many equal ones around the threshold)
    dims = P.make_dims(1, 1, 256, n // 256, P.PRR_BF16)
    batch = P.make_batch(1, 1, 1, n, None, torch.tensor([n - 5], dtype=torch.int32, device=DEV))
    nbytes = P.prr_keep_workspace_size(dims, batch, budget)
    ws = torch.full((nbytes,), 0xff, dtype=torch.uint8, device=DEV)
    for budget in (50000, 300000):
        keep, kept = torch.zeros(1, 1, budget, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        P.prr_keep_tokens(dims, batch, mass, budget, 4, 100, keep, kept, ws, nbytes)
        torch.cuda.synchronize()
        x = mass.flatten()[:n - 5].clone()
        x[:4] = x[-100:] = 2.0
        want = x.sort(descending=True, stable=True).indices[:budget].sort().values.to(torch.int32)
        assert torch.equal(keep[0, 0], want)


@pytest.mark.gpu
def test_two_graphs_of_one_cache_at_once():
    """Weights by parts of the rows and choices by chunks, captured twice and replayed on two streams at the same time, eager
    calls in between: each has a workspace of its own."""
    from paper_2606_30389_amd import runtime as R
    n = 40000
    cfg = R.PathConfig(num_q_heads=16, num_kv_heads=1, page_size=16, num_tokens=n, k_select=1)
    cache = R.PagedCache(cfg, DEV, k=rand(1, 2500, 16, S.D, seed=1), v=rand(1, 2500, 16, S.D, seed=2))
    batches = [R.Batch(DEV, [300], [3000]), R.Batch(DEV, [200], [2500])]
    whole = R.Batch(DEV, [1], [n])
    from paper_2606_30389_amd import _lib as L
    assert all(L.prr_mass_workspace_size(cache.dims, b.native, None, 0) for b in batches) and L.prr_keep_workspace_size(cache.dims, whole.native, 5)
    qs = [rand(300, 16, S.D, seed=3), rand(200, 16, S.D, seed=4)]
    stats = [cache.prompt(b, q)[1:] for b, q in zip(batches, qs)]
    held = torch.rand(1, 2500, 16, device=DEV)

    def calls(i):
        return (cache.weigh(batches[i], qs[i], *stats[i]), *cache.keep(whole, held, 3000 + i, sink=2, recent=5))

    want = [calls(i) for i in range(2)]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(calls(i))
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(20):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        got = [calls(i) for i in range(2)]
        torch.cuda.synchronize()
        for a, o, w in zip(got, outs, want):
            assert all(torch.equal(x, y) for x, y in zip(a, w)) and all(torch.equal(x, y) for x, y in zip(o, w))
            for x in o:
                x.fill_(2)
        torch.cuda.synchronize()
