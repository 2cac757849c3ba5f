"""prr_prompt_attn against 64 bits: packed and ragged prompts, cached beginnings, rows that see no key, head
shapes, page sizes, both 16-bit types, the keys of few rows split over many workgroups."""
import math

import pytest
import torch

from tests import context_support as S

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f16": torch.float16}


def run_case(new, kv, hq, hkv, dt="bf16", page=16, pad=0, paged=True, spread=1.5, single=False, ml=True, spare=3, edit=None):
    import paper_2606_30389_amd as P
    b = S.Batch(new, kv, page, pad=pad, paged=paged, device=DEV, seed=9, single=single, spare=spare)
    G = hq // hkv
    g = torch.Generator(device=DEV).manual_seed(S.seed_of(new, kv, hq, hkv, dt, page))
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    q = (spread * rand(b.total, hq, S.D)).to(DT[dt])
    cache = [rand(hkv, b.pool, page, S.D).to(DT[dt]) for _ in range(2)]
    if edit:
        edit(b, q, cache)
    used = torch.zeros(b.pool * page, dtype=torch.bool)
    for s in range(len(new)):
        used[b.slots(s, 0, kv[s])] = True
    for c in cache:  # what no sequence holds must not matter
        c.flatten(1, 2)[:, ~used.to(DEV)] = math.nan
    out = torch.full((b.total, hq, S.D), 5.0, dtype=DT[dt], device=DEV)
    m, l = (torch.full((b.total, hq), 5.0, device=DEV) for _ in range(2))
    dims = P.make_dims(hq, hkv, page, b.pool, P.PRR_BF16 if dt == "bf16" else P.PRR_F16)
    batch = b.make(P)
    nbytes = P.prr_prompt_workspace_size(dims, batch)
    ws = torch.full((max(nbytes, 256),), 0xff, dtype=torch.uint8, device=DEV) if nbytes else None
    P.prr_prompt_attn(dims, batch, q, *cache, out, m if ml else None, l if ml else None, ws, nbytes)
    torch.cuda.synchronize()
    eps = S.half_step(DT[dt])
    floor = 2.0 ** -24 if dt == "f16" else 0.0  # a weight or an output below float16's normal range
    for s, rows, pos in b.sequences():
        if not len(rows):
            continue
        slot = b.slots(s, 0, kv[s]).to(DEV)
        rows, pos = rows.to(DEV), pos.to(DEV)
        visible = (torch.arange(kv[s], device=DEV) <= pos[:, None]).repeat_interleave(G, 0)
        for h in range(hkv):
            k, v = (c[h].flatten(0, 1)[slot].double() for c in cache)
            qq = q[rows, h * G:(h + 1) * G].double().reshape(-1, S.D)
            o64, m64, l64, a, mag = S.attend64(qq, k, v, visible)
            seen = l64 > 0
            vmax = v.abs().max() if kv[s] else 0.0
            fl = floor * (1 + kv[s] * vmax)
            got = [x[rows, h * G:(h + 1) * G].double().reshape(-1, *x.shape[2:]) for x in (out, m, l)]
            if not ml:
                got[1], got[2] = m64, l64
            S.check_state(*got, o64, m64, l64, a, mag, eps, eps, kv[s], fl, what=(s, h))
            assert seen.sum() == (pos >= 0).sum() * G
    assert torch.all(out[b.cu[-1]:] == 5.0) and torch.all(m[b.cu[-1]:] == 5.0) and torch.all(l[b.cu[-1]:] == 5.0)
    return P, dims, batch, q, cache, out, m, l, ws, nbytes


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 127, 130, 257, 700])
def test_prompt_lengths(n):
    run_case([n], [n], 16, 1)
    run_case([n], [n], 4, 4, dt="f16", paged=False)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hkv,page", [(1, 1, 16), (32, 2, 16), (28, 4, 64), (5, 1, 32), (8, 8, 256), (6, 2, 128), (36, 3, 16)])
def test_prompt_heads_and_pages(hq, hkv, page, dt):
    run_case([300, 0, 1, 45], [300, 7, 500, 111], hq, hkv, dt, page, pad=3)


@pytest.mark.gpu
def test_prompt_many_sequences():
    new = [(37 * i) % 23 for i in range(150)]
    kv = [n + (53 * i) % 91 * (i % 3 > 0) for i, n in enumerate(new)]
    run_case(new, kv, 8, 2, pad=2)


@pytest.mark.gpu
@pytest.mark.parametrize("long_at", [0, 700, 1499])
def test_prompt_one_long_among_many(long_at):
    """1500 sequences of 0 to 6 new tokens and one of 600: tiles are numbered by rows."""
    new = [(11 * i) % 7 for i in range(1500)]
    new[long_at] = 600
    kv = [n + (i % 4) * 3 for i, n in enumerate(new)]
    run_case(new, kv, 4, 1, pad=1)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 63, 64, 65, 129])
def test_prompt_tile_numbers(n):
    """Lengths around whole tiles of 128 and 256 rows, in both numberings (one much longer, or all alike)."""
    new = [[31, 32, 33, 64, 0, 1, 63][i % 7] for i in range(n)]
    kv = [x + (1100 if i == n // 2 else 2) for i, x in enumerate(new)]  # (longer than 1024: eight waves)
    run_case(new, kv, 8, 2)
    run_case(new + [500], kv + [500], 8, 2)
    run_case(new, [x + 1 for x in new], 8, 2, dt="f16")


@pytest.mark.gpu
@pytest.mark.parametrize("new,kv", [([3], [5000]), ([1, 2], [3000, 4097]), ([130], [2000])])
@pytest.mark.parametrize("hq,hkv", [(16, 1), (2, 2)])
def test_prompt_few_rows_many_keys(new, kv, hq, hkv):
    """Few rows: the keys are split over workgroups and joined."""
    P, dims, batch, *_ = run_case(new, kv, hq, hkv, pad=1)
    assert P.prr_prompt_workspace_size(dims, batch) > 0


@pytest.mark.gpu
def test_prompt_rows_without_keys():
    """Fewer cached than new tokens: the first new tokens have negative positions and see nothing."""
    run_case([10, 70, 4], [3, 0, 4], 8, 2, pad=2)
    run_case([300], [130], 16, 1, dt="f16")


@pytest.mark.gpu
def test_prompt_single_tokens():
    run_case([1] * 40, [1 + 71 * i % 900 for i in range(40)], 8, 2, single=True)


@pytest.mark.gpu
def test_prompt_without_statistics():
    run_case([33], [90], 4, 2, ml=False)


@pytest.mark.gpu
@pytest.mark.parametrize("spread", [0.0, 12.0])
def test_prompt_flat_and_sharp(spread):
    """All weights equal, and rows that one key takes."""
    run_case([200], [260], 8, 2, spread=spread)
    run_case([200], [260], 8, 2, dt="f16", spread=spread)


@pytest.mark.gpu
def test_prompt_rising_maximum():
    """Later keys with ever larger logits: the running maximum moves in every tile, by less and by more than the
    slack that a reference exponent has."""
    def edit(b, q, cache):
        n = b.kv[0]
        slot = b.slots(0, 0, n).to(DEV)
        q.fill_(1.0)
        ramp = torch.arange(n, device=DEV).float()
        for step, h in ((0.004, 0), (0.02, 1)):
            cache[0][h].flatten(0, 1)[slot] = (ramp * step)[:, None].expand(-1, S.D).to(cache[0].dtype).contiguous()
    run_case([400], [500], 8, 2, edit=edit)
    run_case([400], [500], 8, 2, dt="f16", edit=edit)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hkv,n,past", [(16, 1, 40, 100), (2, 2, 300, 90), (4, 1, 1500, 64)])
def test_prompt_non_finite_tokens_reach_only_who_sees_them(hq, hkv, n, past, dt):
    """Infinities and NaN in a token's keys and values change nothing for the tokens before it."""
    import paper_2606_30389_amd as P
    b = S.Batch([n], [past + n], 16, device=DEV, seed=2)
    g = torch.Generator(device=DEV).manual_seed(n)
    q = torch.randn(n, hq, S.D, generator=g, device=DEV).to(DT[dt])
    cache = [torch.randn(hkv, b.pool, 16, S.D, generator=g, device=DEV).to(DT[dt]) for _ in range(2)]
    dims = P.make_dims(hq, hkv, 16, b.pool, P.PRR_BF16 if dt == "bf16" else P.PRR_F16)
    batch = b.make(P)
    nbytes = P.prr_prompt_workspace_size(dims, batch)
    ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=DEV)

    def run(c):
        out = torch.zeros(n, hq, S.D, dtype=DT[dt], device=DEV)
        P.prr_prompt_attn(dims, batch, q, *c, out, None, None, ws, nbytes)
        torch.cuda.synchronize()
        return out

    clean = run(cache)
    for at in (past + n - 1, past + n // 2, past + 3):
        for i, values in ((0, [math.inf]), (1, [math.inf, -math.inf, math.nan])):
            for x in values:
                dirty = [c.clone() for c in cache]
                dirty[i].flatten(1, 2)[:, b.slots(0, at, at + 1).to(DEV), 5] = x
                got = run(dirty)
                sees = at - past
                assert torch.equal(got[:sees], clean[:sees])
                if i == 1:
                    want = got[sees:, :, 5].float()
                    assert torch.all(want.isnan()) if math.isnan(x) else torch.all(want.isnan() | (want == x))
                    keep = [c for c in range(S.D) if c != 5]
                    assert torch.equal(got[sees:][..., keep], clean[sees:][..., keep])


@pytest.mark.gpu
def test_prompt_replayed_in_a_graph():
    """One capture, replayed with other inputs and lengths in the same buffers, eager work in between."""
    P, dims, batch, q, cache, out, m, l, ws, nbytes = run_case([60, 20], [900, 700], 8, 2, spare=0)
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        P.prr_prompt_attn(dims, batch, q, *cache, out, m, l, ws, nbytes)
    cu, kv_len, _ = batch.tensors
    for i in range(4):
        torch.manual_seed(i)
        q.copy_(torch.randn_like(q))
        cache[0].copy_(torch.randn_like(cache[0]))
        cache[1].copy_(torch.randn_like(cache[1]))
        kv_len.copy_(torch.tensor([900 - 13 * i, 700 - 40 * i], dtype=torch.int32))
        cu.copy_(torch.tensor([0, 60 - i, 80 - 2 * i], dtype=torch.int32))
        want = [torch.full_like(x, 2.0) for x in (out, m, l)]
        P.prr_prompt_attn(dims, batch, q, *cache, *want, ws, nbytes)
        for x in (out, m, l):
            x.fill_(2.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((out, m, l), want))


@pytest.mark.gpu
@pytest.mark.parametrize("new,kv", [([20], [50]), ([20], [9000]), ([700], [2000])])
def test_prompt_nan_is_not_an_empty_state(new, kv):
    """A query of NaN gives NaN, in one part and in many; other rows are untouched."""
    P, dims, batch, q, cache, out, m, l, ws, nbytes = run_case(new, kv, 8, 2)
    want = [x.clone() for x in (out, m, l)]
    q[7, 3] = math.nan
    P.prr_prompt_attn(dims, batch, q, *cache, out, m, l, ws, nbytes)
    torch.cuda.synchronize()
    assert out[7, 3].isnan().all() and l[7, 3].isnan()
    keep = torch.ones(new[0], 8, dtype=torch.bool, device=DEV)
    keep[7, 3] = False
    assert all(torch.equal(x[keep], y[keep]) for x, y in zip((out, m, l), want))
