"""prr_decode_attn against 64 bits: whole caches and page lists, 16-bit and e4m3, ragged batches, empty
sequences, scales of any size, entries out of range, graphs and streams."""
import math

import pytest
import torch

from tests import context_support as S

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f16": torch.float16}


class Case:
    def __init__(self, kv, hq, hkv, dt="bf16", page=16, kind="16", paged=True, lists=None, spread=1.5, scales=(120, 124),
                 pad=0, garbage=True):
        import paper_2606_30389_amd as P
        self.P = P
        self.b = b = S.Batch([1] * len(kv), kv, page, pad=pad, paged=paged, device=DEV, seed=4, single=True)
        self.hq, self.hkv, self.dt, self.kind, self.lists = hq, hkv, dt, kind, lists
        g = torch.Generator(device=DEV).manual_seed(S.seed_of(kv, hq, hkv, dt, page, kind))
        rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
        self.q = (spread * rand(b.total, hq, S.D)).to(DT[dt])
        shape = (hkv, b.pool, page, S.D)
        used = torch.zeros(b.pool * page, dtype=torch.bool)
        for s in range(len(kv)):
            used[b.slots(s, 0, kv[s])] = True
        unused = ~used.to(DEV)
        if kind == "e4m3":
            self.cache = [(40 * rand(*shape)).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for _ in range(2)]
            self.scale = [torch.randint(*scales, shape[:3], generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
            if garbage:
                for c, s in zip(self.cache, self.scale):
                    c.flatten(1, 2)[:, unused] = 0x7f  # NaN
                    s.flatten(1, 2)[:, unused] = 255
        else:
            self.cache = [rand(*shape).to(DT[dt]) for _ in range(2)]
            self.scale = [None, None]
            if garbage:
                for c in self.cache:
                    c.flatten(1, 2)[:, unused] = math.nan
        self.dims = P.make_dims(hq, hkv, page, b.pool, P.PRR_BF16 if dt == "bf16" else P.PRR_F16)
        self.pages = self.count = None
        if lists is not None:
            cap = max(1, max(len(x) for per in lists for x in per))
            pages = torch.full((len(kv), hkv, cap), -3, dtype=torch.int32)
            for s, per in enumerate(lists):
                for h, x in enumerate(per):
                    pages[s, h, :len(x)] = torch.tensor(x, dtype=torch.int32)
            self.pages = pages.to(DEV)
            self.count = torch.tensor([[len(x) for x in per] for per in lists], dtype=torch.int32, device=DEV)
        self.batch = b.make(P)
        self.cap = 0 if lists is None else self.pages.shape[-1]
        self.code = P.PRR_KV_E4M3 if kind == "e4m3" else P.PRR_KV_16
        self.nbytes = P.prr_decode_workspace_size(self.dims, self.batch, self.code, self.cap)
        self.ws = torch.full((max(self.nbytes, 256),), 0xff, dtype=torch.uint8, device=DEV)

    def outputs(self):
        n = self.b.total
        return [torch.full((n, self.hq, S.D), 5.0, device=DEV), torch.full((n, self.hq, S.D), 5.0, dtype=DT[self.dt], device=DEV),
                torch.full((n, self.hq), 5.0, device=DEV), torch.full((n, self.hq), 5.0, device=DEV)]

    def run(self, out=None, stream=None, ws=None):
        out = self.outputs() if out is None else out
        self.P.prr_decode_attn(self.dims, self.batch, self.q, self.code, *self.cache, *self.scale, self.pages, self.count,
                               self.cap, *out, self.ws if ws is None else ws, self.nbytes, stream)
        return out

    def rows(self, i, h, slot):
        if self.kind == "e4m3":
            p = torch.exp2(self.scale[i][h].flatten()[slot].double() - 127)
            return self.cache[i][h].flatten(0, 1)[slot].view(torch.float8_e4m3fn).double() * p[:, None]
        return self.cache[i][h].flatten(0, 1)[slot].double()

    def check(self, out=None, skip=()):
        out = self.run(out)
        torch.cuda.synchronize()
        G, b = self.hq // self.hkv, self.b
        eps = S.half_step(DT[self.dt])
        two = torch.float16 if self.kind == "e4m3" else DT[self.dt]
        # a weight in two float16 terms: one rounding of the rest of one rounding, subnormal below 2^-24; in three
        # bfloat16 ones: one more
        werr, floor = (S.half_step(two) ** 2, 2.0 ** -25) if two == torch.float16 else (S.half_step(two) ** 3, 0.0)
        for s, kv in enumerate(b.kv):
            for h in range(self.hkv):
                pos = torch.arange(kv)
                if self.lists is not None:
                    pg = torch.tensor([p for p in self.lists[s][h] if 0 <= p < -(-kv // b.page) and (s, p) not in skip], dtype=torch.long)
                    pos = (pg[:, None] * b.page + torch.arange(b.page)).flatten()
                    pos = pos[pos < kv]
                elif skip:
                    pos = pos[[(s, int(p) // b.page) not in skip for p in pos]]
                slot = (b.table[s].long()[pos // b.page] * b.page + pos % b.page).to(DEV)
                k, v = self.rows(0, h, slot), self.rows(1, h, slot)
                heads = slice(h * G, (h + 1) * G)
                o64, m64, l64, a, mag = S.attend64(self.q[s, heads].double(), k, v)
                m, l = out[2][s, heads].double(), out[3][s, heads].double()
                fl = floor * len(pos) * float(v.abs().max()) if len(pos) else 0.0
                S.check_state(out[0][s, heads].double(), m, l, o64, m64, l64, a, mag, werr, 2.0 ** -22, len(pos), fl, (s, h))
                S.check_state(out[1][s, heads].double(), m, l, o64, m64, l64, a, mag, werr + eps, eps, len(pos),
                              fl + (2.0 ** -25 if self.dt == "f16" else 0.0), (s, h))
        for x in out:
            assert torch.all(x[len(b.kv):] == 5.0)
        return out


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["16", "e4m3"])
@pytest.mark.parametrize("kv", [0, 1, 15, 16, 17, 127, 128, 129, 1000, 4096, 20011])
def test_decode_lengths(kv, kind):
    Case([kv], 16, 1, kind=kind).check()
    Case([max(1, kv)], 4, 2, dt="f16", kind=kind, paged=False, page=64).check()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["16", "e4m3"])
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hkv,page", [(1, 1, 16), (32, 2, 16), (28, 4, 64), (5, 1, 32), (8, 8, 256), (6, 2, 128), (36, 3, 16)])
def test_decode_heads_and_pages(hq, hkv, page, dt, kind):
    Case([700, 0, 1, 333, 16], hq, hkv, dt, page, kind, pad=2).check()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["16", "e4m3"])
@pytest.mark.parametrize("page", [16, 64])
def test_decode_lists(page, kind):
    n = -(-3001 // page)
    lists = [[list(range(0, n, 2)), [n - 1]], [[], [0]], [[1], list(range(2))]]
    Case([3001, 5, 2 * page], 8, 2, page=page, kind=kind, lists=lists).check()
    # entries out of range, in the middle of a list, are skipped
    Case([3001], 16, 1, page=page, kind=kind, lists=[[[-1, 0, n, 3, 1 << 30, 5]]]).check()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["16", "e4m3"])
def test_decode_bad_table_entries(kind):
    c = Case([400, 90], 4, 2, kind=kind)
    c.b.table[0, 3], c.b.table[1, 5] = 1 << 30, -1
    c.b.d_table.copy_(c.b.table)
    c.b.table[0, 3], c.b.table[1, 5] = 0, 0  # (not used by the check)
    c.check(skip={(0, 3), (1, 5)})


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["16", "e4m3"])
def test_decode_many_sequences(kind):
    Case([1 + (97 * i) % 400 for i in range(90)], 8, 2, kind=kind, pad=1).check()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_decode_e4m3_scales_far_apart(dt):
    """Value scales over 40 powers of two in one row of tokens (a few rows' values outweigh all others), key scales
    small enough that no logit takes over."""
    c = Case([500], 8, 2, dt, kind="e4m3", scales=(110, 122))
    c.scale[1].copy_(torch.randint(70, 110, c.scale[1].shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)).to(torch.uint8))
    c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["16", "e4m3"])
def test_decode_flat_and_sharp(kind):
    Case([600], 8, 2, kind=kind, spread=0.0).check()
    Case([600], 8, 2, "f16", kind=kind, spread=10.0).check()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["16", "e4m3"])
def test_decode_repeats_graphs_and_streams(kind):
    c = Case([2500, 900, 0], 8, 2, kind=kind)
    want = c.check()
    again = c.run()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, again))
    # two calls at once on two streams, each with its workspace
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [c.outputs() for _ in streams]
    wss = [torch.empty_like(c.ws) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(5):
        for o, s, ws in zip(outs, streams, wss):
            c.run(o, s, ws)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for o in outs for x, y in zip(want, o))
    # captured once, replayed as the sequences grow
    out = c.outputs()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[0]):
        c.run(out, streams[0])
    for lens in ([1, 2, 3], [2500, 0, 0], [777, 900, 0], [2500, 900, 0]):
        c.b.d_kv.copy_(torch.tensor(lens, dtype=torch.int32))
        eager = c.run(ws=wss[0])
        for x in out:
            x.fill_(5.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        # (a row's third sequence holds no page of its own: its lengths here stay within its table's width)
        assert all(torch.equal(x[:2], y[:2]) for x, y in zip(eager, out))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["16", "e4m3"])
@pytest.mark.parametrize("kv", [40, 9000])
def test_decode_nan_is_not_an_empty_state(kv, kind):
    """A query or keys of NaN give NaN, in one part and in many; other sequences and heads are untouched."""
    c = Case([kv, 300], 8, 2, kind=kind)
    want = c.check()
    c.q[0, 1] = math.nan
    out = c.run()
    torch.cuda.synchronize()
    assert out[0][0, 1].isnan().all() and out[1][0, 1].isnan().all() and out[3][0, 1].isnan()
    keep = torch.ones(2, 8, dtype=torch.bool, device=DEV)
    keep[0, 1] = False
    assert all(torch.equal(x[keep], y[keep]) for x, y in zip(out, want))
    c.q[0, 1] = 1.0
    slot = c.b.slots(1, 0, 300).to(DEV)
    if kind == "e4m3":
        c.cache[0].view(torch.uint8)[0].flatten(0, 1)[slot] = 0x7f
    else:
        c.cache[0][0].flatten(0, 1)[slot] = math.nan
    out = c.run()
    torch.cuda.synchronize()
    assert out[0][1, :4].isnan().all() and out[3][1, :4].isnan().all()
    assert all(torch.equal(x[1, 4:], y[1, 4:]) for x, y in zip(out, want))
