"""Shaped attention and eviction: the calls whose time is followed.

Kinds of case:

* ``prompt``   attention of packed new tokens whose scores are capped by a tanh or lowered with the distance, with
               a sliding window, documents or a prefix that all its tokens see (``prr_prompt_attn_shaped``).
* ``decode``   the same for one token per sequence (``prr_decode_attn_shaped``).
* ``mass``     the attention weight that each cached token received from new tokens, added to what it received before
               (``prr_key_mass``).
* ``keep``     the tokens of each KV head that stay in a smaller cache: the first, the latest and those of the largest
               mass (``prr_keep_tokens``).
* ``compact``  their rows to other pages (``prr_cache_compact``).

With ``own`` false ``run()`` is the definition in elementary torch operations, in 32 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
D = 128


# ------------------------------------------------------------------------------- cases
# seqs: sequences; new: the most new tokens of one; tokens: the most tokens of one in the cache, the new ones included;
# ragged: lengths from one (the first sequence: the given ones) up to these; pad: rows behind the last sequence.
# cap: of the scores (0: none); slopes: a bias by distance; window: keys that a token sees back from itself (0: all);
# prefix: tokens at the beginning that every token sees; docs: documents side by side in a sequence.

def _case(name, kind, **kw):
    c = dict(kind=kind, hq=32, hkv=2, dtype="bf16", page=16, seqs=1, new=1, tokens=4096, ragged=False, paged=False,
             kv="16", pad=0, cap=0.0, slopes=False, window=0, prefix=0, docs=0, name=name)
    if kind == "mass":
        c.update(last=0, decay=0.0)
    if kind in ("keep", "compact"):
        c.update(budget=1024, sink=4, recent=64)
    c.update(kw)
    return c


def listed():
    return [
        # a short question whose instructions all tokens see, scores falling with the distance: latency counts
        _case("prompt_prefix_200", "prompt", hq=28, hkv=4, page=64, new=200, tokens=200, prefix=120, slopes=True, paged=True),
        # nine packed prompts of a layer with capped scores and a sliding window, rows behind the last
        _case("prompt_window_packed9", "prompt", hkv=8, dtype="f16", seqs=9, new=2000, tokens=2500, ragged=True, paged=True,
              pad=5, cap=30.0, window=1024),
        # 32K tokens of documents side by side, capped scores
        _case("prompt_docs_32k", "prompt", new=32768, tokens=32768, docs=12, cap=50.0),
        # a token over a whole quantised 128K cache, scores falling with the distance
        _case("decode_slopes_128k_e4m3", "decode", tokens=131072, kv="e4m3", slopes=True),
        # the tokens of 32 sequences in a layer with a sliding window and capped scores
        _case("decode_window_batch32", "decode", hkv=8, dtype="f16", seqs=32, tokens=16384, ragged=True, paged=True, cap=50.0,
              window=4096),
        # after a step over selected pages: what the pages' tokens received, added up
        _case("mass_256_pages_e4m3", "mass", tokens=131072, kv="e4m3", listed=256, decay=1.0),
        # a long prompt judged by its last 32 tokens
        _case("mass_last32_128k", "mass", new=64, tokens=131072, last=32),
        # what the tokens of a prompt received from all of it, capped scores
        _case("mass_prompt_8k", "mass", hkv=8, dtype="f16", new=8191, tokens=8191, cap=50.0, paged=True),
        # one sequence of 128K tokens to 8K
        _case("keep_128k", "keep", tokens=131072, budget=8192),
        # 32 sequences to at most 2K tokens each
        _case("keep_batch32", "keep", hkv=8, seqs=32, tokens=16384, ragged=True, paged=True, budget=2048),
        # their rows, in e4m3
        _case("compact_batch32_e4m3", "compact", hkv=8, dtype="f16", seqs=32, tokens=16384, ragged=True, paged=True, kv="e4m3",
              budget=2048),
        # a small cache of a single sequence
        _case("compact_1000", "compact", tokens=5000, budget=1000, paged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "prompt", "decode", "decode", "mass", "mass", "keep", "compact"])
    hkv = rng.choice([1, 2, 4, 8])
    group = rng.choice([g for g in (1, 4, 5, 7, 8, 16) if g * hkv <= 64])
    c = _case("", kind, hq=hkv * group, hkv=hkv, dtype=rng.choice(["bf16", "f16"]), page=rng.choice([16, 16, 32, 64, 128, 256]))
    del c["name"]
    seqs = _log_int(rng, 2, 32) if rng.random() < 0.5 else 1
    if kind == "prompt":
        seqs = min(seqs, 16)
        new = _log_int(rng, 2, 8192 // seqs)
        c.update(seqs=seqs, new=new, tokens=new + (0 if rng.random() < 0.5 else _log_int(rng, 1, 16384 // seqs)))
    elif kind == "mass":
        seqs = min(seqs, 16)
        new = 1 if rng.random() < 0.4 else _log_int(rng, 2, 4096 // seqs)
        c.update(seqs=seqs, new=new, tokens=new + (0 if rng.random() < 0.2 else _log_int(rng, 1, 65536 // seqs)),
                 kv=rng.choice(["16", "e4m3"]), decay=rng.choice([0.0, 0.9, 1.0]), last=rng.choice([0, 0, 16, 33]))
        if new == 1 and rng.random() < 0.5:
            c["listed"] = min(_log_int(rng, 1, 512), -(-c["tokens"] // c["page"]))
    else:
        c.update(seqs=seqs, tokens=_log_int(rng, 1, 131072 // seqs), kv=rng.choice(["16", "e4m3"]))
    if kind in ("prompt", "decode", "mass"):
        c["cap"] = rng.choice([0.0, 30.0, 50.0])
        c["slopes"] = rng.random() < 0.3
        which = rng.choice(["none", "window", "docs", "prefix"])
        if which == "window":
            c["window"] = _log_int(rng, 1, 8192)
        elif which == "docs":
            c["docs"] = _log_int(rng, 2, 40)
        elif which == "prefix":
            c["prefix"] = _log_int(rng, 1, c["tokens"])
    if kind in ("keep", "compact"):
        c["kv"] = c["kv"] if kind == "compact" else "16"
        c["budget"] = _log_int(rng, 1, 16384)
        if kind == "keep":  # some tokens to choose, and some to choose them from
            c["tokens"] = max(c["tokens"], 100)
            c["budget"] = min(max(c["budget"], 8), c["tokens"] * 3 // 4)
        c["sink"] = rng.randint(0, min(8, c["budget"] // 2))
        c["recent"] = rng.randint(0, min(256, c["budget"] // 2 - c["sink"]))
    c.update(ragged=seqs > 1 and rng.random() < 0.7, paged=seqs > 1 or rng.random() < 0.5 or kind == "compact",
             pad=rng.choice([0, 3]) if kind in ("prompt", "mass") and c["new"] > 1 else 0)
    # no more than the largest listed case of the kind
    most = max(work(x)["flops" if kind in ("prompt", "mass") else "bytes"] for x in listed() if x["kind"] == kind)
    while work(c)["flops" if kind in ("prompt", "mass") else "bytes"] > most:
        if kind in ("prompt", "mass") and c["new"] > 1:
            gone = c["new"] // 2
            c["new"] -= gone
            c["tokens"] -= gone
        else:
            c["tokens"] = max(1, c["tokens"] // 2)
            if "budget" in c:
                c.update(budget=max(1, c["budget"] // 2), sink=0, recent=0)
        if "listed" in c:
            c["listed"] = min(c["listed"], -(-c["tokens"] // c["page"]))
    return c


# ------------------------------------------------------------------------------- inputs

def _lengths(c):
    """(new tokens, tokens in the cache) of each sequence, by the case alone."""
    n = c["seqs"]
    if not c["ragged"]:
        return [c["new"]] * n, [c["tokens"]] * n
    r = random.Random(n * 1000003 + c["tokens"])
    new = [c["new"] if i == 0 else r.randint(1, c["new"]) for i in range(n)]
    past = c["tokens"] - c["new"]
    kv = [new[i] + (past if i == 0 else r.choice([0, r.randint(0, past)]) if c["kind"] == "prompt" else r.randint(0, past))
          for i in range(n)]
    return new, kv


def _masks(c):
    """Of each sequence: the tokens of its prefix, and where its documents begin (ascending, the first at 0)."""
    _, kv = _lengths(c)
    r = random.Random(c["tokens"] * 31 + c["docs"])
    prefix = [min(c["prefix"], n) if i == 0 else r.randint(0, min(c["prefix"], n)) for i, n in enumerate(kv)]
    docs = [sorted({0, *(r.randrange(n) for _ in range(c["docs"] - 1))}) for n in kv] if c["docs"] else [[0]] * len(kv)
    return prefix, docs


def _counted(c):
    """New tokens of each sequence that the call looks at."""
    new, _ = _lengths(c)
    return [min(n, c["last"]) if c.get("last") else n for n in new]


def _span(c, kv, prefix, docs, pos):
    """The keys [lo, hi) that tokens at positions pos (a tensor) of a sequence see."""
    lo = torch.zeros_like(pos)
    if c["docs"]:
        starts = torch.tensor(docs, device=pos.device)
        lo = starts[(pos[:, None] >= starts).sum(1) - 1]
    if c["window"]:
        lo = torch.maximum(lo, pos - c["window"] + 1)
    hi = (pos + 1).clamp(min=prefix, max=kv)
    return lo, torch.maximum(lo, hi)


def _seen(c):
    """Pairs of a counted new token and a key that it sees, and keys that some counted token sees."""
    _, kv = _lengths(c)
    prefix, docs = _masks(c)
    pairs = keys = 0
    for n, q, p, d in zip(kv, _counted(c), prefix, docs):
        lo, hi = _span(c, n, p, d, torch.arange(n - q, n))
        pairs += int((hi - lo).sum())
        keys += int(hi.max() - lo.min())
    return pairs, keys


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float16


def prepare(case, seed):
    c, dt = case, _dtype(case)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rand = lambda *shape: torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32)  # noqa: E731
    new, kv = _lengths(c)
    hq, hkv, page, n = c["hq"], c["hkv"], c["page"], c["seqs"]
    per = [-(-t // page) for t in kv]
    width = max(per)
    kept = [min(t, c["budget"]) for t in kv] if "budget" in c else [0] * n
    per_dst = [-(-t // page) for t in kept] if c["kind"] == "compact" else [0] * n
    pool = sum(per) + sum(per_dst) + (7 if c["paged"] else 0)
    s = dict(case=c, dt=dt, max_new=max(new), max_kv=max(kv), width=width, pool=pool)
    # the pages of the sequences lie in the pool in any order; entries behind a sequence's last page are never read
    ids = torch.randperm(pool, generator=torch.Generator().manual_seed(seed)).to(torch.int32) if c["paged"] else torch.arange(pool, dtype=torch.int32)
    at = 0
    for name, counts in (("table", per), ("dst_table", per_dst)):
        table = torch.zeros(n, max(1, max(counts)), dtype=torch.int32)
        for i, x in enumerate(counts):
            table[i, :x] = ids[at:at + x]
            at += x
        s[name] = table.to(DEV)
    cu = [0]
    for x in new:
        cu.append(cu[-1] + x)
    total = cu[-1] + c["pad"]
    s.update(total=total, cu=torch.tensor(cu, dtype=torch.int32, device=DEV), kv_len=torch.tensor(kv, dtype=torch.int32, device=DEV))
    if c["kind"] in ("prompt", "decode", "mass"):
        prefix, docs = _masks(c)
        # capped scores are as large as such layers have them
        s["q"] = ((4.0 if c["cap"] else 1.5) * rand(total, hq, D)).to(dt)
        s["slopes"] = torch.exp2(-8.0 * torch.arange(1, hq + 1, device=DEV) / hq) if c["slopes"] else None
        s["prefix"] = torch.tensor(prefix, dtype=torch.int32, device=DEV) if c["prefix"] else None
        s["first"] = None
        if c["docs"]:
            s["first"] = torch.zeros(total, dtype=torch.int32, device=DEV)
            for i in range(n):
                starts = torch.tensor(docs[i], device=DEV)
                pos = torch.arange(kv[i] - new[i], kv[i], device=DEV)
                s["first"][cu[i]:cu[i + 1]] = starts[(pos[:, None] >= starts).sum(1) - 1].to(torch.int32)
    if c["kind"] == "keep":
        # most of the weight on few tokens, and many that received none
        s["mass"] = torch.exp(2.0 * rand(hkv, pool, page))
        s["mass"].masked_fill_(torch.rand(hkv, pool, page, generator=gen, device=DEV) < 0.3, 0.0)
        s["keep"] = torch.zeros(n, hkv, c["budget"], dtype=torch.int32, device=DEV)
        s["kept"] = torch.zeros(n, dtype=torch.int32, device=DEV)
        return s
    cache = (hkv, pool, page, D)
    names = "k" if c["kind"] == "mass" else "kv"
    for t in names:
        x = rand(*cache)
        if c["kv"] == "e4m3":
            s[t + "_cache"], s[t + "_scale"] = _quantise(x)
        else:
            s[t + "_cache"] = x.to(dt)
    if c["kind"] in ("prompt", "decode"):
        s["out"] = torch.zeros(total, hq, D, dtype=dt, device=DEV)
        s["m"], s["l"] = torch.zeros(total, hq, device=DEV), torch.zeros(total, hq, device=DEV)
        if c["kind"] == "decode":
            s["out32"] = torch.zeros(total, hq, D, device=DEV)
    elif c["kind"] == "mass":
        if "listed" in c:  # distinct pages of each sequence and KV head, ascending
            count = torch.tensor([min(c["listed"], x) for x in per], dtype=torch.int32, device=DEV)
            order = torch.rand(n, hkv, width, generator=gen, device=DEV)
            order.masked_fill_(torch.arange(width, device=DEV) >= torch.tensor(per, device=DEV)[:, None, None], 2.0)
            order = order.argsort(-1)[..., :c["listed"]].contiguous()
            order.masked_fill_(torch.arange(order.shape[-1], device=DEV) >= count[:, None, None], width)
            order = order.sort(-1).values
            s["pages"] = torch.where(order < width, order, 0).to(torch.int32).contiguous()
            s["count"] = count[:, None].expand(-1, hkv).contiguous()
        s["before"] = torch.rand(hkv, pool, page, generator=gen, device=DEV) if c["decay"] else None
        s["mass"] = torch.zeros(hkv, pool, page, device=DEV)
        # the statistics that the attention of these tokens gave
        s["m"], s["l"] = torch.zeros(total, hq, device=DEV), torch.zeros(total, hq, device=DEV)
        for i, rows, pos, z, _ in _scores(s):
            m = z.amax(-1)
            z.sub_(torch.where(m == -math.inf, 0.0, m)[..., None]).exp_()
            s["m"][rows], s["l"][rows] = _by_row(m), _by_row(z.sum(-1))
    else:
        s["mass"] = torch.rand(hkv, pool, page, generator=gen, device=DEV)
        order = torch.rand(n, hkv, s["max_kv"], generator=gen, device=DEV)
        at = torch.arange(s["max_kv"], device=DEV)
        tokens = s["kv_len"].long()[:, None]
        order[(((at < c["sink"]) | (at >= tokens - c["recent"])) & (at < tokens))[:, None].expand(-1, hkv, -1)] = -1.0
        order.masked_fill_((at >= tokens)[:, None], 2.0)
        s["kept"] = torch.tensor(kept, dtype=torch.int32, device=DEV)
        order = order.argsort(-1)[..., :c["budget"]]
        order = torch.where(torch.arange(order.shape[-1], device=DEV) < s["kept"][:, None, None], order, s["max_kv"]).sort(-1).values
        s["keep"] = torch.zeros(n, hkv, c["budget"], dtype=torch.int32, device=DEV)
        s["keep"][..., :order.shape[-1]] = torch.where(order < s["max_kv"], order, 0).to(torch.int32)
    return s


def _quantise(x):
    """e4m3 codes of the rows of x and the bytes of their power-of-two scales."""
    f, e = torch.frexp(x.abs().amax(-1))
    # amax = 2f 2^(e-1) and 448 = 1.75 2^8
    e = (e - 9 + (2 * f > 1.75)).clamp(min=-126)
    return torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


# ------------------------------------------------------------------------------- the plain forms

def _slots(s, i, first, last):
    """Pool slots of positions [first, last) of sequence i."""
    page = s["case"]["page"]
    pos = torch.arange(first, last, device=DEV)
    return s["table"][i].long()[pos // page] * page + pos % page


def _gather(s, t, slot):
    """Cache rows [KV head][...][128] of slots, in 32 bits."""
    x = s[t + "_cache"]
    if x.dtype == torch.float8_e4m3fn:
        x = x.view(torch.uint8).flatten(1, 2)[:, slot].view(torch.float8_e4m3fn).float()
        return torch.ldexp(x, s[t + "_scale"].flatten(1, 2)[:, slot][..., None].int() - 127)
    return x.flatten(1, 2)[:, slot].float()


def _by_row(x):
    """[KV head][group][rows] as [rows][heads]."""
    return x.permute(2, 0, 1).flatten(1)


def _scores(s):
    """Scores of the counted new tokens, some rows and the range of keys that they see at a time: (sequence, rows, the
    positions of the first key and behind the last, scores [KV head][group][rows][keys], slots)."""
    c = s["case"]
    hkv, g = c["hkv"], c["hq"] // c["hkv"]
    new, kv = _lengths(c)
    prefix, docs = _masks(c)
    counted = _counted(c)
    at = 0
    for i in range(c["seqs"]):
        end = at + new[i]
        step = max(1, min(1024, (1 << 30) // (c["hq"] * kv[i])))
        for r0 in range(end - counted[i], end, step):
            rows = torch.arange(r0, min(r0 + step, end), device=DEV)
            pos = kv[i] - end + rows
            # the range of keys, from the lengths alone
            p0, p1 = kv[i] - end + r0, kv[i] - end + min(r0 + step, end) - 1
            k0 = max((max(x for x in docs[i] if x <= p0)) if c["docs"] else 0, p0 - c["window"] + 1 if c["window"] else 0, 0)
            k1 = min(kv[i], max(p1 + 1, prefix[i]))
            slot = _slots(s, i, k0, k1)
            k = _gather(s, "k", slot)
            q = s["q"][rows].float().view(len(rows), hkv, g, D).permute(1, 2, 0, 3).reshape(hkv, -1, D)
            z = (q @ (k * (1 / math.sqrt(D))).transpose(-1, -2).contiguous()).view(hkv, g, len(rows), k1 - k0)
            if c["cap"]:
                z = torch.tanh(z.div_(c["cap"])).mul_(c["cap"])
            at_key = torch.arange(k0, k1, device=DEV)
            if c["slopes"]:
                z -= s["slopes"].view(hkv, g, 1, 1) * (pos[:, None] - at_key).abs().float()
            first = torch.zeros_like(pos)
            if s["first"] is not None:
                first = s["first"][rows].long()
            if c["window"]:
                first = torch.maximum(first, pos - c["window"] + 1)
            last = pos if s["prefix"] is None else torch.maximum(pos, s["prefix"][i].long() - 1)
            z.masked_fill_((at_key < first[:, None]) | (at_key > last[:, None]), -math.inf)
            yield i, rows, (k0, k1), z, slot
        at = end


def _prompt_plain(s):
    for i, rows, _, z, slot in _scores(s):
        v = _gather(s, "v", slot)
        m = z.amax(-1)
        z.sub_(torch.where(m == -math.inf, 0.0, m)[..., None]).exp_()
        l = z.sum(-1)
        o = (z.flatten(1, 2) @ v).view(*z.shape[:3], D) / torch.where(l == 0, 1.0, l)[..., None]
        o = o.permute(2, 0, 1, 3).flatten(1, 2)
        if "out32" in s:
            s["out32"][rows] = o
        s["out"][rows], s["m"][rows], s["l"][rows] = o.to(s["dt"]), _by_row(m), _by_row(l)


def _mass_plain(s):
    c = s["case"]
    new, kv = _lengths(c)
    hkv, page = c["hkv"], c["page"]
    sums = [torch.zeros(hkv, n, device=DEV) for n in kv]
    for i, rows, (k0, k1), z, _ in _scores(s):
        stat = lambda x: x[rows].view(len(rows), hkv, -1).permute(1, 2, 0)[..., None]  # noqa: E731
        m, l = stat(s["m"]), stat(s["l"])
        w = z.sub_(torch.where(m == -math.inf, 0.0, m)).exp_() / torch.where(l == 0, 1.0, l)
        sums[i][:, k0:k1] += w.sum((1, 2))
    for i in range(c["seqs"]):
        slot = _slots(s, i, 0, kv[i])
        if s["before"] is not None:
            sums[i] += c["decay"] * s["before"].flatten(1, 2)[:, slot]
        if "listed" in c:
            per = -(-kv[i] // page)
            on = torch.zeros(hkv, per, dtype=torch.bool, device=DEV)
            on.scatter_(1, torch.where(torch.arange(s["pages"].shape[-1], device=DEV) < s["count"][i][:, None], s["pages"][i].long(),
                                       s["pages"][i, :, :1].long()), True)
            on = on.repeat_interleave(page, 1)[:, :kv[i]]
            sums[i] = torch.where(on, sums[i], s["mass"].flatten(1, 2)[:, slot])
        s["mass"].flatten(1, 2)[:, slot] = sums[i]


def _keep_plain(s):
    c = s["case"]
    _, kv = _lengths(c)
    for i, n in enumerate(kv):
        score = s["mass"].flatten(1, 2)[:, _slots(s, i, 0, n)]
        score[:, :c["sink"]] = math.inf
        score[:, max(0, n - c["recent"]):] = math.inf
        count = min(n, c["budget"])
        # (a stable sort: ties go to the lower position)
        s["keep"][i, :, :count] = score.sort(dim=-1, descending=True, stable=True).indices[:, :count].sort(-1).values.to(torch.int32)
        s["kept"][i] = count


def _compact_plain(s):
    c = s["case"]
    _, kv = _lengths(c)
    page = c["page"]
    head = torch.arange(c["hkv"], device=DEV)[:, None]
    for i, n in enumerate(kv):
        count = min(n, c["budget"])
        src = s["keep"][i, :, :count].long()
        src = s["table"][i].long()[src // page] * page + src % page
        dst = torch.arange(count, device=DEV)
        dst = s["dst_table"][i].long()[dst // page] * page + dst % page
        for name in ("k_cache", "v_cache", "k_scale", "v_scale", "mass"):
            if name in s:
                x = s[name].view(torch.uint8) if s[name].dtype == torch.float8_e4m3fn else s[name]
                x = x.flatten(1, 2)
                x[:, dst] = x[head, src]


# ------------------------------------------------------------------------------- the framework's calls

def _held(s):
    """What a program keeps beside its inputs: the shapes and the workspace."""
    if "held" not in s:
        from paper_2606_30389_amd import _lib as L
        c = s["case"]
        kind = L.PRR_KV_E4M3 if c["kv"] == "e4m3" else L.PRR_KV_16
        dims = L.make_dims(c["hq"], c["hkv"], c["page"], s["pool"], L.PRR_BF16 if c["dtype"] == "bf16" else L.PRR_F16)
        batch = L.make_batch(c["seqs"], s["total"], s["max_new"], s["max_kv"],
                             s["cu"] if c["kind"] in ("prompt", "mass") and c["new"] > 1 else None, s["kv_len"],
                             s["table"] if c["paged"] or c["seqs"] > 1 else None, s["width"])
        shape = cap = None
        if c["kind"] in ("prompt", "decode", "mass"):
            shape = L.make_shape(c["cap"], s["slopes"], c["window"], s["prefix"], s["first"])
            cap = s["pages"].shape[-1] if "pages" in s else 0
        nbytes = {"prompt": lambda: L.prr_prompt_shaped_workspace_size(dims, batch, shape),
                  "decode": lambda: L.prr_decode_shaped_workspace_size(dims, batch, shape, kind, cap),
                  "mass": lambda: L.prr_mass_workspace_size(dims, batch, shape, kind, c["last"], cap),
                  "keep": lambda: L.prr_keep_workspace_size(dims, batch, c["budget"]),
                  "compact": lambda: L.prr_compact_workspace_size(dims, batch, kind, c["budget"], False)}[c["kind"]]()
        ws = torch.empty(nbytes, dtype=torch.uint8, device=DEV) if nbytes else None
        s["held"] = L, dims, batch, shape, kind, cap, ws, nbytes
    return s["held"]


def _run_own(s):
    L, dims, batch, shape, kind, cap, ws, nbytes = _held(s)
    c = s["case"]
    if c["kind"] == "prompt":
        L.prr_prompt_attn_shaped(dims, batch, shape, s["q"], s["k_cache"], s["v_cache"], s["out"], s["m"], s["l"], ws, nbytes)
    elif c["kind"] == "decode":
        L.prr_decode_attn_shaped(dims, batch, shape, s["q"], kind, s["k_cache"], s["v_cache"], s.get("k_scale"), s.get("v_scale"),
                                 None, None, 0, s["out32"], s["out"], s["m"], s["l"], ws, nbytes)
    elif c["kind"] == "mass":
        L.prr_key_mass(dims, batch, shape, s["q"], kind, s["k_cache"], s.get("k_scale"), s["m"], s["l"], c["last"], s.get("pages"),
                       s.get("count"), cap, s["before"], c["decay"], s["mass"], ws, nbytes)
    elif c["kind"] == "keep":
        L.prr_keep_tokens(dims, batch, s["mass"], c["budget"], c["sink"], c["recent"], s["keep"], s["kept"], ws, nbytes)
    else:
        L.prr_cache_compact(dims, batch, s["keep"], s["kept"], c["budget"], kind, s["k_cache"], s["v_cache"], s.get("k_scale"),
                            s.get("v_scale"), s["mass"], s["dst_table"], s["dst_table"].shape[-1], ws, nbytes)


def _outputs(s):
    kind = s["case"]["kind"]
    if kind == "mass":
        return {"mass": s["mass"]}
    if kind == "keep":
        return {"keep": s["keep"], "kept": s["kept"]}
    if kind == "compact":
        out = {t: s[t] for t in ("k_cache", "v_cache", "mass")}
        if s["case"]["kv"] == "e4m3":  # the codes as the numbers they are, beside their rows' powers of two
            out |= {t: s[t].view(torch.float8_e8m0fnu) for t in ("k_scale", "v_scale")}
        return out
    return {t: s[t] for t in ("out", "out32", "m", "l") if t in s}


def run(state):
    if own:
        _run_own(state)
    else:
        {"prompt": _prompt_plain, "decode": _prompt_plain, "mass": _mass_plain, "keep": _keep_plain,
         "compact": _compact_plain}[state["case"]["kind"]](state)
    return _outputs(state)


# ------------------------------------------------------------------------------- work

def work(case):
    c = case
    new, kv = _lengths(c)
    hq, hkv = c["hq"], c["hkv"]
    row = D + 1 if c["kv"] == "e4m3" else 2 * D  # bytes of a cache row
    if c["kind"] == "keep":
        return {"bytes": 4 * hkv * (sum(kv) + sum(min(n, c["budget"]) for n in kv)), "flops": 0}
    if c["kind"] == "compact":
        return {"bytes": hkv * sum(min(n, c["budget"]) for n in kv) * (4 * row + 8 + 4), "flops": 0}
    pairs, keys = _seen(c)
    t = sum(_counted(c))
    if c["kind"] == "mass":
        written = sum(kv)
        if "listed" in c:
            written = keys = sum(min(n, c["listed"] * c["page"]) for n in kv)
            pairs = keys
        return {"bytes": t * hq * (2 * D + 8) + hkv * row * keys + hkv * written * (8 if c["decay"] else 4), "flops": 2 * D * hq * pairs}
    out = 6 * D if c["kind"] == "decode" else 2 * D
    return {"bytes": t * hq * (2 * D + out + 8) + 2 * hkv * row * keys, "flops": 4 * D * hq * pairs}


# ------------------------------------------------------------------------------- in 64 bits

def _rows64(s, t, h, seq, pos):
    """Rows of the cache of KV head h at positions of a sequence, in 64 bits."""
    page = s["case"]["page"]
    phys, off = s["table"][seq].long()[pos // page], pos % page
    x = s[t + "_cache"][h]
    if x.dtype != torch.float8_e4m3fn:
        return x[phys, off].double()
    x = x.view(torch.uint8)[phys, off].view(torch.float8_e4m3fn).double()
    return x * torch.exp2(s[t + "_scale"][h][phys, off].double() - 127)[:, None]


def _weights64(s, i, h, rows, pos, n, keys):
    """Scores of the query heads of KV head h at rows (positions pos) of sequence i over keys, -inf where hidden."""
    c = s["case"]
    g = c["hq"] // c["hkv"]
    heads = slice(h * g, (h + 1) * g)
    prefix, docs = _masks(c)
    q = s["q"][rows][:, heads].double()
    z = torch.matmul(q.reshape(-1, D), _rows64(s, "k", h, i, keys).T.contiguous()).view(len(rows), g, len(keys)) / math.sqrt(D)
    if c["cap"]:
        z = c["cap"] * torch.tanh(z / c["cap"])
    if c["slopes"]:
        z = z - s["slopes"][heads].double()[:, None] * (pos[:, None, None] - keys).abs()
    lo, hi = _span(c, n, prefix[i], docs[i], pos)
    return torch.where(((keys >= lo[:, None]) & (keys < hi[:, None]))[:, None], z, -math.inf)


def _pieces(s, i, n, q, at):
    """(rows, positions, keys) of the last q of the new tokens of a sequence that end at row `at`, 512 rows at a time."""
    c = s["case"]
    prefix, docs = _masks(c)
    for r0 in range(at - q, at, 512):
        rows = torch.arange(r0, min(r0 + 512, at), device=DEV)
        pos = n - at + rows
        lo, hi = _span(c, n, prefix[i], docs[i], pos)
        yield rows, pos, torch.arange(int(lo.min()), int(hi.max()), device=DEV)


def _exact_attention(s):
    c = s["case"]
    new, kv = _lengths(c)
    g = c["hq"] // c["hkv"]
    out = {t: s[t].double().clone() for t in ("out", "m", "l")}
    at = 0
    for i in range(c["seqs"]):
        at += new[i]
        for rows, pos, keys in _pieces(s, i, kv[i], new[i], at):
            for h in range(c["hkv"]):
                heads = slice(h * g, (h + 1) * g)
                z = _weights64(s, i, h, rows, pos, kv[i], keys)
                m = z.max(-1, keepdim=True).values
                p = torch.exp(z - m)
                l = p.sum(-1)
                o = torch.matmul(p.view(-1, len(keys)), _rows64(s, "v", h, i, keys)).view(len(rows), g, D)
                out["out"][rows, heads] = o / l[..., None]
                out["m"][rows, heads], out["l"][rows, heads] = m[..., 0], l
    if "out32" in s:
        out["out32"] = out["out"]
    return out


def _exact_mass(s):
    c = s["case"]
    new, kv = _lengths(c)
    g, page = c["hq"] // c["hkv"], c["page"]
    out = s["mass"].double().clone()
    at = 0
    for i in range(c["seqs"]):
        at += new[i]
        for h in range(c["hkv"]):
            heads = slice(h * g, (h + 1) * g)
            total = torch.zeros(kv[i], dtype=torch.float64, device=DEV)
            for rows, pos, keys in _pieces(s, i, kv[i], _counted(c)[i], at):
                z = _weights64(s, i, h, rows, pos, kv[i], keys)
                m, l = s["m"][rows][:, heads, None].double(), s["l"][rows][:, heads, None].double()
                total[keys] += (torch.exp(z - m) / l).sum((0, 1))
            at_key = torch.arange(kv[i], device=DEV)
            if "listed" in c:
                on = torch.isin(at_key // page, s["pages"][i, h, :int(s["count"][i, h])].long())
                at_key, total = at_key[on], total[on]
            phys, off = s["table"][i].long()[at_key // page], at_key % page
            if s["before"] is not None:
                total = total + c["decay"] * s["before"][h, phys, off].double()
            out[h, phys, off] = total
    return {"mass": out}


def _exact_keep(s):
    c = s["case"]
    _, kv = _lengths(c)
    page = c["page"]
    keep, kept = s["keep"].cpu().clone(), s["kept"].cpu().clone()
    mass, table = s["mass"].double().cpu().numpy(), s["table"].long().cpu().numpy()
    import numpy as np
    for i, n in enumerate(kv):
        pos = np.arange(n)
        kept[i] = count = min(n, c["budget"])
        always = (pos < c["sink"]) | (pos >= n - c["recent"])
        for h in range(c["hkv"]):
            x = mass[h][table[i][pos // page], pos % page]
            order = np.lexsort((pos, -x, ~always))[:count]
            keep[i, h, :count] = torch.from_numpy(np.sort(order).astype(np.int32))
    return {"keep": keep.to(DEV), "kept": kept.to(DEV)}


def _exact_compact(s):
    c = s["case"]
    page = c["page"]
    scales = ("k_scale", "v_scale") if c["kv"] == "e4m3" else ()
    out = {t: s[t].double().clone() for t in ("k_cache", "v_cache", "mass")}
    out |= {t: torch.exp2(s[t].double() - 127) for t in scales}
    for i in range(c["seqs"]):
        count = int(s["kept"][i])
        to = torch.arange(count, device=DEV)
        to_page, to_off = s["dst_table"][i].long()[to // page], to % page
        for h in range(c["hkv"]):
            frm = s["keep"][i, h, :count].long()
            from_page, from_off = s["table"][i].long()[frm // page], frm % page
            for t in out:
                out[t][h, to_page, to_off] = out[t][h, from_page, from_off]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"prompt": _exact_attention, "decode": _exact_attention, "mass": _exact_mass, "keep": _exact_keep,
            "compact": _exact_compact}[case["kind"]](s)
