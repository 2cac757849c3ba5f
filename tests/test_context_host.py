"""The calls around the decode step without a GPU: refusals, rotary frequencies, workspace sizes, and what
the device reads of a batch whose arrays hold anything."""
from __future__ import annotations

import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
FAKE = 0x10000  # an aligned non-null address; every case below fails validation before use


@pytest.fixture(scope="module")
def P():
    import paper_2606_30389_amd as P
    return P


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    d = tmp_path_factory.mktemp("batch_host")
    for src in (os.path.join(HERE, "..", "paper_2606_30389_amd", "csrc", "prr_batch.h"), os.path.join(HERE, "host", "batch_host.cpp")):
        shutil.copy(src, d)
    so = d / "batch_host.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-fsanitize=undefined", "-fno-sanitize-recover", "-o", str(so),
                    str(d / "batch_host.cpp")], check=True)
    return ctypes.CDLL(str(so))


INT = [-2**31, -7, -1, 0, 1, 5, 16, 17, 100, 2**30, 2**31 - 1]


def test_rows_of_a_sequence_stay_in_the_batch(host):
    out = (ctypes.c_int32 * 3)()
    for total, max_q, max_kv in ((17, 5, 100), (1, 0, 0), (2**24, 2**24, 2**30)):
        for a in INT:
            for b in INT:
                cu = (ctypes.c_int32 * 2)(a, b)
                kv = (ctypes.c_int32 * 1)(b)
                host.seq_host(cu, kv, 1, total, max_q, max_kv, 0, out)
                q0, q1, n = out
                assert 0 <= q0 <= q1 <= total and q1 - q0 <= max_q and 0 <= n <= max_kv
                if 0 <= a <= b <= total and b - a <= max_q:
                    assert (q0, q1) == (a, b)
                if 0 <= b <= max_kv:
                    assert n == b
    kv = (ctypes.c_int32 * 3)(4, 5, 6)
    host.seq_host(None, kv, 3, 3, 1, 10, 2, out)
    assert list(out) == [2, 3, 6]


def test_pages_stay_in_the_pool(host):
    table = np.array([[3, -1, 9, 2**30], [10, 0, -2**31, 2**31 - 1]], dtype=np.int32)
    for s in range(2):
        for lp in INT + [2, 3, 4]:
            p = host.page_host(ctypes.c_void_p(table.ctypes.data), 4, 10, s, lp)
            want = int(table[s, lp]) if 0 <= lp < 4 else -1
            assert p == (want if 0 <= want < 10 else -1)
            assert host.page_host(None, 0, 10, 0, lp) == (lp if 0 <= lp < 10 else -1)


# ------------------------------------------------------------------------------- refusals

def _expect(P, status, fn, *args, **kw):
    with pytest.raises(P.PrrError) as e:
        fn(*args, **kw)
    assert e.value.status == status, str(e.value)
    return str(e.value)


def dims(P, **over):
    a = dict(num_q_heads=8, num_kv_heads=2, page_size=16, max_pages=100, dtype=P.PRR_BF16)
    a.update(over)
    return P.make_dims(**a)


def batch(P, **over):
    a = dict(n_seqs=2, total_q=10, max_q=5, max_kv=160, cu_q=FAKE, kv_len=FAKE, page_table=FAKE, table_stride=10)
    a.update(over)
    return P.make_batch(**a)


BAD_BATCH = [dict(n_seqs=0), dict(n_seqs=4097), dict(total_q=0), dict(total_q=(1 << 24) + 1), dict(max_q=-1), dict(max_q=11),
             dict(max_kv=-1), dict(max_kv=161), dict(max_kv=(1 << 30) + 1, table_stride=1 << 30), dict(kv_len=None), dict(kv_len=FAKE + 2),
             dict(cu_q=FAKE + 1), dict(page_table=FAKE + 2), dict(table_stride=0), dict(page_table=None),
             dict(page_table=None, n_seqs=1, max_kv=1601), dict(cu_q=None, total_q=1, max_q=1), dict(cu_q=None, max_q=0)]


def rope(P, d=None, b=None, **over):
    a = dict(q=FAKE, k=FAKE, v=FAKE, positions=None, freqs=FAKE, rot_dim=128, layout=P.PRR_ROPE_HALF, rope_scale=1.0, q_out=FAKE * 2,
             kv_kind=P.PRR_KV_E4M3, k_cache=FAKE, v_cache=FAKE, k_scale=FAKE, v_scale=FAKE, stream=0)
    a.update(over)
    return lambda: P.prr_rope_append(d or dims(P), b or batch(P), **a)


def prompt(P, d=None, b=None, **over):
    a = dict(q=FAKE, k_cache=FAKE, v_cache=FAKE, out_o=FAKE, out_m=FAKE, out_l=FAKE, workspace=FAKE, ws_bytes=1 << 40, stream=0)
    a.update(over)
    return lambda: P.prr_prompt_attn(d or dims(P), b or batch(P), **a)


def decode(P, d=None, b=None, **over):
    a = dict(q=FAKE, kv_kind=P.PRR_KV_E4M3, k_cache=FAKE, v_cache=FAKE, k_scale=FAKE, v_scale=FAKE, pages=FAKE, page_count=FAKE, cap=4,
             out_o32=FAKE, out_o=FAKE, out_m=FAKE, out_l=FAKE, workspace=FAKE, ws_bytes=1 << 40, stream=0)
    a.update(over)
    return lambda: P.prr_decode_attn(d or dims(P), b or batch(P, cu_q=None, max_q=1), **a)


def read(P, d=None, **over):
    a = dict(k_codes=FAKE, v_codes=FAKE, k_scale=FAKE, v_scale=FAKE, page_table=None, num_tokens=100, page_begin=0, page_end=7,
             k_out=FAKE, v_out=FAKE, stream=0)
    a.update(over)
    return lambda: P.prr_cache_read(d or dims(P), **a)


def test_batches_are_checked(P):
    for over in BAD_BATCH:
        _expect(P, P.PRR_ERR_INVALID_ARG, rope(P, b=batch(P, **over)))
        _expect(P, P.PRR_ERR_INVALID_ARG, prompt(P, b=batch(P, **over)))
        assert P.prr_prompt_workspace_size(dims(P), batch(P, **over)) == 0
        one = dict(dict(cu_q=None, max_q=1), **{k: v for k, v in over.items() if k != "max_q" or v < 1})
        if "cu_q" in over and over["cu_q"]:
            one["cu_q"] = over["cu_q"]
        if over != dict(max_q=11):
            _expect(P, P.PRR_ERR_INVALID_ARG, decode(P, b=batch(P, **one)))
    for make in (rope, prompt, decode):
        _expect(P, P.PRR_ERR_UNSUPPORTED, make(P, d=dims(P, head_dim=64)))
        _expect(P, P.PRR_ERR_UNSUPPORTED, make(P, d=dims(P, page_size=48)))
        _expect(P, P.PRR_ERR_UNSUPPORTED, make(P, d=dims(P, num_q_heads=34)))
        _expect(P, P.PRR_ERR_INVALID_ARG, make(P, d=dims(P, num_q_heads=7)))
        _expect(P, P.PRR_ERR_UNSUPPORTED, make(P, d=dims(P, num_kv_heads=5000, num_q_heads=5000)))
    _expect(P, P.PRR_ERR_UNSUPPORTED, read(P, d=dims(P, head_dim=64)))


def test_rope_append_refusals(P):
    bad = P.PRR_ERR_INVALID_ARG
    for over in (dict(q=None, k=None, v=None, q_out=None), dict(k=None), dict(v=None), dict(q=None), dict(q_out=None), dict(q=FAKE + 4),
                 dict(k=FAKE + 4), dict(v=FAKE + 4), dict(q_out=FAKE + 4), dict(rot_dim=-8), dict(rot_dim=136), dict(freqs=None),
                 dict(freqs=FAKE + 4), dict(positions=FAKE + 2), dict(layout=2), dict(rope_scale=math.inf), dict(rope_scale=math.nan),
                 dict(kv_kind=2), dict(k_cache=None), dict(v_cache=None), dict(k_cache=FAKE + 8), dict(k_scale=None), dict(v_scale=None),
                 dict(k_scale=FAKE + 4)):
        _expect(P, bad, rope(P, **over))
    _expect(P, P.PRR_ERR_UNSUPPORTED, rope(P, rot_dim=100))
    d, b = dims(P), batch(P)
    raw = lambda qs, ks, vs, out=FAKE * 2: P._lib._lib.prr_rope_append(  # noqa: E731
        ctypes.byref(d), ctypes.byref(b), FAKE, FAKE, FAKE, qs, ks, vs, None, FAKE, 128, 0, 1.0, out, 0, FAKE, FAKE, None, None, None)
    assert raw(-1024, 256, 256) == bad and raw(1026, 256, 256) == bad and raw(1024, 255, 256) == bad and raw(1024, 256, -4) == bad
    assert raw(2048, 256, 256, FAKE) == bad  # in place, but not dense
    import torch
    x = torch.zeros(10, 8, 128, dtype=torch.bfloat16)
    for wrong in (x[:, :4], x[..., ::2], x.transpose(0, 1), x[0]):
        with pytest.raises(ValueError):
            rope(P, q=wrong)()


def test_prompt_refusals(P):
    bad = P.PRR_ERR_INVALID_ARG
    for over in (dict(q=None), dict(q=FAKE + 8), dict(k_cache=None), dict(v_cache=FAKE + 2), dict(out_o=None), dict(out_m=None),
                 dict(out_l=None), dict(out_l=FAKE + 2)):
        _expect(P, bad, prompt(P, **over))
    d, b = dims(P, max_pages=1 << 12), batch(P, n_seqs=1, total_q=4, max_q=4, max_kv=1 << 16, table_stride=1 << 12)
    need = P.prr_prompt_workspace_size(d, b)
    assert need > 0 and need % 256 == 0
    for over in (dict(workspace=None), dict(workspace=FAKE + 128), dict(ws_bytes=need - 1)):
        _expect(P, P.PRR_ERR_WORKSPACE, prompt(P, d=d, b=b, **over))


def test_decode_refusals(P):
    bad = P.PRR_ERR_INVALID_ARG
    for over in (dict(q=None), dict(q=FAKE + 8), dict(kv_kind=-1), dict(k_cache=None), dict(v_cache=FAKE + 2), dict(k_scale=None),
                 dict(v_scale=FAKE + 4), dict(pages=None), dict(page_count=None), dict(pages=FAKE + 2), dict(cap=0), dict(cap=-1),
                 dict(cap=(1 << 20) + 1), dict(out_o32=None), dict(out_o32=FAKE + 8), dict(out_o=FAKE + 4), dict(out_m=None), dict(out_l=None)):
        _expect(P, bad, decode(P, **over))
    _expect(P, bad, decode(P, b=batch(P, max_q=1)))  # cu_q
    d, b = dims(P, max_pages=1 << 12), batch(P, n_seqs=1, total_q=1, max_q=1, cu_q=None, max_kv=1 << 16, table_stride=1 << 12)
    need = P.prr_decode_workspace_size(d, b, P.PRR_KV_16)
    assert need > 0 and need % 256 == 0
    for over in (dict(workspace=None), dict(workspace=FAKE + 128), dict(ws_bytes=need - 1)):
        _expect(P, P.PRR_ERR_WORKSPACE, decode(P, d=d, b=b, pages=None, page_count=None, cap=0, kv_kind=P.PRR_KV_16, **over))


def test_cache_read_refusals(P):
    for over in (dict(k_codes=None), dict(v_codes=FAKE + 8), dict(k_scale=None), dict(v_scale=FAKE + 4), dict(k_out=None),
                 dict(v_out=FAKE + 8), dict(page_table=FAKE + 2), dict(num_tokens=0), dict(num_tokens=1601), dict(page_begin=-1),
                 dict(page_begin=5, page_end=4), dict(page_end=8), dict(num_tokens=(1 << 30) + 1, page_table=FAKE)):
        _expect(P, P.PRR_ERR_INVALID_ARG, read(P, **over))
    read(P, page_begin=3, page_end=3)()  # nothing to read, nothing launched


def test_no_new_tokens_is_no_work(P):
    prompt(P, b=batch(P, max_q=0))()
    rope(P, b=batch(P, max_q=0))()


def test_workspaces_follow_the_rows_that_can_be_live(P):
    d = dims(P, max_pages=1 << 12)
    few = dict(n_seqs=1, max_q=4, max_kv=1 << 16, table_stride=1 << 12)
    assert P.prr_prompt_workspace_size(d, batch(P, total_q=4, **few)) == P.prr_prompt_workspace_size(d, batch(P, total_q=1 << 24, **few))
    _expect(P, P.PRR_ERR_UNSUPPORTED, prompt(P, d=dims(P, num_q_heads=256, num_kv_heads=256),
                                             b=batch(P, n_seqs=4096, total_q=1 << 24, max_q=1 << 20, table_stride=1 << 12)))


def test_batches_of_the_runtime_are_checked():
    from paper_2606_30389_amd import runtime as R
    for new, kv in (([1], [1, 2]), ([], []), ([-1], [4]), ([1], [-4])):
        with pytest.raises(ValueError):
            R.Batch("cpu", new, kv)
    b = R.Batch("cpu", [1, 1], [3, 4], max_kv=5)
    assert b.cu_q is None and b.total_q == 2 and b.native.max_kv == 5
    b.advance()
    with pytest.raises(ValueError):
        b.advance()
    assert b.kv_len.tolist() == [4, 5]
    for kv in ([1], [1, 6], [-1, 2]):
        with pytest.raises(ValueError):
            b.set_lengths(kv)
    b.set_lengths([0, 1])
    b.advance()
    assert b.kv_len.tolist() == [1, 2]
    p = R.Batch("cpu", [3, 0, 2], [3, 5, 9])
    assert p.cu_q.tolist() == [0, 3, 3, 5] and p.native.max_q == 3 and p.native.total_q == 5


def test_tensors_of_the_runtime_are_checked():
    """Wrong shapes, types and strides are refused before any launch."""
    import torch
    from paper_2606_30389_amd import runtime as R
    pc = R.PathConfig(num_q_heads=4, num_kv_heads=2, page_size=16, num_tokens=64, k_select=1)
    c = R.PagedCache(pc, "cpu")
    q, k = torch.zeros(5, 4, 128, dtype=torch.bfloat16), torch.zeros(5, 2, 128, dtype=torch.bfloat16)
    table = torch.zeros(2, 4, dtype=torch.int32)
    b = R.Batch("cpu", [3, 2], [3, 9], table)
    for bad in (q[:4], q.half(), q[:, :2], q[..., :64], q.view(5, 512)):
        for call in (lambda: c.append(b, bad, k, k), lambda: c.prompt(b, bad), lambda: c.append(b, q, k, k, q_out=bad)):
            with pytest.raises(ValueError):
                call()
    for bad in (k[:4], k.float(), q):
        with pytest.raises(ValueError):
            c.append(b, q, bad, k)
        with pytest.raises(ValueError):
            c.append(b, q, k, bad)
    with pytest.raises(ValueError):
        c.append(b, q, k, k, positions=torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError):
        c.prompt(b, torch.zeros(5, 8, 128, dtype=torch.bfloat16)[:, ::2])
    one = R.Batch("cpu", [1, 1], [3, 9], table)
    for pages, counts in ((torch.zeros(2, 2, 3), torch.zeros(2, 2, dtype=torch.int32)),
                          (torch.zeros(1, 2, 3, dtype=torch.int32), torch.zeros(2, 2, dtype=torch.int32)),
                          (torch.zeros(2, 2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))):
        with pytest.raises(ValueError):
            c.attend(one, q[:2], pages, counts)
    for bad in (table[:1], table.long(), torch.zeros(4, 2, dtype=torch.int32).T):
        with pytest.raises(ValueError):
            R.Batch("cpu", [1, 1], [3, 9], bad)
    with pytest.raises(ValueError):
        R.PagedCache(pc, "cpu", kind="e4m3").prompt(b, q)
    with pytest.raises(ValueError):
        R.PagedCache(pc, "cpu", kind="e4m3").read(64, table[0][:3])
    with pytest.raises(ValueError):
        R.PagedCache(pc, "cpu", k=torch.zeros(2, 3, 16, 128, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        R.PagedCache(pc, "cpu", k=torch.zeros(2, 4, 16, 128, dtype=torch.float16))


def test_outputs_and_devices_of_the_runtime_are_checked():
    """Outputs that are given have the size of what is written; nothing lies on another device."""
    import torch
    from paper_2606_30389_amd import runtime as R
    pc = R.PathConfig(num_q_heads=4, num_kv_heads=2, page_size=16, num_tokens=64, k_select=1)
    c, e = R.PagedCache(pc, "cpu"), R.PagedCache(pc, "cpu", kind="e4m3")
    q, ml = torch.zeros(2, 4, 128, dtype=torch.bfloat16), torch.zeros(2, 4)
    b, elsewhere = R.Batch("cpu", [1, 1], [3, 9]), R.Batch("meta", [1, 1], [3, 9])
    for out in ((q[:1], ml, ml), (q.float(), ml, ml), (q, ml[:1], ml), (q, ml, ml.double()), (q, ml), (None, ml, ml)):
        with pytest.raises(ValueError):
            c.prompt(b, q, out=out)
    for out in ((q, q, ml, ml), (q.float(), q.float(), ml, ml), (q.float(), q, ml[:, :2], ml), (q.float(), q, ml, ml[:1]),
                (q.float()[:1], None, ml, ml), (q.float(), q, ml), (None, q, ml, ml), (q.float(), q, None, ml)):
        with pytest.raises(ValueError):
            c.attend(b, q, out=out)
    for call in (lambda: c.prompt(elsewhere, q), lambda: c.attend(elsewhere, q), lambda: c.append(elsewhere, None, q[:, :2], q[:, :2]),
                 lambda: c.attend(b, q.to("meta")), lambda: c.append(b, q, q[:, :2], q[:, :2], R.Rope("meta")),
                 lambda: R.Batch("cpu", [1], [3], torch.zeros(1, 4, dtype=torch.int32, device="meta"))):
        with pytest.raises(ValueError):
            call()
    pages = torch.zeros(2, 4, 16, 128, dtype=torch.bfloat16)
    for out in ((pages[:, :3], pages), (pages, pages.float()), (pages,), (pages, pages.to("meta"))):
        with pytest.raises(ValueError):
            e.read(64, out=out)
    for args in (dict(page_begin=3, page_end=2), dict(page_begin=-1), dict(page_table=torch.zeros(4, dtype=torch.int64)),
                 dict(page_table=torch.zeros(8, dtype=torch.int32)[::2])):
        with pytest.raises(ValueError):
            e.read(64, **args)


# ------------------------------------------------------------------------------- frequencies

@pytest.mark.parametrize("rot", [4, 64, 96, 128])
@pytest.mark.parametrize("base", [10000.0, 500000.0])
def test_rope_freqs(P, rot, base):
    i = np.arange(rot // 2)
    w = base ** (-2.0 * i / rot)
    f, L, lo, hi = 8.0, 8192, 1.0, 32.0
    got, s = P.prr_rope_freqs(P.PRR_ROPE_PLAIN, rot, base)
    np.testing.assert_allclose(got, w, rtol=1e-14)
    assert s == 1.0
    got, s = P.prr_rope_freqs(P.PRR_ROPE_LINEAR, rot, base, f)
    np.testing.assert_allclose(got, w / f, rtol=1e-14)
    got, s = P.prr_rope_freqs(P.PRR_ROPE_NTK, rot, base, f)
    np.testing.assert_allclose(got, (base * f ** (rot / (rot - 2))) ** (-2.0 * i / rot), rtol=1e-13)
    # the slowest pair is interpolated by exactly f, the fastest not at all
    assert got[0] == 1.0 and abs(got[-1] * f / w[-1] - 1) < 1e-12
    got, s = P.prr_rope_freqs(P.PRR_ROPE_BY_PARTS, rot, base, f, L, lo, hi)
    turns = L * w / (2 * math.pi)
    g = np.clip((turns - lo) / (hi - lo), 0, 1)
    np.testing.assert_allclose(got, g * w + (1 - g) * w / f, rtol=1e-13)
    assert np.allclose(got[turns >= hi], w[turns >= hi], rtol=1e-15) and np.allclose(got[turns <= lo] * f, w[turns <= lo], rtol=1e-15)
    assert s == 1.0
    got, s = P.prr_rope_freqs(P.PRR_ROPE_YARN, rot, base, f, L, lo, hi)
    at = lambda r: rot * math.log(L / (r * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
    a, b = max(math.floor(at(hi)), 0), min(math.ceil(at(lo)), rot - 1)
    g = 1 - np.clip((i - a) / max(b - a, 1e-3), 0, 1)
    np.testing.assert_allclose(got, g * w + (1 - g) * w / f, rtol=1e-13)
    assert abs(s - (0.1 * math.log(f) + 1)) < 1e-7
    # a factor of one changes nothing
    for kind in (P.PRR_ROPE_LINEAR, P.PRR_ROPE_NTK, P.PRR_ROPE_BY_PARTS, P.PRR_ROPE_YARN):
        got, s = P.prr_rope_freqs(kind, rot, base, 1.0, L, lo, hi)
        np.testing.assert_allclose(got, w, rtol=1e-14)
        assert s == 1.0


def test_rope_freqs_refusals(P):
    ok = dict(kind=P.PRR_ROPE_YARN, rot_dim=64, base=10000.0, factor=2.0, trained_len=4096, lo=1.0, hi=32.0)
    P.prr_rope_freqs(**ok)
    for over in (dict(kind=5), dict(kind=-1), dict(rot_dim=0), dict(rot_dim=63), dict(rot_dim=130), dict(base=1.0), dict(base=math.inf),
                 dict(base=math.nan), dict(factor=0.5), dict(factor=math.nan), dict(trained_len=0), dict(lo=0.0), dict(lo=32.0),
                 dict(hi=math.inf), dict(kind=P.PRR_ROPE_NTK, rot_dim=2)):
        _expect(P, P.PRR_ERR_INVALID_ARG, P.prr_rope_freqs, **dict(ok, **over))
