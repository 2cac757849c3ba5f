"""Shaped attention and eviction without a GPU: the keys that a token sees whatever the device arrays hold, refusals,
workspace sizes, and what the runtime checks before a launch."""
from __future__ import annotations

import ctypes
import math
import os
import shutil
import subprocess

import pytest

from tests.shape_support import Shape, keep_of

HERE = os.path.dirname(os.path.abspath(__file__))
FAKE = 0x10000  # an aligned non-null address; every case below fails validation before use


@pytest.fixture(scope="module")
def P():
    import paper_2606_30389_amd as P
    return P


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    d = tmp_path_factory.mktemp("shape_host")
    for src in (os.path.join(HERE, "..", "paper_2606_30389_amd", "csrc", "prr_shape.h"), os.path.join(HERE, "host", "shape_host.cpp")):
        shutil.copy(src, d)
    so = d / "shape_host.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-fsanitize=undefined", "-fno-sanitize-recover", "-o", str(so),
                    str(d / "shape_host.cpp")], check=True)
    return ctypes.CDLL(str(so))


INT = [-2**31, -7, -1, 0, 1, 5, 16, 99, 100, 101, 2**30, 2**31 - 1]


def test_spans_stay_in_the_sequence(host):
    import torch
    out = (ctypes.c_int32 * 2)()
    for kv in (1, 17, 100, 2**30):
        for pos in [x for x in INT if -2**24 <= x < kv] + [kv - 1]:
            for window in (0, 1, 16, 99, 2**30):
                for first in [None] + INT:
                    for prefix in [None] + INT:
                        f = None if first is None else (ctypes.c_int32 * 1)(first)
                        p = None if prefix is None else (ctypes.c_int32 * 1)(prefix)
                        host.span_host(window, p, f, pos, 0, 0, kv, out)
                        lo, hi = out
                        assert 0 <= lo <= hi <= kv
                        if kv > 100:
                            continue
                        want = Shape(window=window, first=None if first is None else [first], prefix=None if prefix is None else [prefix])
                        see = want.visible(0, torch.tensor([0]), torch.tensor([pos]), kv)[0].nonzero()[:, 0].tolist()
                        assert see == list(range(lo, hi)), (kv, pos, window, first, prefix)


def test_keep_of_small_cases():
    nan = math.nan
    assert keep_of([1.0, 3.0, 3.0, 2.0], 2, 0, 0) == [1, 2]
    assert keep_of([3.0, 3.0, 3.0, 3.0], 2, 0, 0) == [0, 1]
    assert keep_of([1.0, 3.0, 3.0, 2.0], 2, 1, 1) == [0, 3]
    assert keep_of([nan, -math.inf, nan, 0.0], 2, 0, 0) == [1, 3]
    assert keep_of([nan, 1.0], 5, 0, 0) == [0, 1]


# ------------------------------------------------------------------------------- refusals

def _expect(P, status, fn, *args, **kw):
    with pytest.raises(P.PrrError) as e:
        fn(*args, **kw)
    assert e.value.status == status, str(e.value)


def dims(P, **over):
    a = dict(num_q_heads=8, num_kv_heads=2, page_size=16, max_pages=100, dtype=P.PRR_BF16)
    a.update(over)
    return P.make_dims(**a)


def batch(P, **over):
    a = dict(n_seqs=2, total_q=10, max_q=5, max_kv=160, cu_q=FAKE, kv_len=FAKE, page_table=FAKE, table_stride=10)
    a.update(over)
    return P.make_batch(**a)


def one(P, **over):
    return batch(P, **dict(dict(cu_q=None, max_q=1), **over))


def prompt(P, d=None, b=None, shape=None, **over):
    a = dict(q=FAKE, k_cache=FAKE, v_cache=FAKE, out_o=FAKE, out_m=FAKE, out_l=FAKE, workspace=FAKE, ws_bytes=1 << 40, stream=0)
    a.update(over)
    return lambda: P.prr_prompt_attn_shaped(d or dims(P), b or batch(P), shape, **a)


def decode(P, d=None, b=None, shape=None, **over):
    a = dict(q=FAKE, kv_kind=P.PRR_KV_E4M3, k_cache=FAKE, v_cache=FAKE, k_scale=FAKE, v_scale=FAKE, pages=FAKE, page_count=FAKE, cap=4,
             out_o32=FAKE, out_o=FAKE, out_m=FAKE, out_l=FAKE, workspace=FAKE, ws_bytes=1 << 40, stream=0)
    a.update(over)
    return lambda: P.prr_decode_attn_shaped(d or dims(P), b or one(P), shape, **a)


def mass(P, d=None, b=None, shape=None, **over):
    a = dict(q=FAKE, kv_kind=P.PRR_KV_E4M3, k_cache=FAKE, k_scale=FAKE, m=FAKE, l=FAKE, last=0, pages=None, page_count=None, cap=0,
             mass_in=FAKE, decay=1.0, mass_out=FAKE, workspace=FAKE, ws_bytes=1 << 40, stream=0)
    a.update(over)
    return lambda: P.prr_key_mass(d or dims(P), b or batch(P), shape, **a)


def keep(P, d=None, b=None, **over):
    a = dict(mass=FAKE, budget=20, sink=4, recent=5, keep=FAKE, kept_len=2 * FAKE, workspace=FAKE, ws_bytes=1 << 40, stream=0)
    a.update(over)
    return lambda: P.prr_keep_tokens(d or dims(P), b or batch(P), **a)


def compact(P, d=None, b=None, **over):
    a = dict(keep=FAKE, kept_len=FAKE, budget=20, kv_kind=P.PRR_KV_E4M3, k_cache=FAKE, v_cache=FAKE, k_scale=FAKE, v_scale=FAKE, mass=FAKE,
             dst_table=None, dst_stride=0, workspace=FAKE, ws_bytes=1 << 40, stream=0)
    a.update(over)
    return lambda: P.prr_cache_compact(d or dims(P), b or batch(P), **a)


BAD_BATCH = [dict(n_seqs=0), dict(n_seqs=4097), dict(total_q=0), dict(max_q=11), dict(max_kv=-1), dict(max_kv=161), dict(kv_len=None),
             dict(cu_q=FAKE + 1), dict(page_table=FAKE + 2), dict(table_stride=0), dict(page_table=None)]


def test_batches_and_dims_are_checked(P):
    for make in (prompt, mass, keep, compact):
        for over in BAD_BATCH:
            _expect(P, P.PRR_ERR_INVALID_ARG, make(P, b=batch(P, **over)))
    for over in BAD_BATCH:
        if "max_q" not in over and "cu_q" not in over:
            _expect(P, P.PRR_ERR_INVALID_ARG, decode(P, b=one(P, **over)))
    for make in (prompt, decode, mass, keep, compact):
        for over in (dict(head_dim=64), dict(page_size=48), dict(num_q_heads=34), dict(num_kv_heads=5000, num_q_heads=5000)):
            _expect(P, P.PRR_ERR_UNSUPPORTED, make(P, d=dims(P, **over)))
        _expect(P, P.PRR_ERR_INVALID_ARG, make(P, d=dims(P, num_q_heads=7)))
    bad = batch(P, n_seqs=0)
    assert P.prr_prompt_shaped_workspace_size(dims(P), bad, None) == P.prr_mass_workspace_size(dims(P), bad, None, 0) == 0
    assert P.prr_keep_workspace_size(dims(P), bad, 5) == P.prr_compact_workspace_size(dims(P), bad, 0, 5) == 0


def test_shapes_are_checked(P):
    for over in (dict(cap=-1.0), dict(cap=math.nan), dict(cap=math.inf), dict(cap=2.0 ** -11), dict(cap=2.0 ** 21), dict(window=-1),
                 dict(window=2 ** 30 + 1), dict(slopes=FAKE + 2), dict(first=FAKE + 1), dict(prefix=FAKE + 2)):
        sh = P.make_shape(**over)
        for make in (prompt, decode, mass):
            _expect(P, P.PRR_ERR_INVALID_ARG, make(P, shape=sh))
        assert P.prr_prompt_shaped_workspace_size(dims(P), batch(P), sh) == 0


def test_attention_refusals(P):
    bad, sh = P.PRR_ERR_INVALID_ARG, P.make_shape(cap=5.0, window=7)
    for over in (dict(q=None), dict(q=FAKE + 8), dict(k_cache=None), dict(v_cache=FAKE + 2), dict(out_o=None), dict(out_m=None), dict(out_l=None)):
        _expect(P, bad, prompt(P, shape=sh, **over))
    for over in (dict(q=None), dict(kv_kind=2), dict(k_cache=None), dict(k_scale=None), dict(pages=None), dict(cap=0), dict(out_o32=None),
                 dict(out_o=FAKE + 4), dict(out_m=None)):
        _expect(P, bad, decode(P, shape=sh, **over))
    _expect(P, bad, decode(P, b=batch(P, max_q=1), shape=sh))  # cu_q


def test_windows_bound_the_workspaces(P):
    d = dims(P, max_pages=1 << 12)
    few = dict(n_seqs=1, max_kv=1 << 16, table_stride=1 << 12)
    p, t = batch(P, total_q=4, max_q=4, **few), one(P, total_q=1, **few)
    plain = P.prr_prompt_workspace_size(d, p)
    assert plain == P.prr_prompt_shaped_workspace_size(d, p, None) == P.prr_prompt_shaped_workspace_size(d, p, P.make_shape())
    whole = P.prr_prompt_shaped_workspace_size(d, p, P.make_shape(cap=5.0))
    assert 0 < P.prr_prompt_shaped_workspace_size(d, p, P.make_shape(window=5000)) < whole
    assert P.prr_prompt_shaped_workspace_size(d, p, P.make_shape(window=100)) == 0
    assert P.prr_prompt_shaped_workspace_size(d, p, P.make_shape(window=5000, prefix=FAKE)) == whole
    plain = P.prr_decode_workspace_size(d, t, 0)
    assert plain == P.prr_decode_shaped_workspace_size(d, t, None, 0) > P.prr_decode_shaped_workspace_size(d, t, P.make_shape(window=5000), 0) > 0
    sh = P.make_shape(window=5000)
    need = P.prr_prompt_shaped_workspace_size(d, p, sh)
    for over in (dict(workspace=None), dict(workspace=FAKE + 128), dict(ws_bytes=need - 1)):
        _expect(P, P.PRR_ERR_WORKSPACE, prompt(P, d=d, b=p, shape=sh, **over))


def test_mass_refusals(P):
    bad = P.PRR_ERR_INVALID_ARG
    for over in (dict(q=None), dict(q=FAKE + 8), dict(kv_kind=2), dict(kv_kind=-1), dict(k_cache=None), dict(k_cache=FAKE + 4), dict(k_scale=None),
                 dict(k_scale=FAKE + 8), dict(m=None), dict(l=FAKE + 2), dict(last=-1), dict(pages=FAKE), dict(page_count=FAKE),
                 dict(pages=FAKE, page_count=FAKE, cap=0), dict(mass_in=FAKE + 1), dict(decay=math.nan), dict(decay=math.inf), dict(mass_out=None),
                 dict(pages=FAKE, page_count=FAKE, cap=4)):  # (the last: lists with cu_q)
        _expect(P, bad, mass(P, **over))
    lists = dict(b=one(P), pages=FAKE, page_count=FAKE, cap=4)
    for over in (dict(pages=FAKE + 2), dict(page_count=FAKE + 2), dict(cap=(1 << 20) + 1), dict(cap=-1)):
        _expect(P, bad, mass(P, **dict(lists, **over)))
    d, b = dims(P), batch(P, n_seqs=1, total_q=4000, max_q=4000)
    need = P.prr_mass_workspace_size(d, b, None, P.PRR_KV_16)
    assert need > 0 and need % 256 == 0
    for over in (dict(workspace=None), dict(workspace=FAKE + 128), dict(ws_bytes=need - 1)):
        _expect(P, P.PRR_ERR_WORKSPACE, mass(P, d=d, b=b, kv_kind=P.PRR_KV_16, **over))
    mass(P, b=batch(P, max_kv=0))()  # no tokens, nothing launched


def test_keep_refusals(P):
    bad = P.PRR_ERR_INVALID_ARG
    for over in (dict(mass=None), dict(mass=FAKE + 8), dict(budget=0), dict(budget=2 ** 30 + 1), dict(sink=-1), dict(recent=-1), dict(sink=16),
                 dict(recent=2 ** 31 - 1), dict(keep=None), dict(keep=FAKE + 2), dict(kept_len=None), dict(kept_len=FAKE)):  # (kv_len)
        _expect(P, bad, keep(P, **over))
    d, b = dims(P, max_pages=1 << 13), batch(P, max_kv=100000, table_stride=1 << 13)
    need = P.prr_keep_workspace_size(d, b, 20)
    assert need > 0 and need % 256 == 0 and P.prr_keep_workspace_size(dims(P), batch(P), 20) == 0
    for over in (dict(workspace=None), dict(workspace=FAKE + 128), dict(ws_bytes=need - 1)):
        _expect(P, P.PRR_ERR_WORKSPACE, keep(P, d=d, b=b, **over))


def test_compact_refusals(P):
    bad = P.PRR_ERR_INVALID_ARG
    for over in (dict(keep=None), dict(keep=FAKE + 2), dict(kept_len=None), dict(budget=0), dict(kv_kind=3), dict(k_cache=None),
                 dict(v_cache=FAKE + 8), dict(k_scale=None), dict(v_scale=FAKE + 4), dict(mass=FAKE + 2), dict(dst_table=FAKE, dst_stride=5),
                 dict(dst_table=2 * FAKE, dst_stride=1), dict(dst_table=2 * FAKE, dst_stride=0), dict(dst_table=FAKE * 2 + 2, dst_stride=5)):
        _expect(P, bad, compact(P, **over))
    need = P.prr_compact_workspace_size(dims(P), batch(P), P.PRR_KV_E4M3, 20, True)
    assert need >= 2 * 2 * 20 * (2 * 128 + 6) and need % 256 == 0
    assert P.prr_compact_workspace_size(dims(P), batch(P), P.PRR_KV_E4M3, 20, False) == 0
    for over in (dict(workspace=None), dict(workspace=FAKE + 128), dict(ws_bytes=need - 1)):
        _expect(P, P.PRR_ERR_WORKSPACE, compact(P, **over))
    compact(P, b=batch(P, max_kv=0))()  # no tokens, nothing launched


def test_the_runtime_checks(P):
    """Wrong shapes, types, strides and devices are refused before any launch."""
    import torch
    from paper_2606_30389_amd import runtime as R
    pc = R.PathConfig(num_q_heads=4, num_kv_heads=2, page_size=16, num_tokens=64, k_select=1)
    c = R.PagedCache(pc, "cpu")
    table = torch.zeros(2, 4, dtype=torch.int32)
    q, ml = torch.zeros(5, 4, 128, dtype=torch.bfloat16), torch.zeros(5, 4)
    b, t = R.Batch("cpu", [3, 2], [3, 9], table), R.Batch("cpu", [1, 1], [3, 9], table)
    held = torch.zeros(2, 4, 16)
    f32, i32 = dict(dtype=torch.float32), dict(dtype=torch.int32)
    for sh in (R.Shape(slopes=torch.zeros(3, **f32)), R.Shape(slopes=torch.zeros(4, dtype=torch.float64)), R.Shape(slopes=torch.zeros(8, **f32)[::2]),
               R.Shape(first=torch.zeros(4, **i32)), R.Shape(first=torch.zeros(5, dtype=torch.int64)), R.Shape(prefix=torch.zeros(1, **i32)),
               R.Shape(prefix=torch.zeros(2, **i32, device="meta"))):
        for call in (lambda: c.prompt(b, q, shape=sh), lambda: c.weigh(b, q, ml, ml, shape=sh)):
            with pytest.raises(ValueError):
                call()
    with pytest.raises(ValueError):
        c.attend(t, q[:2], shape=R.Shape(slopes=torch.zeros(3)))
    lists = torch.zeros(2, 2, 3, **i32), torch.zeros(2, 2, **i32)
    for call in (lambda: c.weigh(b, q[:4], ml, ml), lambda: c.weigh(b, q, ml[:4], ml), lambda: c.weigh(b, q, ml, ml.double()),
                 lambda: c.weigh(b, q, ml, ml, before=held[:1]), lambda: c.weigh(b, q, ml, ml, out=held.double()),
                 lambda: c.weigh(b, q, ml, ml, out=torch.zeros(2, 16, 4).transpose(1, 2)),
                 lambda: c.weigh(t, q[:2], ml[:2], ml[:2], pages=lists[0][:1], counts=lists[1]),
                 lambda: c.weigh(t, q[:2], ml[:2], ml[:2], pages=lists[0]),
                 lambda: c.keep(b, held[:, :3], 5), lambda: c.keep(b, held.double(), 5), lambda: c.keep(b, held, 0),
                 lambda: c.keep(b, held, 5, out=(torch.zeros(2, 2, 4, **i32), torch.zeros(2, **i32))),
                 lambda: c.keep(b, held, 5, out=(torch.zeros(2, 2, 5, **i32), torch.zeros(1, **i32))),
                 lambda: c.compact(b, torch.zeros(2, 1, 5, **i32), torch.zeros(2, **i32)),
                 lambda: c.compact(b, torch.zeros(2, 2, 5), torch.zeros(2, **i32)),
                 lambda: c.compact(b, torch.zeros(2, 2, 5, **i32), torch.zeros(3, **i32)),
                 lambda: c.compact(b, torch.zeros(2, 2, 5, **i32), torch.zeros(2, **i32), mass=held[:1]),
                 lambda: c.compact(b, torch.zeros(2, 2, 5, **i32), torch.zeros(2, **i32), dst_table=torch.zeros(1, 4, **i32)),
                 lambda: c.keep(R.Batch("meta", [1, 1], [3, 9]), held, 5)):
        with pytest.raises(ValueError):
            call()
