"""PagedCache, Batch and LayerState on streams of their own, in graphs, and as a sequence grows."""
import math

import pytest
import torch

from tests import context_support as S

DEV = "cuda:0"


def busy(stream, ms=20):
    """Work on `stream` that takes some time."""
    with torch.cuda.stream(stream):
        x = torch.ones(4096, 4096, device=DEV)
        for _ in range(ms):
            x = x @ x * 1e-4
    return x


def layer(tokens, hq=8, hkv=2, page=16, **kw):
    from paper_2606_30389_amd import runtime as R
    return R.LayerState(R.PathConfig(num_q_heads=hq, num_kv_heads=hkv, page_size=page, num_tokens=tokens, k_select=4, **kw), DEV)


def rand(*shape, seed=0, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


@pytest.mark.gpu
def test_layer_of_fewer_tokens_than_it_was_made_for():
    """A layer made for 4096 tokens holds 1000, then 1001."""
    from paper_2606_30389_amd import runtime as R
    st, ref = layer(4096), layer(1001)
    qkv = rand(1001, 12, S.D, seed=2)
    q, k, v = qkv[:, :8], qkv[:, 8:10], qkv[:, 10:]
    stack = R.DecodeStack([st], [q[-1].contiguous()], DEV)
    stack.set_tokens(1000)
    out = st.prefill(q[:1000], k[:1000], v[:1000])
    stack.set_tokens(1001)
    st.append(q[1000:], k[1000:], v[1000:])
    ref.prefill(q, k, v)
    want = layer(1000).prefill(q[:1000], k[:1000], v[:1000])
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(out, want))
    pages = ref.k.shape[1]
    assert torch.equal(st.k[:, :pages], ref.k) and torch.equal(st.v[:, :pages], ref.v)
    assert torch.equal(st.meta[:, :pages], ref.meta)
    assert torch.all(st.k[:, pages:] == 0)


@pytest.mark.gpu
@pytest.mark.parametrize("by_address", [False, True])
def test_layer_calls_without_a_batch_on_another_stream(by_address):
    """prefill and append make their batch for the stream of the call: what the current stream allocates meanwhile does
    not get its memory."""
    n0, n = 100, 130
    st, ref = layer(n), layer(n)
    qkv = rand(n, 12, S.D, seed=1)
    q, k, v = qkv[:, :8], qkv[:, 8:10], qkv[:, 10:]
    stream = torch.cuda.Stream()
    given = stream.cuda_stream if by_address else stream
    torch.cuda.synchronize()
    held = busy(stream)
    st.cfg.num_tokens = ref.cfg.num_tokens = n0
    out = st.prefill(q[:n0], k[:n0], v[:n0], stream=given)
    scribble = [torch.full((2,), 7 + i, dtype=torch.int32, device=DEV) for i in range(64)]
    for t in range(n0, n):
        st.cfg.num_tokens = t + 1
        st.append(q[t:t + 1], k[t:t + 1], v[t:t + 1], stream=given)
        scribble.append(torch.full((1,), 3, dtype=torch.int32, device=DEV))
        scribble.append(torch.full((2,), 3, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    want = ref.prefill(q[:n0], k[:n0], v[:n0])
    ref.cfg.num_tokens = n
    ref.build_meta()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(out, want))
    assert torch.equal(st.k.flatten(1, 2)[:, :n], k.transpose(0, 1)) and torch.equal(st.v.flatten(1, 2)[:, :n], v.transpose(0, 1))
    assert torch.all(st.k.flatten(1, 2)[:, n:] == 0)
    del held


@pytest.mark.gpu
def test_two_graphs_of_one_cache_replayed_at_once():
    """Two prompts and a token's attention, each split into parts, captured on the one stream that captures use and replayed on
    streams of their own at the same time, eager calls in between."""
    from paper_2606_30389_amd import _lib as L
    from paper_2606_30389_amd import runtime as R
    tokens = 40000
    pc = R.PathConfig(num_q_heads=16, num_kv_heads=1, page_size=16, num_tokens=tokens, k_select=1)
    cache = R.PagedCache(pc, DEV)
    cache.k.copy_(rand(*cache.k.shape, seed=3))
    cache.v.copy_(rand(*cache.v.shape, seed=4))
    batches = [R.Batch(DEV, [16], [tokens]), R.Batch(DEV, [16], [tokens - 5]), R.Batch(DEV, [1], [tokens])]
    assert L.prr_prompt_workspace_size(cache.dims, batches[0].native) and L.prr_decode_workspace_size(cache.dims, batches[2].native, 0)
    qs = [rand(16, 16, S.D, seed=5), rand(16, 16, S.D, seed=6), rand(1, 16, S.D, seed=7)]
    call = [cache.prompt, cache.prompt, cache.attend]
    want = [f(b, q) for f, b, q in zip(call, batches, qs)]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for f, b, q in zip(call, batches, qs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(f(b, q))
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(20):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        got = [f(b, q) for f, b, q in zip(call, batches, qs)]
        torch.cuda.synchronize()
        for g, o, w in zip(got, outs, want):
            assert all(torch.equal(x, y) for x, y in zip(g, w)) and all(torch.equal(x, y) for x, y in zip(o, w))
            for x in o:
                x.fill_(2.0)
        torch.cuda.synchronize()


@pytest.mark.gpu
def test_workspaces_are_not_kept():
    """Calls that need ever larger workspaces, on two streams, leave nothing allocated behind."""
    from paper_2606_30389_amd import runtime as R
    pc = R.PathConfig(num_q_heads=16, num_kv_heads=1, page_size=16, num_tokens=65536, k_select=1)
    cache, other = R.PagedCache(pc, DEV), torch.cuda.Stream()
    q = rand(64, 16, S.D, seed=8)
    batches = [R.Batch(DEV, [64], [n]) for n in (4096, 16384, 65536)]
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    for b in batches:
        cache.prompt(b, q)
        cache.prompt(b, q, stream=other)
        cache.prompt(b, q, stream=other.cuda_stream)
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() == before


@pytest.mark.gpu
def test_cache_of_given_codes_and_scales():
    """An e4m3 cache made from another's codes and scales answers as that one."""
    from paper_2606_30389_amd import runtime as R
    pc = R.PathConfig(num_q_heads=8, num_kv_heads=2, page_size=16, num_tokens=320, k_select=1)
    one = R.PagedCache(pc, DEV, kind="e4m3")
    one.append(R.Batch(DEV, [300], [300]), None, 5 * rand(300, 2, S.D, seed=9), 0.1 * rand(300, 2, S.D, seed=10))
    two = R.PagedCache(pc, DEV, kind="e4m3", k=one.k, v=one.v, k_scale=one.k_scale, v_scale=one.v_scale)
    b, q = R.Batch(DEV, [1], [300]), rand(1, 8, S.D, seed=11)
    got, want = two.attend(b, q), one.attend(b, q)
    torch.cuda.synchronize()
    assert one.k_scale[:, :18].unique().numel() > 1
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert all(torch.equal(x, y) for x, y in zip(two.read(300), one.read(300)))


@pytest.mark.gpu
@pytest.mark.parametrize("n,new,rows", [(40, 40, 64), (200, 3, 512), (33, 0, 5)])
def test_prefill_with_rows_behind_the_sequence(n, new, rows):
    """A given batch with more rows than tokens: the tokens are served, the rows behind them are left, and the metadata is that of
    the whole context."""
    from paper_2606_30389_amd import runtime as R
    st, ref = layer(n), layer(n)
    for x in (st, ref):
        x.k.copy_(rand(*x.k.shape, seed=12))
        x.v.copy_(rand(*x.v.shape, seed=13))
        x.build_meta()
    q, k, v = rand(rows, 8, S.D, seed=14), rand(rows, 2, S.D, seed=15), rand(rows, 2, S.D, seed=16)
    out = st.prefill(q, k, v, batch=R.Batch(DEV, [new], [n], total_q=rows))
    torch.cuda.synchronize()
    for x in out:
        assert torch.all(x[new:] == 0)
    if new:
        want = ref.prefill(q[:new].contiguous(), k[:new], v[:new])
        torch.cuda.synchronize()
        assert all(torch.equal(x[:new], y) for x, y in zip(out, want))
    assert torch.equal(st.k, ref.k) and torch.equal(st.meta, ref.meta)


@pytest.mark.gpu
def test_layers_serve_one_sequence():
    from paper_2606_30389_amd import runtime as R
    st = layer(64)
    before = st.k.clone()
    table = torch.arange(8, dtype=torch.int32, device=DEV).view(2, 4) % 4
    two = R.Batch(DEV, [1, 1], [30, 20], table)
    q, k = rand(2, 8, S.D), rand(2, 2, S.D)
    for call in (lambda: st.prefill(q, k, k, batch=two), lambda: st.append(q, k, k, batch=two)):
        with pytest.raises(ValueError):
            call()
    torch.cuda.synchronize()
    assert torch.equal(st.k, before)


@pytest.mark.gpu
@pytest.mark.parametrize("schedule", ["serial", "fused"])
def test_a_layer_grows_to_its_pages(schedule):
    """A layer of 20 tokens with room for 512, a budget of 8 pages: appended and stepped until it has 300, the step attends
    what is selected."""
    import paper_2606_30389_amd as P
    from paper_2606_30389_amd import runtime as R
    n0, n, hq, hkv = 20, 300, 8, 2
    pc = R.PathConfig(num_q_heads=hq, num_kv_heads=hkv, page_size=16, num_tokens=n0, k_select=8, max_pages=32)
    st = R.LayerState(pc, DEV)
    qbuf = torch.empty(1, hq, S.D, dtype=torch.bfloat16, device=DEV)
    stack = R.DecodeStack([st], [qbuf], DEV)
    qkv = rand(n, hq + 2 * hkv, S.D, seed=17)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    st.prefill(q[:n0], k[:n0], v[:n0])
    one = R.Batch(DEV, [1], [n0], max_kv=512)
    s = torch.cuda.current_stream()
    for t in range(n0, n):
        stack.set_tokens(t + 1)
        one.advance()
        st.append(q[t:t + 1], k[t:t + 1], v[t:t + 1], batch=one, q_out=qbuf)
        if schedule == "serial":
            stack.step(P.PRR_SCHED_FUSED_SERIAL, s)
        else:
            stack.step(P.PRR_SCHED_FUSED_PREFILL if t == n0 else P.PRR_SCHED_FUSED_PRR, s)
            if t == n0:
                continue
        if t % 29 and t != n - 1:
            continue
        torch.cuda.synchronize()
        assert st.sel_count.tolist() == [min(8, -(-(t + 1) // 16))] * hkv
        listed = st.cache().attend(one, qbuf, st.sel[None].contiguous(), st.sel_count[None].contiguous())
        torch.cuda.synchronize()
        # the same keys in float32, by two kernels: 2^-15 of the values' size
        assert (st.out_o32 - listed[0][0]).abs().max() <= 2.0 ** -15 * v.abs().max()
        assert torch.allclose(st.out_m, listed[2][0], rtol=1e-5, atol=1e-5)
    with pytest.raises(ValueError):
        stack.set_tokens(513)
    assert pc.num_tokens == n


@pytest.mark.gpu
def test_captured_layer_calls_need_a_batch():
    """Without one they are refused, and the capture goes on; with one, the replays follow the batch's lengths."""
    from paper_2606_30389_amd import runtime as R
    st = layer(64)
    q, k = rand(1, 8, S.D, seed=18), rand(1, 2, S.D, seed=19)
    one, qbuf = R.Batch(DEV, [1], [60], max_kv=64), torch.empty_like(q)
    out = [torch.empty(1, 8, S.D, device=DEV), None, torch.empty(1, 8, device=DEV), torch.empty(1, 8, device=DEV)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(ValueError):
            st.append(q, k, k)
        one.advance()
        st.append(q, k, k, batch=one, q_out=qbuf)
        st.cache().attend(one, qbuf, out=out)
    for t in range(61, 65):
        graph.replay()
        torch.cuda.synchronize()
        assert int(one.kv_len) == t
        filled = st.k.flatten(1, 2)[:, 60:].ne(0).any(-1)
        assert torch.all(filled[:, :t - 60]) and not filled[:, t - 60:].any()
        want = st.cache().attend(R.Batch(DEV, [1], [t], max_kv=64), qbuf)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip([out[0], *out[2:]], [want[0], *want[2:]]))


@pytest.mark.gpu
def test_the_default_stream_by_its_address():
    """Calls of several parts on stream 0, given as a number, as a stream and not at all, from another current stream too."""
    from paper_2606_30389_amd import runtime as R
    pc = R.PathConfig(num_q_heads=16, num_kv_heads=1, page_size=16, num_tokens=20000, k_select=1)
    cache = R.PagedCache(pc, DEV, k=rand(1, 1250, 16, S.D, seed=20), v=rand(1, 1250, 16, S.D, seed=21))
    q, b, one = rand(8, 16, S.D, seed=22), R.Batch(DEV, [8], [20000]), R.Batch(DEV, [1], [20000])
    want = cache.prompt(b, q), cache.attend(one, q[:1])
    default, other = torch.cuda.default_stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for current in (default, other):
        for given in (None, 0, default, other, other.cuda_stream):
            with torch.cuda.stream(current):
                got = cache.prompt(b, q, stream=given), cache.attend(one, q[:1], stream=given)
                assert torch.cuda.current_stream() == current
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for g, w in zip(got, want) for x, y in zip(g, w))
