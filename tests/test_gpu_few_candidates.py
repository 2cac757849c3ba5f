"""The fused step with small budgets: now and then exactly as many pages reach the bound of the step before as are selected."""
import numpy as np
import pytest
import torch

import oracle as O

DEV = "cuda:0"


@pytest.mark.gpu
@pytest.mark.parametrize("late", [0, 1, 2])
@pytest.mark.parametrize("k,page,chunk", [(1, 16, 8), (2, 16, 2), (5, 64, 2), (8, 16, 8), (20, 16, 4)])
def test_exact_output_of_many_steps(k, page, chunk, late):
    """Attention over exactly the selected pages, 250 random queries of four KV heads, whatever was speculated."""
    import paper_2606_30389_amd as P
    from paper_2606_30389_amd import runtime as R
    hq, hkv, pages, steps = 8, 4, 60, 250
    n = pages * page - 3
    g = torch.Generator(device=DEV).manual_seed(k)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV).to(torch.bfloat16)  # noqa: E731
    cfg = R.PathConfig(num_q_heads=hq, num_kv_heads=hkv, page_size=page, num_tokens=n, k_select=k, chunk_pages=chunk)
    st = R.LayerState(cfg, DEV, k=rand(hkv, pages, page, 128), v=rand(hkv, pages, page, 128))
    st.build_meta()
    qbuf = rand(1, hq, 128)
    stack = R.DecodeStack([st], [qbuf], DEV)
    stack.params.late_spec = late
    s = torch.cuda.current_stream()
    stack.step(P.PRR_SCHED_FUSED_PREFILL, s)
    outs, queries, hits = [], rand(steps, 1, hq, 128), 0
    for i in range(steps):
        qbuf.copy_(queries[i])
        stack.step(P.PRR_SCHED_FUSED_PRR, s)
        outs.append((st.out_o32.clone(), st.sel.clone(), st.sel_count.clone()))
        hits += (k - st.missed).sum()
    torch.cuda.synchronize()
    assert int(hits) > 0  # (some of what was speculated is used)
    k64, v64 = (x.double().cpu().numpy() for x in (st.k, st.v))
    meta = O.page_metadata_minmax(k64, page, n)
    for i, (o, sel, count) in enumerate(outs):
        _, want, (o64, _, _) = O.serial_step(queries[i, 0].double().cpu().numpy(), k64, v64, page, n, k, meta=meta)
        for h in range(hkv):
            assert np.array_equal(np.sort(sel[h, :int(count[h])].cpu().numpy()), want[h]), (i, h)
        e = np.abs(o.cpu().numpy() - o64).max(1)
        assert e.max() < 1e-4, (i, e)
