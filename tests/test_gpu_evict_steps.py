"""A layer that evicts, and goes on in each of the decode step's schedules."""
import numpy as np
import pytest
import torch

import oracle as O
from tests import context_support as S

DEV = "cuda:0"


def rand(*shape, seed=0, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("schedule", ["SERIAL", "TWO_STREAM", "FUSED_SERIAL", "FUSED_PRR"])
def test_steps_after_an_eviction(schedule):
    """Prefill, steps, eviction, steps over the smaller cache (its predictions begin empty), another eviction, steps: each
    step's output as 64 bits give it for the pages of the largest scores."""
    import paper_2606_30389_amd as P
    from paper_2606_30389_amd import runtime as R
    n, hq, hkv, page, k = 900, 8, 2, 16, 8
    cfg = R.PathConfig(num_q_heads=hq, num_kv_heads=hkv, page_size=page, num_tokens=n, k_select=k, max_pages=64)
    st = R.LayerState(cfg, DEV)
    qbuf = torch.zeros(1, hq, S.D, dtype=torch.bfloat16, device=DEV)
    stack = R.DecodeStack([st], [qbuf], DEV)
    rope = R.Rope(DEV)
    kind = getattr(P, "PRR_SCHED_" + schedule)
    torch.cuda.synchronize()
    s, p = torch.cuda.Stream(), torch.cuda.Stream()
    true, seed = 0, 0

    def prefill(count):
        nonlocal true, seed
        q_rot = torch.zeros(count, hq, S.D, dtype=torch.bfloat16, device=DEV)
        pos = torch.arange(true, true + count, dtype=torch.int32, device=DEV)
        _, m, l = st.prefill(rand(count, hq, S.D, seed=seed), rand(count, hkv, S.D, seed=seed + 1), rand(count, hkv, S.D, seed=seed + 2),
                             rope, positions=pos, q_out=q_rot)
        true, seed = true + count, seed + 3
        return q_rot, m, l

    def steps(count):
        nonlocal true, seed
        for _ in range(count):
            stack.set_tokens(st.cfg.num_tokens + 1)
            st.append(rand(1, hq, S.D, seed=seed), rand(1, hkv, S.D, seed=seed + 1), rand(1, hkv, S.D, seed=seed + 2), rope, q_out=qbuf,
                      positions=torch.tensor([true], dtype=torch.int32, device=DEV))
            true, seed = true + 1, seed + 3
            stack.step(kind, s, p if schedule == "TWO_STREAM" else None)
            torch.cuda.synchronize()
            t = st.cfg.num_tokens
            pages = -(-t // page)
            k64, v64 = (x[:, :pages].double().cpu().numpy() for x in (st.k, st.v))
            _, sel, (o64, _, _) = O.serial_step(qbuf[0].double().cpu().numpy(), k64, v64, page, t, k)
            for h in range(hkv):
                assert np.array_equal(np.sort(st.sel.cpu().numpy()[h, :int(st.sel_count[h])]), sel[h])
            assert np.abs(st.out_o32.cpu().numpy() - o64).max() < 1e-4

    with torch.cuda.stream(s):
        stats = prefill(n)
        if schedule in ("TWO_STREAM", "FUSED_PRR"):
            stack.step(P.PRR_SCHED_PREFILL if schedule == "TWO_STREAM" else P.PRR_SCHED_FUSED_PREFILL, s)
        steps(3)
        # the prompt's last tokens decide again over what is there by now
        stack.set_tokens(n)
        stack.set_tokens(st.evict(*stats, 300, sink=4, recent=50, last=32))
        steps(20)
        stack.set_tokens(st.cfg.num_tokens + 40)
        stats = prefill(40)
        kept = st.evict(*stats, 200, sink=4, recent=50)
        assert kept == 200
        stack.set_tokens(kept)
        steps(4)
