"""Rows that give no weight, whatever they hold."""
import math

import pytest
import torch

from tests import context_support as S

DEV = "cuda:0"


def rand(*shape, seed=0, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["16", "e4m3"])
@pytest.mark.parametrize("n,past,hq", [(1, 300, 4), (50, 70, 4), (64, 4000, 16), (700, 300, 1), (300, 0, 7)])
def test_rows_without_weight_give_none_whatever_they_hold(n, past, hq, kind):
    """Queries of NaN and infinity whose l is 0: the mass of the other rows alone, to the bit."""
    import paper_2606_30389_amd as P
    kv = n + past
    pages = -(-kv // 16)
    dims = P.make_dims(hq, 1, 16, pages, P.PRR_BF16)
    k = rand(1, pages, 16, S.D, seed=1)
    scale, code = None, P.PRR_KV_16
    if kind == "e4m3":
        k, code = k.float().to(torch.float8_e4m3fn).view(torch.uint8), P.PRR_KV_E4M3
        scale = torch.full((1, pages, 16), 127, dtype=torch.uint8, device=DEV)
    q = rand(n, hq, S.D, seed=2)
    m, l = torch.rand(n, hq, device=DEV) + 3, torch.rand(n, hq, device=DEV) + 1
    none = torch.rand(n, hq, device=DEV, generator=torch.Generator(device=DEV).manual_seed(5)) < 0.2
    none[n // 2] = True
    l[none] = 0.0
    batch = P.make_batch(1, n, n, kv, torch.tensor([0, n], dtype=torch.int32, device=DEV) if n > 1 else None,
                         torch.tensor([kv], dtype=torch.int32, device=DEV))
    for sh in (None, P.make_shape(2.0), P.make_shape(2.0, torch.ones(hq, device=DEV)), P.make_shape(window=100)):
        nbytes = P.prr_mass_workspace_size(dims, batch, sh, code)
        ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=DEV)

        def run(q, m):
            mass = torch.zeros(1, pages, 16, device=DEV)
            P.prr_key_mass(dims, batch, sh, q, code, k, scale, m, l, 0, None, None, 0, None, 0.0, mass, ws, nbytes)
            torch.cuda.synchronize()
            return mass

        want = run(q, m)
        assert want.isfinite().all() and (want.any() or bool(none.all()))
        for x in (math.nan, math.inf, -math.inf, 3e38):
            odd, mx = q.clone(), m.clone()
            odd[none] = x
            mx[none] = x
            assert torch.equal(run(odd, mx), want), x
