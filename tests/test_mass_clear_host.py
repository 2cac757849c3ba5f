"""prr_mass_clear without a GPU: what is refused before a launch."""
import pytest

FAKE = 0x10000  # an aligned non-null address; every case below fails validation before use


@pytest.fixture(scope="module")
def P():
    import paper_2606_30389_amd as P
    return P


def clear(P, from_len=FAKE, mass=FAKE, d=(), **over):
    a = dict(n_seqs=2, total_q=10, max_q=5, max_kv=160, cu_q=FAKE, kv_len=FAKE, page_table=FAKE, table_stride=10)
    a.update(over)
    dims = dict(num_q_heads=8, num_kv_heads=2, page_size=16, max_pages=100, dtype=P.PRR_BF16)
    dims.update(d)
    P.prr_mass_clear(P.make_dims(**dims), P.make_batch(**a), from_len, mass, stream=0)


def test_mass_clear_refusals(P):
    for over in (dict(n_seqs=0), dict(n_seqs=4097), dict(total_q=0), dict(max_q=11), dict(max_kv=-1), dict(max_kv=161), dict(kv_len=None),
                 dict(cu_q=FAKE + 1), dict(page_table=FAKE + 2), dict(table_stride=0), dict(page_table=None), dict(from_len=None),
                 dict(from_len=FAKE + 2), dict(mass=None), dict(mass=FAKE + 1)):
        with pytest.raises(P.PrrError) as e:
            clear(P, **over)
        assert e.value.status == P.PRR_ERR_INVALID_ARG, over
    for d in (dict(head_dim=64), dict(page_size=48), dict(num_kv_heads=5000, num_q_heads=5000)):
        with pytest.raises(P.PrrError) as e:
            clear(P, d=d)
        assert e.value.status == P.PRR_ERR_UNSUPPORTED, d
    clear(P, max_kv=0)  # no tokens, nothing launched
