"""Numbers of rows near 2^31, to which the size of a tile is added in 32 bits; dry runs."""
import pytest


@pytest.fixture(scope="module")
def mf():
    import __graft_entry__ as g
    g.build()
    import paper_2107_06960_gb300 as mf
    return mf


MOST = (1 << 31) - 1


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("n_kv", [0, 64])
@pytest.mark.parametrize("n_q", [MOST, MOST - 200, MOST - 60000])
def test_rows_near_32_bits_are_refused(mf, n_q, n_kv, dtype):
    for make in (lambda: mf.CrossAttention(1, n_q, n_kv, 1, 1, 64, dtype=dtype, dry_run=True),
                 lambda: mf.PrefixAttention(1, 1, n_q, n_kv, n_kv, 1, 1, 64, dtype=dtype, dry_run=True),
                 lambda: mf.CrossAttention(n_q, 1, n_kv, 1, 1, 64, dtype=dtype, dry_run=True)):
        with pytest.raises(mf.MafatError) as e:
            make()
        assert mf.STATUS[e.value.status] == "EUNSUPPORTED", str(e.value)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("kernel", [1, 2])
def test_rows_below_are_counted_right(mf, kernel, dtype):
    n_q = MOST - 70000
    s = mf.CrossAttention(1, n_q, 64, 1, 1, 64, dtype=dtype, kernel=kernel, splits=1, dry_run=True).stats()
    tiles = [-(-n_q // rows) for rows in ([16, 8] if kernel == 1 else [128, 256, 64])]
    assert s["ctas"][0] in tiles or (kernel == 1 and dtype == 0 and s["ctas"][0] == 304)
