"""Tiles of few rows where a CTA takes several items: each item's queries, whatever keys the item before had."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_attention import _cross, _prefix  # noqa: E402


@pytest.fixture(scope="module")
def mf():
    import paper_2107_06960_gb300 as mf
    return mf


def _several_items(stats, which, items):
    assert 0 < stats["ctas"][which] < items * stats["splits"][which]


# Keys of a part go to four warps in runs of 16, queries to the same warps in fours of 16 rows: with at most 16, 32 or 48 keys
# three, two or one of the warps have queries to copy and no key.
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,H,Hk", [(1, 64, 8), (2, 64, 8), (3, 40, 8), (1, 40, 8)])
@pytest.mark.parametrize("S", [1, 16, 20, 48, 70])
def test_items_with_few_keys(mf, S, T, H, Hk, D):
    B = 64
    plan = mf.CrossAttention(B, T, S, H, Hk, D, kernel=mf.ATTN_ROWS)
    _several_items(plan.stats(), 0, B * Hk * -(-T * H // Hk // 16))
    _cross(mf, B, T, S, H, Hk, D, mf.BF16, kernel=mf.ATTN_ROWS, repeat=3)


# 64 sequences are ordered by their lengths, 160 are taken as they are given
@pytest.mark.parametrize("B", [64, 160])
@pytest.mark.parametrize("T,H,Hk", [(1, 64, 8), (2, 32, 8)])
@pytest.mark.parametrize("S", [48, 100])
def test_items_after_empty_ones(mf, S, T, H, Hk, B):
    """Lengths of zero before others, in runs as long as the grid and in turn."""
    lens = [0, 20, 0, 48, 1, 0, 16, 33]
    for n in (lens, [0] * 40 + lens * 3 + [0] * 5):
        _cross(mf, B, T, S, H, Hk, 64, mf.BF16, kv_len=(n * B)[:B], kernel=mf.ATTN_ROWS, poison=True, repeat=3)


@pytest.mark.parametrize("splits", [2, 7])
def test_items_of_empty_parts(mf, splits):
    """Lengths far below the room leave most parts without a key."""
    B, T, S, H, Hk = 40, 2, 640, 32, 4
    plan = mf.CrossAttention(B, T, S, H, Hk, 64, kernel=mf.ATTN_ROWS, splits=splits)
    _several_items(plan.stats(), 0, B * Hk)
    _cross(mf, B, T, S, H, Hk, 64, mf.BF16, kv_len=[(50 * i) % 700 for i in range(B)], kernel=mf.ATTN_ROWS, splits=splits,
           poison=True, repeat=3)


def test_items_by_the_plans_own_choice(mf):
    plan = mf.CrossAttention(64, 1, 20, 64, 8, 64)
    _several_items(plan.stats(), 0, 64 * 8)
    _cross(mf, 64, 1, 20, 64, 8, 64, mf.BF16, repeat=3)
    plan = mf.PrefixAttention(4, 64, 1, 676, 30, 64, 8, 64)
    _several_items(plan.stats(), 1, 256 * 8)
    _prefix(mf, 4, 64, 1, 676, 30, 64, 8, 64, mf.BF16, own_len=[(7 * i) % 32 for i in range(256)], poison=True)
