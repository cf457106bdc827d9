"""Prompts of a thousand tokens over their own keys, causal, with and without a shared prefix."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_attention import _prefix  # noqa: E402


@pytest.fixture(scope="module")
def mf():
    import paper_2107_06960_gb300 as mf
    return mf


@pytest.mark.parametrize("kernel", [0, 1, 2])
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("splits", [0, 3])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,R,T,P,S,own", [
    (1, 1, 1100, 0, 1100, None),            # a prompt alone
    (1, 2, 1024, 200, 1400, [1400, 1100]),  # behind earlier tokens and a prefix
    (2, 1, 515, 130, 700, [515, 700]),
    (1, 3, 900, 0, 1000, [300, 0, 1000])])  # fewer keys than tokens: the first tokens read nothing
def test_long_prompts(mf, G, R, T, P, S, own, D, splits, dtype, kernel):
    _prefix(mf, G, R, T, P, S, 4, 2, D, dtype, own_len=own, kernel=kernel, splits=splits, poison=True)
