"""The quantised append in head order with several blocks to a page and several kv heads, where a block is neither a page's
rows nor its neighbours' in memory."""
import numpy as np
import pytest

from tests.test_paged8_gpu import S, slots_of, write_case  # noqa: F401 (S: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,D,Rd,ps,bt", [(8, 4, 128, 128, 32, 8), (14, 2, 64, 32, 128, 16), (5, 5, 256, 256, 64, 1),
                                               (16, 8, 128, 64, 128, 32), (6, 3, 64, 64, 64, 32), (4, 2, 80, 80, 48, 12)])
@pytest.mark.parametrize("variant", ["VARIANT_AUTO", "VARIANT_GENERIC"])
def test_write_several_blocks_to_a_page(S, Hq, Hkv, D, Rd, ps, bt, variant):  # noqa: F811
    g = np.random.default_rng(D + ps + bt)
    runs = [(0, 1), (bt - 1, 2), (5, bt), None, (0, ps + 3), (ps - 2, 7)] + [(int(g.integers(0, ps)), 1) for _ in range(7)]
    P = sum(-(-(r[0] + r[1]) // ps) for r in runs if r) + 3
    assert write_case(S, g, S.BF16, False, False, Hq, Hkv, D, Rd, ps, bt, "head", slots_of(g, runs, P, ps, bt), P,
                      variant=getattr(S, variant)) == 0
