"""Paged attention: values that are not finite, and values that a 16-bit type holds badly."""
import numpy as np
import pytest
import torch

from tests import paged as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S(built_lib):
    from paper_2609_37241_gb300 import scm
    return scm


def stream():
    return torch.cuda.current_stream().cuda_stream


def attend(S, b, Hq, Hkv, D, ps, dt, scale, variant="AUTO"):
    s = S.Scm()
    v = getattr(S, "VARIANT_" + variant)
    index = s.register(S.make_spec(S.OP_PAGED_ATTN, dt, [Hq, Hkv, D, ps], 1, 1 << 20, layout=S.LAYOUT_ANY, variant=v))
    work = torch.zeros(s.workspace(index), device="cuda")
    args = S.make_args(S.OP_PAGED_ATTN, [b["q"], b["kc"], b["vc"], b["table"], b["cu"], b["kv"], work, b["out"], b["lse"]],
                       scalar=scale)
    assert s.invoke(args, stream()) == (S.OK, index), S.trident_scm_last_error()
    assert S.trident_scm_device_status(s.h, stream())[1] == 0
    s.close()
    return b["out"].cpu().double(), b["lse"].cpu().double()


@pytest.mark.parametrize("variant", ["AUTO", "GENERIC"])
@pytest.mark.parametrize("new,kv,D", [([2, 3], [2000, 600], 128), ([1, 300], [900, 2500], 128), ([70], [3000], 64),
                                      ([2, 130], [500, 1200], 256)])
def test_rows_of_q_that_are_not_finite(S, new, kv, D, variant):
    """NaN or infinity in a row of q makes that row NaN, its lse too (not the -inf of a row without keys);
    the other rows are right."""
    Hq, Hkv, ps, dt, scale = 8, 2, 16, S.BF16, 0.08
    b = R.batch(np.random.default_rng(21), new, kv, Hq, Hkv, D, ps, dt, tail=1)
    out, lse, wgt = R.attention(b["q"].cpu(), b["kc"].cpu(), b["vc"].cpu(), b["table"].cpu(), b["cu"].tolist(), kv, ps, scale)
    bad = torch.zeros(out.shape[:2], dtype=torch.bool)
    last = sum(new) - 1
    for t, h, e, x in ((0, 3, 5, float("nan")), (last, 0, D - 1, float("inf")), (last, 6, 0, -float("inf"))):
        b["q"][t, h, e] = x
        bad[t, h] = True
    got, got_lse = attend(S, b, Hq, Hkv, D, ps, dt, scale, variant)
    assert torch.isnan(got_lse[bad]).all() and torch.isnan(got[bad]).all()
    assert (got_lse[-1] == -float("inf")).all() and (got[-1] == 0).all()  # the row of no request
    good = ~bad
    good[-1] = False
    assert ((got - out).abs() <= R.attn_tolerance(out, wgt, dt, max(kv), 5.0))[good].all()
    assert ((got_lse - lse).abs() <= R.LSE_TOLERANCE + 2.0 ** -21 * lse.abs())[good].all()
