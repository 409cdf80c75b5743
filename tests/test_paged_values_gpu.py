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


@pytest.mark.parametrize("new,kv,D", [([1], [60000], 128), ([2, 4], [3000, 9000], 64), ([3], [7000], 256),
                                      ([130], [6000], 128), ([200], [5000], 64), ([140], [4000], 256)])
def test_numerators_below_the_smallest_of_fp16(S, new, kv, D):
    """Keys with a score 18 below the largest, e^-18 = 2^-26 of it, make the output: the largest ones' v is 0."""
    Hq, Hkv, ps, dt = 8, 2, 16, S.FP16
    g = np.random.default_rng(22)
    b = R.batch(g, new, kv, Hq, Hkv, D, ps, dt)
    b["q"].zero_()
    b["q"][..., 0] = 1.0
    tab = b["table"].cpu().numpy()
    for r, L in enumerate(kv):
        level = torch.zeros(-(-L // ps) * ps)
        level[:L] = torch.where(torch.arange(L) % 512 < 64, 18.0, 0.0)  # 64 of 512 keys: some in every part and tile run
        v = torch.from_numpy(g.uniform(50, 150, (level.numel(), Hkv, D)).astype(np.float32)).half()
        v[level > 0] = 0.0
        for j in range(-(-L // ps)):
            n = min(ps, L - j * ps)
            b["kc"][int(tab[r, j]), :, :n, 0] = level[j * ps:j * ps + n].half().cuda()
            b["vc"][int(tab[r, j]), :, :n] = v[j * ps:j * ps + n].transpose(0, 1).cuda()
    ref = R.attention(b["q"].cpu(), b["kc"].cpu(), b["vc"].cpu(), b["table"].cpu(), b["cu"].tolist(), kv, ps, 1.0)
    got, got_lse = attend(S, b, Hq, Hkv, D, ps, dt, 1.0)
    out, lse, wgt = ref
    # the output's rounding and the numerators', and of each numerator at most 2^-32 of the largest (half a step
    # below fp16's normal numbers, times 2^-7), with at least 64 largest ones to 512 keys; the output's own
    # smallest step. The scores are exact, up to fp32's roundings of scale and maximum (within 2^-12).
    u = R.UNIT[dt]
    tol = u * out.abs() * (1 + u) + (1.05 * u + 2.0 ** -12) * wgt + 512 / 64 * 2.0 ** -32 * 150 + 2.0 ** -25
    assert ((got - out).abs() <= tol).all(), ((got - out).abs() / tol).max()
    assert out.abs().max() > 20 * tol.max()  # what was lost before is seen here
    assert ((got_lse - lse).abs() <= R.LSE_TOLERANCE + 2.0 ** -21 * lse.abs()).all()
