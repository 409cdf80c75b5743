"""Attention over 8-bit caches column by column: what blocks of small scale add has to show where blocks of large scale add
nothing, as far down as the numerators reach (include/trident_scm.h, PAGED_ATTN8)."""
import numpy as np
import pytest
import torch

from tests import paged as R
from tests import paged8 as Q
from tests.test_paged8_gpu import attend

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S(built_lib):
    from paper_2609_37241_gb300 import scm
    return scm


def bound(ref, wgt, level, dtype, n_keys, variant):
    """Q.tolerance, and half of fp16's smallest step for outputs below its normal numbers. The kernel of any alignment holds
    its numerators in fp32, so that of the other terms the output's rounding and the scores' error (2^-12 of the weights) are
    left."""
    least = 2.0 ** -25 if R.TORCH[dtype] == torch.float16 else 0.0
    if variant == "VARIANT_GENERIC":
        return 1.01 * R.UNIT[dtype] * ref.abs() + 2.0 ** -12 * wgt + least
    return Q.tolerance(ref, wgt, level, dtype, n_keys) + least


def check(b, ps, dt, scale, out, lse, variant):
    ref, want, wgt, level = Q.reference(b, ps, scale)
    tol = bound(ref, wgt, level, dt, int(b["kv"].max()), variant)
    assert ((out.cpu().double() - ref).abs() <= tol).all()
    assert ((lse.cpu().double() - want).abs() <= R.LSE_TOLERANCE).all()
    return ref, tol


@pytest.mark.parametrize("dtype", ["BF16", "FP16"])
@pytest.mark.parametrize("variant", ["VARIANT_AUTO", "VARIANT_GENERIC"])
@pytest.mark.parametrize("new", [1, 3, 150])
@pytest.mark.parametrize("gap", [8, 20, 28, 44])
def test_columns_without_the_large_block(S, gap, new, variant, dtype):
    """All keys weigh the same; one block's scale is 2^gap times the others', and its codes are zeros in half of the columns.
    There the output is what the other blocks add. Down to 2^-28 of the largest numerator it has to show in fp16 numerators
    too, and at 2^-40 and less only in those of the kernel of any alignment."""
    D, L, dt, g = 128, 96, getattr(S, dtype), np.random.default_rng(gap)
    b = Q.batch(g, [new], [L + new], 4, 1, D, 16, 16, dt)
    pages = b["table"].cpu().long()[0, :-(-(L + new) // 16)]
    b["q"].fill_(1.0)
    live = b["vc"].view(torch.uint8) != 0x7f  # rows of no request stay NaN codes
    v = torch.from_numpy(Q.codes_of(g.uniform(64.0, 440.0, b["vc"].shape))).cuda()
    v[pages[2], :, :, D // 2:] = 0
    b["vc"].view(torch.uint8).copy_(torch.where(live, v, b["vc"].view(torch.uint8)))
    b["kc"].view(torch.uint8)[live] = int(Q.codes_of(np.full(1, 0.25))[0])
    b["ks"].view(torch.uint8)[pages] = 127
    top = gap // 2 if dtype == "BF16" else min(gap // 2, 8)  # outputs of the large block within fp16's range
    b["vs"].view(torch.uint8)[pages] = 127 + max(top - gap, Q.LO)
    b["vs"].view(torch.uint8)[pages[2]] = 127 + top
    out, lse = attend(S, b, 4, 1, D, 16, 16, dt, D ** -0.5, getattr(S, variant))
    ref, tol = check(b, 16, dt, D ** -0.5, out, lse, variant)
    if gap <= 28 or (variant == "VARIANT_GENERIC" and dtype == "BF16"):  # the bound tells blocks that show from lost ones
        assert (ref[..., D // 2:].abs() > 2 * tol[..., D // 2:]).all()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("variant", ["VARIANT_AUTO", "VARIANT_GENERIC"])
@pytest.mark.parametrize("new", [1, 3, 150])
def test_weights_that_go_against_the_scales(S, D, variant, new):
    """Blocks' value scales from 2^-16 to 2^16 with weights as far the other way, so that all blocks add about as much."""
    dt, g, L, ps = S.BF16, np.random.default_rng(D + new), 700, 16
    b = Q.batch(g, [new], [L], 4, 2, D, ps, ps, dt)
    e = g.integers(-16, 17, b["vs"].shape)
    b["vs"].view(torch.uint8).copy_(torch.from_numpy(e + 127))
    b["q"].zero_()
    b["q"][..., 0] = 1.0
    score = -e * np.log(2.0)  # of the block's keys, by their first element
    ek = np.vectorize(Q.exponent)(np.abs(score))
    first = torch.from_numpy(Q.codes_of(score * np.exp2(-ek.astype(float)))).cuda()
    kc = b["kc"].view(torch.uint8)
    live = kc[..., :1] != 0x7f
    kc[:] = torch.where(live, torch.zeros_like(kc), kc)
    kc[..., :1] = torch.where(live, first.expand(-1, -1, ps)[..., None], kc[..., :1])
    b["ks"].view(torch.uint8).copy_(torch.from_numpy(ek + 127))
    out, lse = attend(S, b, 4, 2, D, ps, ps, dt, 1.0, getattr(S, variant))
    ref, tol = check(b, ps, dt, 1.0, out, lse, variant)
    # without the blocks below 2^-8 (and, again, those above 2^8) it would be another output
    for away in (e < -8, e > 8):
        c = dict(b, vc=b["vc"].clone())
        c["vc"].view(torch.uint8).masked_fill_(torch.from_numpy(away).cuda()[..., None] & live, 0)
        assert ((Q.reference(c, ps, 1.0)[0] - ref).abs() > 2 * tol).double().mean() > 0.5
