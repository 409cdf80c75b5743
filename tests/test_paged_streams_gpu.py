"""Paged attention on two streams at once where both kernels of a call run on each: chunks beside decodes and drafts, with a
workspace for each stream, over caches of 8 and of 16 bits."""
import numpy as np
import pytest
import torch

from tests import paged as R
from tests.test_paged8_serving_gpu import attention_call

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S(built_lib):
    from paper_2609_37241_gb300 import scm
    return scm


def call(S, scm, g, bits, new, kv):
    """A batch with a workspace of its own and the call's arguments; the batch holds every tensor that they point to."""
    op, fixed = (S.OP_PAGED_ATTN8, [8, 2, 128, 16, 16]) if bits == 8 else (S.OP_PAGED_ATTN, [8, 2, 128, 16])
    i = scm.register(S.make_spec(op, S.BF16, fixed, 1, 1 << 20, layout=S.LAYOUT_ANY))
    work = torch.zeros(scm.workspace(i), device="cuda")
    if bits == 8:
        return attention_call(S, scm, g, new, kv, 128, 16, S.BF16, work)
    b = R.batch(g, new, kv, 8, 2, 128, 16, S.BF16)
    args = S.make_args(op, [b["q"], b["kc"], b["vc"], b["table"], b["cu"], b["kv"], work, b["out"], b["lse"]], scalar=128 ** -0.5)
    return dict(b, work=work), args


@pytest.mark.parametrize("bits", [(8, 8), (8, 16), (16, 16)])
def test_both_kernels_on_each_of_two_streams(S, bits):
    """Every result equals the one that the call gave alone, bit for bit, and no status is set."""
    scm, g = S.Scm(flags=S.OPT_PDL), np.random.default_rng(6)
    shapes = [([600, 1, 9, 1], [2200, 900, 64, 4000]), ([600, 500, 1, 3], [2200, 2300, 700, 3000])]
    pairs = [call(S, scm, g, n, *shape) for n, shape in zip(bits, shapes)]
    here = torch.cuda.current_stream().cuda_stream
    alone = []
    for b, args in pairs:
        assert scm.invoke(args, here)[0] == S.OK, S.trident_scm_last_error()
        alone.append((b["out"].clone(), b["lse"].clone()))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in pairs]
    for _ in range(30):
        for b, _ in pairs:
            b["out"].fill_(float("nan"))
            b["lse"].fill_(float("nan"))
        torch.cuda.synchronize()
        for _ in range(3):
            for (_, args), stream in zip(pairs, streams):
                assert scm.invoke(args, stream.cuda_stream)[0] == S.OK
        torch.cuda.synchronize()
        for (b, _), (out, lse) in zip(pairs, alone):
            assert torch.equal(b["out"], out) and torch.equal(b["lse"], lse)
    assert S.trident_scm_device_status(scm.h, here)[1] == 0
    scm.close()
