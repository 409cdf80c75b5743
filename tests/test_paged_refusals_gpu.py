"""Calls of paged attention that are refused at the launch: nothing has been written, and the next call is right."""
import numpy as np
import pytest
import torch

from tests import paged as R

pytestmark = pytest.mark.gpu

HQ, HKV, D, PS = 8, 2, 128, 2048


@pytest.fixture(scope="module")
def S(built_lib):
    from paper_2609_37241_gb300 import scm
    return scm


def desc(S, t, **change):
    """A tensor's descriptor, with some of it changed."""
    dtype = {torch.bfloat16: S.BF16, torch.int32: S.I32, torch.float32: S.FP32}[t.dtype]
    return dict(dict(addr=t.data_ptr(), dtype=dtype, shape=tuple(t.shape), stride=tuple(t.stride()), device=t.device.index),
                **change)


def refused_then_right(S, status, change, flags=0):
    """A call that launches both kernels on one page per request, with `change` made to its tensors."""
    stream = torch.cuda.current_stream().cuda_stream
    s = S.Scm(flags=S.OPT_PDL | flags)
    index = s.register(S.make_spec(S.OP_PAGED_ATTN, S.BF16, [HQ, HKV, D, PS], 1, 1 << 20, layout=S.LAYOUT_ANY))
    work = torch.zeros(s.workspace(index), device="cuda")
    b = R.batch(np.random.default_rng(31), [1, 300], [700, 2000], HQ, HKV, D, PS, S.BF16, spare=0)
    ts = [b["q"], b["kc"], b["vc"], b["table"], b["cu"], b["kv"], work, b["out"], b["lse"]]
    ref = R.attention(b["q"].cpu(), b["kc"].cpu(), b["vc"].cpu(), b["table"].cpu(), b["cu"].tolist(), [700, 2000], PS, 0.1)
    assert s.invoke(S.make_args(S.OP_PAGED_ATTN, change([desc(S, t) for t in ts], b), scalar=0.1), stream)[0] == status
    torch.cuda.synchronize()
    assert torch.isnan(b["out"]).all() and torch.isnan(b["lse"]).all()
    assert s.invoke(S.make_args(S.OP_PAGED_ATTN, ts, scalar=0.1), stream) == (S.OK, index)
    assert S.trident_scm_device_status(s.h, stream)[1] == 0
    out, lse, wgt = ref
    assert ((b["out"].cpu().double() - out).abs() <= R.attn_tolerance(out, wgt, S.BF16, 2000, 5.0)).all()
    s.close()


def test_a_tensor_map_that_cannot_be_made(S):
    """Pages 2^40 bytes apart, of which the call would read the first only: TMA takes less. (The caches' span
    holds the other tensors, which the overlap check refuses where strides differ.)"""
    first = torch.zeros(2, 2, dtype=torch.int32, device="cuda")

    def change(ts, b):
        ts[3] = desc(S, first)
        for k in (1, 2):
            ts[k] = dict(ts[k], stride=(1 << 39,) + ts[k]["stride"][1:])
        return ts

    refused_then_right(S, S.ERR_CUDA, change, S.OPT_NO_ALIAS_CHECK)


def wide_table(b, width):
    t = torch.zeros(b["table"].shape[0], width, dtype=torch.int32, device="cuda")
    t[:, :b["table"].shape[1]] = b["table"]
    return t


def test_a_table_of_nearly_2_to_the_31_keys(S):
    """Key numbers are 32-bit; the kernels look a little past the last one."""
    refused_then_right(S, S.ERR_INVALID, lambda ts, b: ts[:3] + [desc(S, wide_table(b, (1 << 20) - 1))] + ts[4:])


def test_a_table_just_below(S):
    stream = torch.cuda.current_stream().cuda_stream
    s = S.Scm()
    index = s.register(S.make_spec(S.OP_PAGED_ATTN, S.BF16, [HQ, HKV, D, PS], 1, 1 << 20, layout=S.LAYOUT_ANY))
    work = torch.zeros(s.workspace(index), device="cuda")
    b = R.batch(np.random.default_rng(32), [1, 300], [700, 2000], HQ, HKV, D, PS, S.BF16, spare=0)
    out, lse, wgt = R.attention(b["q"].cpu(), b["kc"].cpu(), b["vc"].cpu(), b["table"].cpu(), b["cu"].tolist(), [700, 2000], PS,
                                0.1)
    table = wide_table(b, (1 << 20) - 3)
    ts = [b["q"], b["kc"], b["vc"], table, b["cu"], b["kv"], work, b["out"], b["lse"]]
    assert s.invoke(S.make_args(S.OP_PAGED_ATTN, ts, scalar=0.1), stream) == (S.OK, index)
    assert S.trident_scm_device_status(s.h, stream)[1] == 0
    assert ((b["out"].cpu().double() - out).abs() <= R.attn_tolerance(out, wgt, S.BF16, 2000, 5.0)).all()
    s.close()
