"""Host side of the paged ops: registration, selection, refusals and the frequency table (no GPU)."""
import math

import numpy as np
import pytest

BASE = 0x10000000


@pytest.fixture(scope="module")
def S(built_lib):
    from paper_2609_37241_gb300 import scm
    return scm


def dense(shape):
    st, n = [], 1
    for d in reversed(shape):
        st.insert(0, n)
        n *= d
    return tuple(st)


class Mem:
    """Tensor descriptors at addresses of their own."""

    def __init__(self):
        self.at = BASE

    def __call__(self, dtype, shape, stride=None, offset=0):
        d = dict(addr=self.at + offset, dtype=dtype, shape=tuple(shape), stride=tuple(stride or dense(shape)), device=0)
        self.at += 1 << 24
        return d


def map_args(S, B=3, F=20, M=4, N=16, **kw):
    m = Mem()
    i = S.I32
    t = [m(i, (B,)), m(i, (B,)), m(i, (F,)), m(i, (1,)), m(i, (B, M)), m(i, (B + 1,)), m(i, (B,)), m(i, (N,)), m(i, (N,)),
         m(i, (1,))]
    return t, dict(scalar=16.0, **kw)


def rope_args(S, qk=False, T=4, Hq=4, Hkv=2, D=64, R=32, P=8, ps=16):
    m = Mem()
    a = S.BF16
    t = [m(a, (T, Hq, D)), m(a, (T, Hkv, D)), m(a, (T, Hkv, D)), m(S.I32, (T,)), m(S.I32, (T,)), m(S.FP32, (R // 2, 2)),
         m(a, (T, Hq, D)), m(a, (P, Hkv, ps, D)), m(a, (P, Hkv, ps, D))]
    if qk:
        t += [m(S.FP32, (D,)), m(S.FP32, (D,))]
    return t, dict(scalar=1.0)


def attn_args(S, T=5, B=2, Hq=8, Hkv=2, D=128, P=9, ps=16, M=4, W=0):
    m = Mem()
    a = S.BF16
    t = [m(a, (T, Hq, D)), m(a, (P, Hkv, ps, D)), m(a, (P, Hkv, ps, D)), m(S.I32, (B, M)), m(S.I32, (B + 1,)),
         m(S.I32, (B,)), m(S.FP32, (W,)), m(a, (T, Hq, D)), m(S.FP32, (T, Hq))]
    return t, dict(scalar=0.1)


def table(S):
    s = S.Scm(flags=S.OPT_DRY_RUN)
    assert s.register(S.make_spec(S.OP_PAGE_MAP, S.I32, [], 1, 64, align_bytes=4)) == 0
    assert s.register(S.make_spec(S.OP_ROPE_PAGED_KV, S.BF16, [4, 2, 64, 32, 16], 1, 64)) == 1
    assert s.register(S.make_spec(S.OP_QKNORM_ROPE_PAGED_KV_INTERLEAVED, S.BF16, [4, 2, 64, 32, 16], 1, 64)) == 2
    assert s.register(S.make_spec(S.OP_PAGED_ATTN, S.BF16, [8, 2, 128, 16], 1, 64, layout=S.LAYOUT_ANY)) == 3
    return s


def test_each_op_selects_its_version(S):
    s = table(S)
    t, kw = map_args(S)
    assert s.invoke(S.make_args(S.OP_PAGE_MAP, t, **kw)) == (S.OK, 0)
    t, kw = rope_args(S)
    assert s.invoke(S.make_args(S.OP_ROPE_PAGED_KV, t, **kw)) == (S.OK, 1)
    assert s.invoke(S.make_args(S.OP_ROPE_PAGED_KV_INTERLEAVED, t, **kw)) == (S.MISS, -1)
    t, kw = rope_args(S, qk=True)
    assert s.invoke(S.make_args(S.OP_QKNORM_ROPE_PAGED_KV_INTERLEAVED, t, **kw)) == (S.OK, 2)
    t, kw = attn_args(S)
    assert s.invoke(S.make_args(S.OP_PAGED_ATTN, t, **kw)) == (S.OK, 3)
    s.close()


def test_in_place_and_shared_buffers(S):
    s = table(S)
    t, kw = rope_args(S)
    t[6] = dict(t[0])  # q_out = q
    assert s.invoke(S.make_args(S.OP_ROPE_PAGED_KV, t, **kw)) == (S.OK, 1)
    t, kw = rope_args(S)
    st = (2 * 2 * 16 * 64, 16 * 64, 64, 1)  # k and v pages of one buffer
    t[7] = dict(t[7], stride=st)
    t[8] = dict(t[7], addr=t[7]["addr"] + 2 * 2 * 16 * 64, stride=st)
    assert s.invoke(S.make_args(S.OP_ROPE_PAGED_KV, t, **kw)) == (S.OK, 1)
    t[8] = dict(t[7])  # k and v on the same bytes
    assert s.invoke(S.make_args(S.OP_ROPE_PAGED_KV, t, **kw))[0] == S.ERR_INVALID
    t, kw = attn_args(S)
    t[7] = dict(t[0])  # other blocks still read q
    assert s.invoke(S.make_args(S.OP_PAGED_ATTN, t, **kw))[0] == S.ERR_INVALID
    t, kw = map_args(S)
    t[6] = dict(t[0])
    assert s.invoke(S.make_args(S.OP_PAGE_MAP, t, **kw))[0] == S.ERR_INVALID
    s.close()


def test_guards_miss(S):
    s = table(S)

    def miss(make, op, k, **change):
        t, kw = make(S)
        t[k].update(change)
        assert s.invoke(S.make_args(op, t, **kw)) == (S.MISS, -1), (op, k, change)

    a = S.OP_PAGED_ATTN
    miss(attn_args, a, 0, dtype=S.FP16)                                   # mixed activations
    miss(attn_args, a, 3, dtype=S.I64)
    miss(attn_args, a, 4, shape=(4,), stride=(1,))                        # cu_q of another length
    miss(attn_args, a, 5, stride=(2,))
    miss(attn_args, a, 2, shape=(9, 2, 8, 128))                           # v pages of another size
    miss(attn_args, a, 1, stride=(2 * 16 * 128, 16 * 128, 128, 2))        # rows not packed
    miss(attn_args, a, 1, stride=(2 * 16 * 128, 64, 128, 1))              # heads overlap rows
    miss(attn_args, a, 1, addr=BASE + 2)                                  # not 16-byte aligned
    miss(attn_args, a, 8, shape=(5, 4), stride=(4, 1))
    r = S.OP_ROPE_PAGED_KV
    miss(rope_args, r, 5, shape=(8, 2), stride=(2, 1))                    # another R
    miss(rope_args, r, 5, stride=(4, 1))
    miss(rope_args, r, 3, shape=(3,))
    miss(rope_args, r, 7, stride=(0, 16 * 64, 64, 1))                     # pages on the same bytes
    p = S.OP_PAGE_MAP
    miss(map_args, p, 1, dtype=S.I64)
    miss(map_args, p, 8, shape=(15,), stride=(1,))
    miss(map_args, p, 4, stride=(3, 1))                                   # table rows overlap
    t, kw = map_args(S, B=65)                                             # past the bucket
    assert s.invoke(S.make_args(p, t, **kw)) == (S.MISS, -1)
    s.close()


@pytest.mark.parametrize("scalar", [0.0, -1.0, math.nan, math.inf, 1e-60])
def test_scalars_are_checked(S, scalar):
    s = table(S)
    t, kw = attn_args(S)
    assert s.invoke(S.make_args(S.OP_PAGED_ATTN, t, scalar=scalar))[0] == S.ERR_INVALID
    t, kw = rope_args(S)
    assert s.invoke(S.make_args(S.OP_ROPE_PAGED_KV, t, scalar=scalar))[0] == S.ERR_INVALID
    t, kw = map_args(S)
    assert s.invoke(S.make_args(S.OP_PAGE_MAP, t, scalar=scalar))[0] == S.ERR_INVALID
    assert s.invoke(S.make_args(S.OP_PAGE_MAP, t, scalar=16.5))[0] == S.ERR_INVALID
    s.close()


def test_malformed_tensors(S):
    s = table(S)
    for k, change in ((0, dict(addr=0)), (1, dict(shape=(-1, 2, 16, 128))), (2, dict(dtype=9)), (4, dict(addr=BASE + 1))):
        t, kw = attn_args(S)
        t[k].update(change)
        assert s.invoke(S.make_args(S.OP_PAGED_ATTN, t, **kw))[0] == S.ERR_INVALID, k
    t, kw = attn_args(S)
    assert s.invoke(S.make_args(S.OP_PAGED_ATTN, t[:-1], **kw))[0] == S.ERR_INVALID
    s.close()


def test_registration_refusals(S):
    s = S.Scm(flags=S.OPT_DRY_RUN)
    bad = [dict(op=S.OP_PAGE_MAP, dtype=S.BF16, fixed=[], rank=1), dict(op=S.OP_PAGE_MAP, dtype=S.I32, fixed=[], rank=2),
           dict(op=S.OP_PAGE_MAP, dtype=S.I32, fixed=[4], rank=1), dict(op=13, dtype=S.BF16, fixed=[]),
           dict(op=S.OP_PAGE_MAP, dtype=S.I32, fixed=[], rank=1, variant=S.VARIANT_VECTOR),
           dict(op=S.OP_ROPE_PAGED_KV, dtype=S.FP32, fixed=[4, 2, 64, 32, 16]),
           dict(op=S.OP_ROPE_PAGED_KV, dtype=S.BF16, fixed=[4, 2, 64, 33, 16]),
           dict(op=S.OP_ROPE_PAGED_KV, dtype=S.BF16, fixed=[4, 2, 64, 66, 16]),
           dict(op=S.OP_ROPE_PAGED_KV, dtype=S.BF16, fixed=[4, 2, 64, 32, 16], rope_theta=1e4),
           dict(op=S.OP_ROPE_PAGED_KV, dtype=S.BF16, fixed=[4, 2, 64, 8, 16], variant=S.VARIANT_VECTOR),
           dict(op=S.OP_PAGED_ATTN, dtype=S.BF16, fixed=[6, 4, 64, 16]), dict(op=S.OP_PAGED_ATTN, dtype=S.BF16, fixed=[6, 2, 520, 16]),
           dict(op=S.OP_PAGED_ATTN, dtype=S.FP32, fixed=[8, 2, 64, 16])]
    for d in bad:
        with pytest.raises(S.ScmError):
            s.register(S.make_spec(tok_lo=1, tok_hi=8, **d))
    assert s.register(S.make_spec(S.OP_PAGED_ATTN, S.BF16, [8, 2, 64, 16], 1, 8)) == 0
    with pytest.raises(S.ScmError):
        s.workspace(0)  # a dry-run SCM has no device
    assert S.trident_scm_workspace(s.h, 5)[0] == S.ERR_INVALID
    s.close()


def test_rope_freqs(S):
    R, theta = 128, 500000.0
    f = np.array([theta ** (-2.0 * i / R) for i in range(R // 2)])

    def got(*a, **kw):
        st, v = S.trident_rope_freqs(theta, R, *a, **kw)
        assert st == S.OK
        v = np.array(v, np.float64).reshape(-1, 2)
        assert (np.abs(v[:, 1]) <= np.abs(v[:, 0]) * 2.0 ** -24).all()
        return v.sum(1)

    tol = dict(rtol=2.0 ** -46, atol=0)  # two fp32 of 24 bits, and the fp64 power's own rounding
    np.testing.assert_allclose(got(), f, **tol)
    np.testing.assert_allclose(got(S.ROPE_LINEAR, factor=4.0), f / 4, **tol)
    base = got(S.ROPE_BASE, factor=8.0)
    np.testing.assert_allclose(base[0], 1.0, **tol)
    np.testing.assert_allclose(base[-1], f[-1] / 8, rtol=1e-13)
    turns = 8192 * f / (2 * math.pi)
    keep = np.clip((turns - 1) / 31, 0, 1)
    np.testing.assert_allclose(got(S.ROPE_PARTS, factor=8.0, context=8192.0), f * (keep + (1 - keep) / 8), rtol=1e-13)
    for a in ((theta, 127), (theta, 0), (theta, 1026), (0.0, 128), (math.inf, 128)):
        assert S.trident_rope_freqs(*a)[0] == S.ERR_INVALID
    for kw in (dict(scaling=4), dict(scaling=S.ROPE_LINEAR, factor=0.5), dict(scaling=S.ROPE_PARTS, factor=2.0),
               dict(scaling=S.ROPE_PARTS, factor=2.0, context=8.0, slow=4.0, fast=4.0)):
        assert S.trident_rope_freqs(theta, 128, **kw)[0] == S.ERR_INVALID
    assert S.trident_rope_freqs(theta, 2, S.ROPE_BASE, 2.0)[0] == S.ERR_INVALID
