"""Host side of the ops over caches held in 8 bits: registration, selection and refusals (no GPU)."""
import math

import pytest

from tests.test_paged_host import Mem


@pytest.fixture(scope="module")
def S(built_lib):
    from paper_2609_37241_gb300 import scm
    return scm


def pools(S, m, P, Hkv, ps, D, bt):
    return [m(S.E4M3, (P, Hkv, ps, D)), m(S.E4M3, (P, Hkv, ps, D)), m(S.E8M0, (P, Hkv, ps // bt)), m(S.E8M0, (P, Hkv, ps // bt))]


def write_args(S, qk=False, T=4, Hq=4, Hkv=2, D=64, Rd=32, P=8, ps=16, bt=8):
    m = Mem()
    a = S.BF16
    t = [m(a, (T, Hq, D)), m(a, (T, Hkv, D)), m(a, (T, Hkv, D)), m(S.I32, (T,)), m(S.I32, (T,)), m(S.FP32, (Rd // 2, 2)),
         m(a, (T, Hq, D)), *pools(S, m, P, Hkv, ps, D, bt)]
    return t + ([m(S.FP32, (D,)), m(S.FP32, (D,))] if qk else []), dict(scalar=1.0)


def read_args(S, T=5, B=3, Hkv=2, D=64, P=8, ps=16, bt=8, M=4):
    m = Mem()
    t = [*pools(S, m, P, Hkv, ps, D, bt), m(S.I32, (B, M)), m(S.I32, (B + 1,)), m(S.I32, (B,)), m(S.BF16, (T, Hkv, D)),
         m(S.BF16, (T, Hkv, D))]
    return t, {}


def attn_args(S, T=5, B=2, Hq=8, Hkv=2, D=128, P=9, ps=16, bt=16, M=4, W=0):
    m = Mem()
    a = S.BF16
    t = [m(a, (T, Hq, D)), *pools(S, m, P, Hkv, ps, D, bt), m(S.I32, (B, M)), m(S.I32, (B + 1,)), m(S.I32, (B,)), m(S.FP32, (W,)),
         m(a, (T, Hq, D)), m(S.FP32, (T, Hq))]
    return t, dict(scalar=0.1)


def table(S):
    s = S.Scm(flags=S.OPT_DRY_RUN)
    assert s.register(S.make_spec(S.OP_ROPE_PAGED_KV8, S.BF16, [4, 2, 64, 32, 16, 8], 1, 64)) == 0
    assert s.register(S.make_spec(S.OP_QKNORM_ROPE_PAGED_KV8_INTERLEAVED, S.BF16, [4, 2, 64, 32, 16, 8], 1, 64)) == 1
    assert s.register(S.make_spec(S.OP_PAGED_READ8, S.BF16, [2, 64, 16, 8], 1, 64)) == 2
    assert s.register(S.make_spec(S.OP_PAGED_ATTN8, S.BF16, [8, 2, 128, 16, 16], 1, 64, layout=S.LAYOUT_ANY)) == 3
    return s


def test_each_op_selects_its_version(S):
    s = table(S)
    for make, op, want in ((write_args, S.OP_ROPE_PAGED_KV8, 0), (lambda S: write_args(S, qk=True), S.OP_QKNORM_ROPE_PAGED_KV8_INTERLEAVED, 1),
                           (read_args, S.OP_PAGED_READ8, 2), (attn_args, S.OP_PAGED_ATTN8, 3)):
        t, kw = make(S)
        assert s.invoke(S.make_args(op, t, **kw)) == (S.OK, want)
    t, kw = write_args(S)
    assert s.invoke(S.make_args(S.OP_ROPE_PAGED_KV8_INTERLEAVED, t, **kw)) == (S.MISS, -1)
    s.close()


def test_guards_miss(S):
    s = table(S)

    def miss(make, op, k, **change):
        t, kw = make(S)
        t[k].update(change)
        assert s.invoke(S.make_args(op, t, **kw)) == (S.MISS, -1), (op, k, change)

    w, r, a = S.OP_ROPE_PAGED_KV8, S.OP_PAGED_READ8, S.OP_PAGED_ATTN8
    miss(write_args, w, 7, dtype=S.U8)                                      # bytes are no codes
    miss(write_args, w, 9, dtype=S.U8)
    miss(write_args, w, 9, dtype=S.E4M3)
    miss(write_args, w, 9, shape=(8, 2, 1), stride=(2, 1, 1))               # another block
    miss(write_args, w, 10, shape=(8, 2, 3), stride=(6, 3, 1))
    miss(write_args, w, 9, stride=(4, 1, 1))                                # scales on the same bytes
    miss(write_args, w, 8, stride=(2 * 16 * 64, 8, 64, 1))                  # heads overlap rows
    miss(write_args, w, 7, addr=0x10000000 + 8)                             # codes not 16-byte aligned
    miss(write_args, w, 0, dtype=S.FP16)
    miss(write_args, w, 5, shape=(8, 2), stride=(2, 1))                     # another R
    miss(read_args, r, 7, dtype=S.FP16)
    miss(read_args, r, 8, shape=(5, 2, 32), stride=(64, 32, 1))
    miss(read_args, r, 6, shape=(2,))
    miss(read_args, r, 5, shape=(3,))
    miss(attn_args, a, 1, dtype=S.BF16)
    miss(attn_args, a, 3, shape=(9, 2, 2), stride=(4, 2, 1))
    miss(attn_args, a, 10, shape=(5, 4), stride=(4, 1))
    t, kw = attn_args(S)
    t[3].update(addr=t[3]["addr"] + 5)                                      # scales at any byte
    assert s.invoke(S.make_args(a, t, **kw)) == (S.OK, 3)
    t, kw = attn_args(S)
    t[3].update(shape=(9, 2, 0), stride=(0, 0, 1))
    assert s.invoke(S.make_args(a, t, **kw)) == (S.MISS, -1)
    s.close()


def test_shared_buffers(S):
    """k and v of one buffer, a page's codes and scales behind one another; nothing on another's bytes."""
    s = table(S)
    n, rec = 2 * 16 * 64, 2 * 2 * 16 * 64 + 16

    def record(t, ks=0):
        st, base = (rec, 16 * 64, 64, 1), t[7]["addr"]
        t[7] = dict(t[7], stride=st)
        t[8] = dict(t[8], addr=base + n, stride=st)
        t[9] = dict(t[9], addr=base + 2 * n + ks, stride=(rec, 2, 1))
        t[10] = dict(t[10], addr=base + 2 * n + 4, stride=(rec, 2, 1))

    t, kw = write_args(S)
    record(t)
    assert s.invoke(S.make_args(S.OP_ROPE_PAGED_KV8, t, **kw)) == (S.OK, 0)
    record(t, ks=3)  # a k scale on a v scale's byte
    assert s.invoke(S.make_args(S.OP_ROPE_PAGED_KV8, t, **kw))[0] == S.ERR_INVALID
    record(t, ks=-1)  # ... and on a code's
    assert s.invoke(S.make_args(S.OP_ROPE_PAGED_KV8, t, **kw))[0] == S.ERR_INVALID
    t, kw = write_args(S)  # a block's scales side by side: k's and v's in turn
    t[9] = dict(t[9], stride=(8, 4, 2))
    t[10] = dict(t[10], addr=t[9]["addr"] + 1, stride=(8, 4, 2))
    assert s.invoke(S.make_args(S.OP_ROPE_PAGED_KV8, t, **kw)) == (S.OK, 0)
    t[10] = dict(t[10], addr=t[9]["addr"] + 2)
    assert s.invoke(S.make_args(S.OP_ROPE_PAGED_KV8, t, **kw))[0] == S.ERR_INVALID
    t, kw = write_args(S)
    t[6] = dict(t[0])  # q in place
    assert s.invoke(S.make_args(S.OP_ROPE_PAGED_KV8, t, **kw)) == (S.OK, 0)
    t, kw = read_args(S)
    t[8] = dict(t[7])
    assert s.invoke(S.make_args(S.OP_PAGED_READ8, t, **kw))[0] == S.ERR_INVALID
    t, kw = read_args(S)
    t[7] = dict(t[7], addr=t[0]["addr"])
    assert s.invoke(S.make_args(S.OP_PAGED_READ8, t, **kw))[0] == S.ERR_INVALID
    t, kw = attn_args(S)
    t[9] = dict(t[0])
    assert s.invoke(S.make_args(S.OP_PAGED_ATTN8, t, **kw))[0] == S.ERR_INVALID
    s.close()


@pytest.mark.parametrize("scalar", [0.0, -1.0, math.nan, math.inf, 1e-60])
def test_scalars_are_checked(S, scalar):
    s = table(S)
    for make, op in ((write_args, S.OP_ROPE_PAGED_KV8), (attn_args, S.OP_PAGED_ATTN8)):
        t, _ = make(S)
        assert s.invoke(S.make_args(op, t, scalar=scalar))[0] == S.ERR_INVALID
    s.close()


def test_registration_refusals(S):
    s = S.Scm(flags=S.OPT_DRY_RUN)
    w, r, a = S.OP_ROPE_PAGED_KV8, S.OP_PAGED_READ8, S.OP_PAGED_ATTN8
    for op, dtype, fixed, kw in (
            (w, S.BF16, [4, 2, 64, 32, 16, 5], {}), (w, S.BF16, [4, 2, 64, 32, 16, 32], {}), (w, S.BF16, [4, 2, 64, 33, 16, 16], {}),
            (w, S.BF16, [4, 2, 64, 66, 16, 16], {}), (w, S.BF16, [4, 2, 64, 32, 16], {}), (w, S.FP32, [4, 2, 64, 32, 16, 16], {}),
            (w, S.E4M3, [4, 2, 64, 32, 16, 16], {}), (w, S.BF16, [4, 2, 1026, 32, 16, 16], {}),
            (w, S.BF16, [4, 2, 64, 8, 16, 16], dict(variant=S.VARIANT_VECTOR)), (r, S.BF16, [2, 64, 16, 3], {}),
            (r, S.FP32, [2, 64, 16, 16], {}), (r, S.BF16, [2, 2048, 16, 16], {}), (r, S.BF16, [2, 64, 16, 16], dict(rank=3)),
            (a, S.BF16, [6, 4, 64, 16, 16], {}), (a, S.BF16, [6, 2, 520, 16, 16], {}), (a, S.BF16, [6, 2, 64, 16, 6], {}),
            (a, S.FP32, [8, 2, 64, 16, 16], {}), (a, S.BF16, [8, 2, 96, 16, 16], dict(variant=S.VARIANT_VECTOR))):
        with pytest.raises(S.ScmError):
            s.register(S.make_spec(op, dtype, fixed, 1, 8, **kw))
    s.close()


def test_other_ops_miss_on_codes(S):
    s = S.Scm(flags=S.OPT_DRY_RUN)
    s.register(S.make_spec(S.OP_SILU, S.BF16, [64], 1, 8))
    m = Mem()
    assert s.invoke(S.make_args(S.OP_SILU, [m(S.E4M3, (4, 64)), m(S.E4M3, (4, 64))])) == (S.MISS, -1)
    with pytest.raises(S.ScmError):
        s.register(S.make_spec(S.OP_SILU, S.E4M3, [64], 1, 8))
    s.close()


def test_torch_dtypes(S):
    import torch
    x = torch.zeros(2, 3, dtype=torch.uint8)
    args = S.make_args(S.OP_SILU, [x.view(torch.float8_e4m3fn), x.view(torch.float8_e8m0fnu)])
    assert (args.t[0].dtype, args.t[1].dtype) == (S.E4M3, S.E8M0) == (7, 8)
