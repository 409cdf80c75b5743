"""The ops over paged caches held in 8 bits, on the GPU against their formulas in 64 bits."""
import numpy as np
import pytest
import torch

from tests import paged as R
from tests import paged8 as Q

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S(built_lib):
    from paper_2609_37241_gb300 import scm
    return scm


def stream():
    return torch.cuda.current_stream().cuda_stream


def i32(x):
    return torch.tensor(np.asarray(x, np.int32)).cuda()


# ---------------------------------------------------------------- the quantised append
OPS = {(False, False): "OP_ROPE_PAGED_KV8", (True, False): "OP_ROPE_PAGED_KV8_INTERLEAVED",
       (False, True): "OP_QKNORM_ROPE_PAGED_KV8", (True, True): "OP_QKNORM_ROPE_PAGED_KV8_INTERLEAVED"}


def slots_of(g, runs, P, ps, bt):
    """Slots of consecutive tokens: for each (start in a page, length) pages of their own; None: a padding token."""
    ids, at, slots = g.permutation(P).tolist(), 0, []
    for run in runs:
        if run is None:
            slots.append(-1)
            continue
        start, n = run
        pages = ids[at:at + -(-(start + n) // ps)]
        at += len(pages)
        slots += [pages[j // ps] * ps + j % ps for j in range(start, start + n)]
    return slots


def write_case(S, g, dt, inter, qk, Hq, Hkv, D, Rd, ps, bt, order, slots, P, k_size=1.0, variant=None, bad_pos=(), fused=True):
    """Runs one call; returns (got, want) pieces after checking them."""
    T = len(slots)
    op = getattr(S, OPS[inter, qk])
    s = S.Scm()
    s.register(S.make_spec(op, dt, [Hq, Hkv, D, Rd, ps, bt], 1, 1 << 20, layout=S.LAYOUT_ANY,
                           align_bytes=16 if D % 16 == 0 else 2,
                           variant=S.VARIANT_AUTO if variant is None else variant))
    act = R.TORCH[dt]
    rows = torch.from_numpy(g.standard_normal((T, Hq + 2 * Hkv, D)) * np.exp(g.standard_normal((T, Hq + 2 * Hkv, 1))))
    rows[:, Hq:Hq + Hkv] *= k_size
    qkv = rows.to(act).cuda()
    q, k, v = qkv.split([Hq, Hkv, Hkv], 1)
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    pos = g.integers(0, 60000, T)
    for t in bad_pos:
        pos[t] = -5 if t % 2 else 1 << 24
    freqs = S.rope_freqs(10000.0, Rd)
    kc, vc, ks, vs = Q.pool(g, P, Hkv, ps, D, bt, order)
    for c in (ks, vs):
        c.view(torch.uint8)[::5] = 127 - 40  # scales outside the range
    gam = [torch.from_numpy(g.standard_normal(D) * 0.1 + 1).float().cuda() for _ in range(2)] if qk else []
    mag, eps = 1.25, 1e-6
    q_out = torch.full((T, Hq, D), 7.0, dtype=act, device="cuda")
    before = [c.cpu().contiguous().view(torch.uint8).numpy().copy() for c in (kc, vc, ks, vs)]
    args = S.make_args(op, [q, k, v, i32(pos), i32(slots), freqs, q_out, kc, vc, ks, vs, *gam], eps=eps, scalar=mag)
    assert s.invoke(args, stream()) == (S.OK, 0), S.trident_scm_last_error()
    bits = S.trident_scm_device_status(s.h, stream())[1]
    f = freqs.double().sum(1).cpu()
    skip = [not 0 <= p < 1 << 24 for p in pos]
    live = torch.tensor([not x for x in skip])
    P64 = torch.tensor(np.where(skip, 0, pos))
    ref_q = R.rotate(q.cpu().double(), P64, f, mag, inter, gam[0].cpu().double() if qk else None, eps)
    ref_k = R.rotate(k.cpu().double(), P64, f, mag, inter, gam[1].cpu().double() if qk else None, eps)
    # q: its rounding, and cos and sin to 2e-6 of a pair's magnitude
    size = q.cpu().double().abs().amax(-1, keepdim=True) * (1 if not qk else 0) + (0 if not qk else 16.0)
    tol = 1.01 * R.UNIT[dt] * ref_q.abs() + 8e-6 * size
    got_q = q_out.cpu().double()
    assert ((got_q - ref_q).abs() <= tol)[live].all()
    assert (got_q[~live] == 7.0).all()
    # the caches: v bit for bit, k within the rounding to its code
    want_e = [np.clip(b.astype(int) - 127, Q.LO, Q.HI) for b in before[2:]]
    codes = [b.copy() for b in before[:2]]
    Q.append(codes[1], want_e[1], v.cpu().double().numpy(), slots, skip, bt)
    Q.append(codes[0], want_e[0], ref_k.numpy(), slots, skip, bt)
    got = [c.cpu().contiguous().view(torch.uint8).numpy() for c in (kc, vc, ks, vs)]
    touched = np.zeros((P, ps // bt), bool)
    written = np.zeros((P, ps), bool)
    for t, x in enumerate(slots):
        if 0 <= x < P * ps:
            touched[x // ps, x % ps // bt] = True
            written[x // ps, x % ps] = not skip[t]
    unknown = np.zeros((P, ps), bool)
    for t, x in enumerate(slots):
        if skip[t] and 0 <= x < P * ps:
            unknown[x // ps, x % ps] = True
    for c in (2, 3):  # untouched blocks keep their scale's byte
        same = np.where(touched[:, None], want_e[c - 2] + 127, before[c])
        if c == 3:
            assert (got[c] == same).all()
        else:
            assert (np.abs(got[c].astype(int) - same) <= 1)[np.broadcast_to(touched[:, None], same.shape)].all()
            assert (got[c] == same).mean() > 0.95 and (got[c] == same)[np.broadcast_to(~touched[:, None], same.shape)].all()
    known = np.broadcast_to(~unknown[:, None, :, None], got[1].shape)
    assert (got[1] == codes[1])[known].all()
    val = Q.values(torch.from_numpy(got[0]), torch.from_numpy(got[2]).view(Q.E8M0)).numpy()
    ref = Q.values(torch.from_numpy(codes[0]), torch.from_numpy((want_e[0] + 127).astype(np.uint8)).view(Q.E8M0)).numpy()
    e = np.repeat(np.exp2(got[2].astype(float) - 127), bt, 2)[..., None]
    # rows of the call against their values, within half a step; rows that a block held exactly where the scales agree
    exact = np.zeros(val.shape)
    for t, x in enumerate(slots):
        if 0 <= x < P * ps and not skip[t]:
            exact[x // ps, :, x % ps] = ref_k[t].numpy()
    w = np.broadcast_to(written[:, None, :, None], val.shape)
    ksize = 16.0 if qk else k.cpu().double().abs().max().item()
    assert (np.abs(val - exact) <= 1.001 * 2.0 ** -4 * np.abs(exact) + 2.0 ** -10 * e + 1e-5 * ksize)[w].all()
    same_e = np.repeat(got[2] == np.where(touched[:, None], want_e[0] + 127, before[2]), bt, 2)[..., None]
    assert (val == ref)[~w & known & np.broadcast_to(same_e, val.shape)].all()
    s.close()
    return bits


@pytest.mark.parametrize("Hq,Hkv,D,Rd,ps,bt,order", [
    (4, 1, 128, 128, 16, 16, "head"), (7, 7, 64, 32, 8, 1, "token"), (28, 4, 128, 64, 24, 8, "pair"),
    (3, 2, 96, 48, 4, 2, "padded"), (8, 2, 256, 64, 32, 32, "record"), (6, 2, 160, 160, 48, 24, "token"),
    (2, 1, 36, 10, 16, 4, "head"), (32, 8, 128, 128, 64, 64, "head"), (5, 5, 512, 2, 4, 4, "token"),
    (4, 2, 64, 64, 128, 128, "head"), (4, 2, 128, 32, 256, 256, "token")])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("qk", [False, True])
@pytest.mark.parametrize("dtype", ["BF16", "FP16"])
def test_write(S, Hq, Hkv, D, Rd, ps, bt, order, inter, qk, dtype):
    g = np.random.default_rng(D + ps + 3 * bt + inter)
    runs = [(0, 1), (5 % ps, 3), (ps - 1, 2), None, (0, 2 * ps + 3), (1 % ps, 1), (0, bt), (bt // 2, bt // 2 + 1), None, None]
    runs += [(int(g.integers(0, ps)), 1) for _ in range(9)]
    P = sum(-(-(r[0] + r[1]) // ps) for r in runs if r) + 3
    slots = slots_of(g, runs, P, ps, bt)
    bits = write_case(S, g, getattr(S, dtype), inter, qk, Hq, Hkv, D, Rd, ps, bt, order, slots, P)
    assert bits == 0


@pytest.mark.parametrize("k_size", [1e-9, 2.0 ** -20, 1.0, 3e4])
@pytest.mark.parametrize("variant", ["VARIANT_AUTO", "VARIANT_GENERIC"])
def test_write_scales_over_their_range(S, k_size, variant):
    """Zeros, tiny and large magnitudes, and blocks whose scale grows by much."""
    g = np.random.default_rng(5)
    slots = slots_of(g, [(3, 1), (0, 40), (7, 30), (15, 1)], 9, 16, 16)
    assert write_case(S, g, S.BF16, False, False, 4, 2, 128, 128, 16, 16, "head", slots, 9, k_size=k_size,
                      variant=getattr(S, variant)) == 0


@pytest.mark.parametrize("variant", ["VARIANT_AUTO", "VARIANT_GENERIC"])
@pytest.mark.parametrize("bt", [1, 16, 64])
def test_write_bad_positions_and_slots(S, variant, bt):
    g = np.random.default_rng(6)
    slots = slots_of(g, [(0, 70), (9, 5), None, (63, 2)], 8, 64, bt)
    slots[80 - 6] = 8 * 64  # past the cache
    bits = write_case(S, g, S.BF16, False, True, 4, 2, 128, 64, 64, bt, "head", slots, 8, bad_pos=(0, 5, 17, 71),
                      variant=getattr(S, variant))
    assert bits == S.DEVERR_POS | S.DEVERR_SLOT


@pytest.mark.parametrize("T", [1, 3, 17, 300, 2000])
@pytest.mark.parametrize("bt", [1, 8, 16, 32])
def test_write_many_tokens(S, T, bt):
    """Decode steps (a run per token) beside prompts, over the counts at which the split of the work changes."""
    g = np.random.default_rng(T + bt)
    runs, left = [], T
    while left > 0:
        n = min(left, int(g.choice([1, 1, 1, 1, 40, 300])))
        runs.append((int(g.integers(0, 32)), n))
        left -= n
    P = sum(-(-(r[0] + r[1]) // 32) for r in runs) + 1
    slots = slots_of(g, runs, P, 32, bt)
    assert write_case(S, g, S.FP16, False, False, 4, 2, 64, 64, 32, bt, "token", slots, P) == 0


def test_write_not_finite(S):
    """Infinities become the largest code under the largest scale; NaN stays and does not count for the scale."""
    for variant in (S.VARIANT_AUTO, S.VARIANT_GENERIC):
        s = S.Scm()
        s.register(S.make_spec(S.OP_ROPE_PAGED_KV8, S.BF16, [2, 1, 64, 64, 16, 16], 1, 64, variant=variant))
        q = torch.randn(4, 2, 64, device="cuda").bfloat16()
        k, v = torch.ones(4, 1, 64, device="cuda").bfloat16(), torch.ones(4, 1, 64, device="cuda").bfloat16()
        v[1, 0, 3], v[2, 0, 4] = float("nan"), float("-inf")
        kc, vc = (torch.zeros(3, 1, 16, 64, dtype=torch.uint8, device="cuda").view(Q.E4M3) for _ in range(2))
        ks, vs = (torch.full((3, 1, 1), 127, dtype=torch.uint8, device="cuda").view(Q.E8M0) for _ in range(2))
        args = S.make_args(S.OP_ROPE_PAGED_KV8, [q, k, v, i32([0] * 4), i32([0, 16, 17, 35]), S.rope_freqs(1e4, 64), q.clone(),
                                                 kc, vc, ks, vs], scalar=1.0)
        assert s.invoke(args, stream()) == (S.OK, 0)
        got, e = vc.cpu().float(), vs.cpu().view(torch.uint8).flatten().tolist()
        assert e == [127 - 8, 127 + 32, 127]
        assert (got[0, 0, 0] == 256).all() and (got[2, 0, 3] == 1).all()
        assert torch.isnan(got[1, 0, 0, 3]) and got[1, 0, 1, 4] == -448 and got[1, 0, 0, 0] == 0
        s.close()


# ---------------------------------------------------------------- reading back
@pytest.mark.parametrize("Hkv,D,ps,bt,order", [
    (1, 128, 16, 16, "head"), (7, 64, 8, 1, "token"), (4, 128, 24, 8, "pair"), (2, 96, 4, 2, "padded"),
    (2, 256, 32, 32, "record"), (2, 36, 16, 4, "head"), (8, 128, 64, 64, "token"), (1, 512, 4, 4, "token"), (3, 16, 16, 16, "head")])
@pytest.mark.parametrize("dtype", ["BF16", "FP16"])
@pytest.mark.parametrize("variant", ["VARIANT_AUTO", "VARIANT_GENERIC"])
def test_read(S, Hkv, D, ps, bt, order, dtype, variant):
    dt, g = getattr(S, dtype), np.random.default_rng(D + ps)
    first, new = [0, 3, 5, 0, 17, 1], [1, 0, 40, 33, 2, 0]
    b = Q.batch(g, new, [f + n for f, n in zip(first, new)], 1, Hkv, D, ps, bt, dt, order, tail=5)
    s = S.Scm()
    s.register(S.make_spec(S.OP_PAGED_READ8, dt, [Hkv, D, ps, bt], 1, 1 << 20, layout=S.LAYOUT_ANY, variant=getattr(S, variant),
                           align_bytes=16 if D % 16 == 0 else 2))
    T = sum(new) + 5
    outs = [torch.full((T, Hkv + 1, D), 7.0, dtype=R.TORCH[dt], device="cuda") for _ in range(2)]
    args = S.make_args(S.OP_PAGED_READ8, [b["kc"], b["vc"], b["ks"], b["vs"], b["table"], b["cu"], i32(first),
                                          *[o[:, :Hkv] for o in outs]])
    assert s.invoke(args, stream()) == (S.OK, 0), S.trident_scm_last_error()
    assert S.trident_scm_device_status(s.h, stream())[1] == 0
    table = b["table"].cpu().long()
    for o, c, sc in zip(outs, (b["kc"], b["vc"]), (b["ks"], b["vs"])):
        x, at = Q.values(c.view(torch.uint8), sc), 0
        for r, (f, n) in enumerate(zip(first, new)):
            j = torch.arange(f, f + n)
            want = x[table[r, j // ps], :, j % ps].to(R.TORCH[dt])
            assert torch.equal(o[at:at + n, :Hkv].cpu(), want)
            at += n
        assert (o[sum(new):] == 7.0).all() and (o[:, Hkv:] == 7.0).all()
    s.close()


@pytest.mark.parametrize("variant", ["VARIANT_AUTO", "VARIANT_GENERIC"])
def test_read_bad_places(S, variant):
    """A page or a position out of range gives rows of zeros and the status bit, and touches nothing else."""
    g = np.random.default_rng(1)
    b = Q.batch(g, [4, 4, 4], [20, 20, 20], 1, 2, 64, 16, 16, S.BF16)
    b["table"][1, 1] = 1 << 30
    s = S.Scm()
    s.register(S.make_spec(S.OP_PAGED_READ8, S.BF16, [2, 64, 16, 16], 1, 64, variant=getattr(S, variant)))
    M = b["table"].shape[1]
    k, v = (torch.full((12, 2, 64), 7.0, device="cuda").bfloat16() for _ in range(2))
    args = S.make_args(S.OP_PAGED_READ8, [b["kc"], b["vc"], b["ks"], b["vs"], b["table"], b["cu"], i32([-2, 16, 16 * M - 1]), k, v])
    assert s.invoke(args, stream()) == (S.OK, 0)
    assert S.trident_scm_device_status(s.h, stream())[1] == S.DEVERR_TABLE
    for o in (k, v):
        assert (o[:2] == 0).all() and (o[4:8] == 0).all() and (o[9:] == 0).all() and (o[2:4] != 0).any()
    s.close()


def test_read_many_requests(S):
    g = np.random.default_rng(2)
    new = [int(x) for x in g.integers(0, 4, 1500)]
    first = [int(x) for x in g.integers(0, 9, 1500)]
    b = Q.batch(g, new, [f + n for f, n in zip(first, new)], 1, 1, 64, 8, 8, S.FP16)
    s = S.Scm()
    s.register(S.make_spec(S.OP_PAGED_READ8, S.FP16, [1, 64, 8, 8], 1, 1 << 20))
    k, v = (torch.zeros(sum(new), 1, 64, dtype=torch.float16, device="cuda") for _ in range(2))
    assert s.invoke(S.make_args(S.OP_PAGED_READ8, [b["kc"], b["vc"], b["ks"], b["vs"], b["table"], b["cu"], i32(first), k, v]),
                    stream()) == (S.OK, 0)
    r = torch.repeat_interleave(torch.arange(1500), torch.tensor(new))
    j = torch.tensor(first)[r] + torch.arange(sum(new)) - b["cu"].cpu().long()[r]
    for o, c, sc in ((k, "kc", "ks"), (v, "vc", "vs")):
        x = Q.values(b[c].view(torch.uint8), b[sc])
        assert torch.equal(o.cpu(), x[b["table"].cpu().long()[r, j // 8], :, j % 8].half())
    s.close()


# ---------------------------------------------------------------- attention
def attend(S, b, Hq, Hkv, D, ps, bt, dt, scale, variant=None, twice=True):
    s = S.Scm(flags=S.OPT_PDL)
    i = s.register(S.make_spec(S.OP_PAGED_ATTN8, dt, [Hq, Hkv, D, ps, bt], 1, 1 << 20, layout=S.LAYOUT_ANY,
                               align_bytes=16 if D % 16 == 0 else 2,
                               variant=S.VARIANT_AUTO if variant is None else variant))
    work = torch.zeros(s.workspace(i), device="cuda")
    args = S.make_args(S.OP_PAGED_ATTN8, [b["q"], b["kc"], b["vc"], b["ks"], b["vs"], b["table"], b["cu"], b["kv"], work,
                                          b["out"], b["lse"]], scalar=scale)
    assert s.invoke(args, stream()) == (S.OK, 0), S.trident_scm_last_error()
    out, lse = b["out"].clone(), b["lse"].clone()
    if twice:  # the workspace is left ready, and the result does not depend on which block ends last
        assert s.invoke(args, stream()) == (S.OK, 0)
        assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(b["out"])) and \
            torch.equal(torch.nan_to_num(lse), torch.nan_to_num(b["lse"]))
    assert S.trident_scm_device_status(s.h, stream())[1] == 0
    s.close()
    return out, lse


def check(b, ps, dt, scale, out, lse):
    ref, want, wgt, level = Q.reference(b, ps, scale)
    tol = Q.tolerance(ref, wgt, level, dt, max(b["kv"].tolist(), default=0))
    err = (out.cpu().double() - ref).abs()
    assert (err <= tol).all(), ((err - tol).max(), (err / tol.clamp(min=1e-300)).max())
    none = torch.isinf(want)
    assert torch.equal(torch.isinf(lse.cpu()), none)
    assert ((lse.cpu().double() - want)[~none].abs() <= R.LSE_TOLERANCE).all()


@pytest.mark.parametrize("Hq,Hkv,D,ps,bt,order", [
    (8, 2, 128, 16, 16, "head"), (7, 1, 64, 8, 1, "token"), (28, 4, 128, 24, 8, "pair"), (4, 4, 256, 32, 32, "record"),
    (6, 2, 96, 4, 2, "padded"), (8, 1, 128, 64, 32, "token"), (16, 2, 64, 128, 128, "head"), (40, 8, 128, 16, 4, "head"),
    (3, 1, 36, 16, 16, "head"), (8, 2, 256, 16, 1, "token")])
@pytest.mark.parametrize("dtype", ["BF16", "FP16"])
@pytest.mark.parametrize("new,kv", [
    ([1], [1]), ([1, 1, 1], [5, 300, 77]), ([1, 0, 4, 9], [0, 3, 4, 200]), ([37], [64]), ([200, 1, 30], [260, 900, 17]),
    ([5, 5], [3, 5])])
def test_attention(S, Hq, Hkv, D, ps, bt, order, dtype, new, kv):
    dt, g = getattr(S, dtype), np.random.default_rng(D + sum(kv))
    b = Q.batch(g, new, kv, Hq, Hkv, D, ps, bt, dt, order, tail=2, strided=D != 128)
    scale = D ** -0.5
    out, lse = attend(S, b, Hq, Hkv, D, ps, bt, dt, scale)
    check(b, ps, dt, scale, out, lse)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("variant", ["VARIANT_AUTO", "VARIANT_GENERIC"])
@pytest.mark.parametrize("new", [1, 3, 150])
def test_attention_scales_far_apart(S, D, variant, new):
    """Value scales from 2^-32 to 2^32 in one request, the small ones where the weights are: what a block adds counts by
    its products, not by its weight alone."""
    dt, g = S.BF16, np.random.default_rng(new)
    L = 700
    b = Q.batch(g, [new], [L], 4, 2, D, 16, 16, dt)
    e = g.integers(-32, 33, b["vs"].shape)
    b["vs"] = Q.scale_bytes(torch.from_numpy(e)).cuda()
    ek = torch.from_numpy(g.integers(-32, -4, b["ks"].shape))  # scores stay moderate
    b["ks"] = Q.scale_bytes(ek).cuda()
    scale = D ** -0.5
    out, lse = attend(S, b, 4, 2, D, 16, 16, dt, scale, getattr(S, variant))
    check(b, 16, dt, scale, out, lse)


@pytest.mark.parametrize("variant", ["VARIANT_AUTO", "VARIANT_GENERIC"])
@pytest.mark.parametrize("new", [1, 140])
def test_attention_large_values_of_no_weight(S, variant, new):
    """A block of huge values that the softmax gives next to nothing, beside small ones that it gives all: both show."""
    D, L, g = 128, 96, np.random.default_rng(3)
    b = Q.batch(g, [new], [L + new], 4, 1, D, 16, 16, S.BF16, size=1.0)
    t = b["table"].cpu().long()[0]
    b["q"].fill_(1.0)
    for j in range(-(-(L + new) // 16)):
        key = -2.0 if j == 2 else 0.25  # scores: 2 * 128^0.5 apart
        b["kc"].view(torch.uint8)[t[j]] = int(Q.codes_of(np.full(1, key))[0])
        b["ks"].view(torch.uint8)[t[j]] = 127
        b["vs"].view(torch.uint8)[t[j]] = 127 + (30 if j == 2 else -30)
    out, lse = attend(S, b, 4, 1, D, 16, 16, S.BF16, D ** -0.5, getattr(S, variant))
    check(b, 16, S.BF16, D ** -0.5, out, lse)


@pytest.mark.parametrize("new,kv", [([1] * 9, [2000, 5, 900, 4000, 1, 700, 3333, 64, 1500]), ([600], [2500]),
                                    ([1, 400, 1, 7, 1], [900, 1300, 3000, 64, 2000])])
@pytest.mark.parametrize("D,ps,bt", [(128, 16, 16), (64, 32, 8), (256, 64, 64), (128, 128, 1)])
@pytest.mark.parametrize("dtype", ["BF16", "FP16"])
def test_attention_long(S, new, kv, D, ps, bt, dtype):
    dt, g = getattr(S, dtype), np.random.default_rng(D + ps + len(new))
    b = Q.batch(g, new, kv, 8, 2, D, ps, bt, dt)
    out, lse = attend(S, b, 8, 2, D, ps, bt, dt, D ** -0.5)
    check(b, ps, dt, D ** -0.5, out, lse)


@pytest.mark.parametrize("kv", [[260, 385], [384, 400], [300, 527], [200, 1025], [416, 1039]])
@pytest.mark.parametrize("D,ps,bt,G", [(64, 8, 8, 4), (64, 128, 32, 7), (128, 16, 16, 4), (128, 8, 2, 8), (128, 256, 128, 3),
                                       (256, 64, 16, 4), (256, 16, 1, 2), (256, 128, 64, 4)])
@pytest.mark.parametrize("dtype", ["BF16", "FP16"])
def test_attention_tiles(S, kv, D, ps, bt, G, dtype):
    """Requests of many rows whose keys end at, before and behind a tile's or a 16's border, from the first token on (kv as
    many as rows: 300 and 260) or with fewer keys than rows (rows that see none), in pages below, of and above a tile."""
    dt, g = getattr(S, dtype), np.random.default_rng(D + ps + sum(kv))
    b = Q.batch(g, [260, 300], kv, G, 1, D, ps, bt, dt, tail=1)
    out, lse = attend(S, b, G, 1, D, ps, bt, dt, D ** -0.5)
    check(b, ps, dt, D ** -0.5, out, lse)


@pytest.mark.parametrize("new", [1, 130])
@pytest.mark.parametrize("what", ["nan", "inf"])
def test_attention_row_not_finite(S, new, what):
    """A row of q that is not finite makes its own out and lse NaN, and nobody else's."""
    g = np.random.default_rng(8)
    b = Q.batch(g, [new, new], [300, 300], 4, 1, 128, 16, 16, S.BF16)
    b["q"][0, 1, 5] = float(what)
    out, lse = attend(S, b, 4, 1, 128, 16, 16, S.BF16, 0.1)
    assert torch.isnan(out[0, 1]).all() and torch.isnan(lse[0, 1])
    b["q"][0, 1, 5] = 0
    ref, want, _, _ = Q.reference(b, 16, 0.1)
    keep = torch.ones(out.shape[:2], dtype=torch.bool)
    keep[0, 1] = False
    assert torch.isfinite(out.cpu()[keep]).all() and (out.cpu().double() - ref)[keep].abs().max() < 0.2
    assert (lse.cpu().double() - want)[keep].abs().max() < R.LSE_TOLERANCE
