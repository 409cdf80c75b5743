"""The paged ops on the GPU against their formulas in 64 bits."""
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


def i32(x):
    return torch.tensor(np.asarray(x, np.int32)).cuda()


# ---------------------------------------------------------------- page map
def run_map(S, ctx, new, free, head, table, ps, N, expect_bits=0):
    s = S.Scm()
    s.register(S.make_spec(S.OP_PAGE_MAP, S.I32, [], 1, 1 << 20, layout=S.LAYOUT_ANY, align_bytes=4))
    B, M = table.shape
    wide = torch.full((B, M + 3), -7, dtype=torch.int32, device="cuda")  # rows of a wider table
    wide[:, :M] = i32(table)
    out = [torch.full((n,), -99, dtype=torch.int32, device="cuda") for n in (B + 1, B, N, N, 1)]
    args = S.make_args(S.OP_PAGE_MAP, [i32(ctx), i32(new), i32(free), i32([head]), wide[:, :M], *out], scalar=ps)
    for _ in range(2):  # the same call again gives the same (its inputs stay)
        assert s.invoke(args, stream()) == (S.OK, 0), S.trident_scm_last_error()
    bits = S.trident_scm_device_status(s.h, stream())[1]
    cu, kv, pos, slot, at, want, ok = R.page_map(ctx, new, free, head, table, ps, N)
    got = [x.tolist() for x in out]
    assert got == [cu, kv, pos, slot, [at]]
    assert (wide[:, :M].cpu().numpy() == want).all() and (wide[:, M:] == -7).all()
    assert bits == expect_bits and ok == (not expect_bits & S.DEVERR_PAGES)
    s.close()


def random_map(g, B, ps, ctx_hi, new_hi, M_extra=2):
    ctx = [int(x) for x in g.integers(0, ctx_hi + 1, B)]
    new = [int(x) for x in g.integers(0, new_hi + 1, B)]
    need = [-(-(c + n) // ps) for c, n in zip(ctx, new)]
    have = [-(-c // ps) for c in ctx]
    P = sum(need) + 40
    ids = g.permutation(P).astype(np.int32)
    table = np.full((B, max(need) + M_extra), -1, np.int32)
    at = 0
    for b in range(B):
        table[b, :have[b]] = ids[at:at + have[b]]
        at += have[b]
    return ctx, new, ids[at:], table


@pytest.mark.parametrize("B,ps,ctx_hi,new_hi,pad,head", [
    (1, 16, 0, 1, 0, 0), (1, 1, 5, 3, 7, 2), (64, 16, 8192, 1, 0, 5), (64, 16, 100, 0, 3, 0), (255, 24, 300, 9, 1, 0),
    (256, 8, 64, 64, 5, 1), (257, 32, 500, 40, 0, 0), (1000, 16, 70, 33, 100, 3), (3, 65536, 70000, 5000, 2, 0)])
def test_page_map(S, B, ps, ctx_hi, new_hi, pad, head):
    g = np.random.default_rng(B + ps)
    ctx, new, free, table = random_map(g, B, ps, ctx_hi, new_hi)
    run_map(S, ctx, new, free, head, table, ps, sum(new) + pad)


def test_page_map_one_long_chunk_among_decodes(S):
    g = np.random.default_rng(5)
    ctx, new, _, _ = random_map(g, 300, 16, 200, 1)
    new[137] = 5000
    need = [-(-(c + n) // 16) for c, n in zip(ctx, new)]
    table = np.full((300, max(need)), -1, np.int32)
    ids = g.permutation(sum(need)).astype(np.int32)
    at = 0
    for b, c in enumerate(ctx):
        table[b, :-(-c // 16)] = ids[at:at + -(-c // 16)]
        at += -(-c // 16)
    run_map(S, ctx, new, ids[at:], 0, table, 16, sum(new))


@pytest.mark.parametrize("what", ["tokens", "pages", "columns", "negative ctx", "negative new", "head", "huge"])
def test_page_map_hands_out_all_or_nothing(S, what):
    g = np.random.default_rng(3)
    ctx, new, free, table = random_map(g, 40, 16, 90, 20, M_extra=0)
    N, head = sum(new) + 4, 0
    if what == "tokens": N = sum(new) - 1
    if what == "pages": free = free[:sum(-(-(c + n) // 16) - -(-c // 16) for c, n in zip(ctx, new)) - 1]
    if what == "columns": table = table[:, :-1]
    if what == "negative ctx": ctx[7] = -1
    if what == "negative new": new[39] = -3
    if what == "head": head = len(free) + 1
    if what == "huge": new[3] = 2 ** 31 - 1
    run_map(S, ctx, new, free, head, table, 16, N, expect_bits=S.DEVERR_PAGES)


def test_page_map_table_entry_that_is_no_page(S):
    table = np.array([[4, -5, -1], [3, 2 ** 30, -1]], np.int32)
    run_map(S, [20, 17], [2, 3], np.array([9], np.int32), 0, table, 16, 6, expect_bits=S.DEVERR_TABLE)


# ---------------------------------------------------------------- paged RoPE
OPS = {(False, False): "OP_ROPE_PAGED_KV", (True, False): "OP_ROPE_PAGED_KV_INTERLEAVED",
       (False, True): "OP_QKNORM_ROPE_PAGED_KV", (True, True): "OP_QKNORM_ROPE_PAGED_KV_INTERLEAVED"}


@pytest.mark.parametrize("T,Hq,Hkv,D,Rd,ps,order", [
    (1, 4, 1, 128, 128, 16, "head"), (5, 7, 7, 64, 32, 8, "token"), (65, 28, 4, 128, 64, 24, "pair"),
    (33, 3, 2, 96, 48, 1, "padded"), (40, 8, 2, 256, 64, 32, "head"), (700, 6, 2, 160, 160, 16, "token"),
    (9, 2, 1, 36, 10, 16, "head"), (1030, 32, 8, 128, 128, 16, "head"), (3, 5, 5, 512, 2, 4, "token")])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("qk", [False, True])
@pytest.mark.parametrize("dtype", ["BF16", "FP16"])
def test_rope_paged(S, T, Hq, Hkv, D, Rd, ps, order, inter, qk, dtype):
    dt = getattr(S, dtype)
    g = np.random.default_rng(T * 7 + D + inter)
    op = getattr(S, OPS[inter, qk])
    s = S.Scm()
    s.register(S.make_spec(op, dt, [Hq, Hkv, D, Rd, ps], 1, 1 << 20, layout=S.LAYOUT_ANY))
    s.register(S.make_spec(op, dt, [Hq, Hkv, D, Rd, ps], 1, 1 << 20, layout=S.LAYOUT_ANY, align_bytes=2,
                           variant=S.VARIANT_GENERIC))
    qkv = torch.from_numpy(g.standard_normal((T, Hq + 2 * Hkv, D), dtype=np.float32)).to(R.TORCH[dt]).cuda()
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    P = -(-T // ps) + 2
    kc, vc = R.pool(g, P, Hkv, ps, D, dt, order)
    slots = g.permutation(P * ps)[:T].astype(np.int32)
    slots[g.random(T) < 0.1] = -1  # padding
    pos = g.integers(0, 1 << 24, T).astype(np.int32)
    pos[: T // 2] = g.integers(0, 9000, T // 2)
    mag = 1.25
    freqs = S.rope_freqs(10000.0, Rd, S.ROPE_LINEAR, 2.0)
    gam = [torch.from_numpy(g.normal(1, 0.1, D).astype(np.float32)).cuda() for _ in range(2)] if qk else []
    aligned = D % 8 == 0
    f = freqs.cpu().double().sum(1)
    x64 = qkv.cpu().double()
    want_q = R.rotate(x64[:, :Hq], torch.from_numpy(pos), f, mag, inter, gam[0].cpu().double() if qk else None, 1e-6)
    want_k = R.rotate(x64[:, Hq:Hq + Hkv], torch.from_numpy(pos), f, mag, inter, gam[1].cpu().double() if qk else None, 1e-6)
    # the output's rounding, and 8e-6 of the pair's size: sine and cosine to 2^-20 and the angle's reduction,
    # with 2^-21 more for the norm's factor and the products
    size = lambda w: w.abs().amax(-1, keepdim=True) * 2 ** 0.5 * 8e-6  # noqa: E731
    u = R.UNIT[dt]
    live = torch.from_numpy(slots >= 0)
    page, at = torch.from_numpy(slots).long() // ps, torch.from_numpy(slots).long() % ps
    for index in ([0, 1] if aligned else [1]):
        kc2, vc2 = kc.clone(memory_format=torch.preserve_format), vc.clone(memory_format=torch.preserve_format)
        if order in ("pair", "padded"):
            kc2, vc2 = kc, vc
        before_k, before_v = kc2.cpu().clone(), vc2.cpu().clone()
        q_out = torch.full((T, Hq, D), float("nan"), dtype=R.TORCH[dt], device="cuda")
        args = S.make_args(op, [q, k, v, i32(pos), i32(slots), freqs, q_out, kc2, vc2, *gam], eps=1e-6, scalar=mag)
        if index == 1:  # one element past a 16-byte boundary: the version of any alignment
            odd = torch.empty(T * Hq * D + 1, dtype=R.TORCH[dt], device="cuda")[1:].view(T, Hq, D)
            q_out = odd.fill_(float("nan"))
            args = S.make_args(op, [q, k, v, i32(pos), i32(slots), freqs, q_out, kc2, vc2, *gam], eps=1e-6, scalar=mag)
        assert s.invoke(args, stream()) == (S.OK, index), S.trident_scm_last_error()
        assert S.trident_scm_device_status(s.h, stream())[1] == 0
        got = q_out.cpu().double()
        assert ((got - want_q).abs() <= u * want_q.abs() * 1.01 + size(want_q) + 2.0 ** -25).all()
        gk, gv = kc2.cpu(), vc2.cpu()
        new_k = gk[page[live], :, at[live]].double()
        w = want_k[live]
        assert ((new_k - w).abs() <= u * w.abs() * 1.01 + size(w) + 2.0 ** -25).all()
        assert torch.equal(gv[page[live], :, at[live]], v.cpu()[live])
        before_k[page[live], :, at[live]] = gk[page[live], :, at[live]]  # nothing else was written
        before_v[page[live], :, at[live]] = gv[page[live], :, at[live]]
        assert torch.equal(gk, before_k) and torch.equal(gv, before_v)
    s.close()


def test_rope_paged_in_place_and_bad_rows(S):
    g = np.random.default_rng(1)
    T, Hq, Hkv, D, ps, P = 12, 4, 2, 64, 16, 3
    for variant in (S.VARIANT_VECTOR, S.VARIANT_GENERIC):
        s = S.Scm()
        s.register(S.make_spec(S.OP_ROPE_PAGED_KV, S.BF16, [Hq, Hkv, D, D, ps], 1, 64, variant=variant))
        q, k, v = (torch.from_numpy(g.standard_normal((T, h, D), dtype=np.float32)).bfloat16().cuda() for h in (Hq, Hkv, Hkv))
        kc, vc = R.pool(g, P, Hkv, ps, D, S.BF16, "head")
        pos, slots = np.arange(T) * 3, np.arange(T)
        pos[2], pos[5], slots[7], slots[9] = -1, 1 << 24, P * ps, 2 ** 31 - 1
        freqs = S.rope_freqs(10000.0, D)
        old, kc0, vc0 = q.cpu().clone(), kc.cpu().clone(), vc.cpu().clone()
        want = R.rotate(old.double(), torch.from_numpy(pos), freqs.cpu().double().sum(1), 1.0, False)
        assert s.invoke(S.make_args(S.OP_ROPE_PAGED_KV, [q, k, v, i32(pos), i32(slots), freqs, q, kc, vc], scalar=1.0),
                        stream()) == (S.OK, 0)
        assert S.trident_scm_device_status(s.h, stream())[1] == S.DEVERR_POS | S.DEVERR_SLOT
        got = q.cpu()
        skip = [2, 5]
        assert torch.equal(got[skip], old[skip])
        rest = [t for t in range(T) if t not in skip]
        tol = 2.0 ** -8 * want.abs() * 1.01 + 8e-6 * want.abs().amax(-1, keepdim=True) * 2 ** 0.5
        assert ((got.double() - want).abs() <= tol)[rest].all()
        for t in (2, 5, 7, 9):  # their slots (where they are one) were not written
            assert torch.equal(kc.cpu()[0, :, t], kc0[0, :, t]) and torch.equal(vc.cpu()[0, :, t], vc0[0, :, t])
        assert torch.equal(kc.cpu()[1:], kc0[1:])
        s.close()


# ---------------------------------------------------------------- paged attention
def check_attn(S, b, Hq, Hkv, D, ps, dt, scale, tail, s, index, work, bits=0):
    args = S.make_args(S.OP_PAGED_ATTN, [b["q"], b["kc"], b["vc"], b["table"], b["cu"], b["kv"], work, b["out"], b["lse"]],
                       scalar=scale)
    assert s.invoke(args, stream()) == (S.OK, index), S.trident_scm_last_error()
    assert S.trident_scm_device_status(s.h, stream())[1] == bits
    kv = b["kv"].tolist()
    out, lse, wgt = R.attention(b["q"].cpu(), b["kc"].cpu(), b["vc"].cpu(), b["table"].cpu(), b["cu"].tolist(), kv, ps, scale)
    got, got_lse = b["out"].cpu().double(), b["lse"].cpu().double()
    assert torch.isfinite(got).all()
    tol = R.attn_tolerance(out, wgt, dt, max(kv + [0]), 5.0)
    worst = ((got - out).abs() - tol).max().item()
    assert worst <= 0, (worst, (got - out).abs().max().item())
    none = torch.isinf(lse)
    assert torch.equal(torch.isinf(got_lse) & (got_lse < 0), none)
    assert (got[none] == 0).all()
    assert ((got_lse - lse).abs() <= R.LSE_TOLERANCE + 2.0 ** -21 * lse.abs())[~none].all()
    return got


def attn_scm(S, dt, Hq, Hkv, D, ps, variant):
    s = S.Scm(flags=S.OPT_PDL)
    index = s.register(S.make_spec(S.OP_PAGED_ATTN, dt, [Hq, Hkv, D, ps], 1, 1 << 20, layout=S.LAYOUT_ANY,
                                   align_bytes=2 if variant == S.VARIANT_GENERIC else 16, variant=variant))
    return s, index, torch.zeros(s.workspace(index), device="cuda")


SHAPES = [  # new tokens, keys, Hq, Hkv, D, ps, order, rows past the last request, strided
    ([1], [1], 4, 1, 128, 16, "head", 0, False),
    ([1], [17], 8, 8, 64, 16, "token", 2, False),
    ([1, 1, 1], [700, 33, 64], 32, 8, 128, 16, "head", 0, True),
    ([1] * 40, list(range(0, 400, 10)), 8, 2, 128, 8, "pair", 3, False),
    ([3, 0, 5, 1, 0], [10, 40, 5, 0, 0], 28, 4, 64, 24, "token", 0, False),
    ([4, 7], [2, 7], 6, 2, 128, 32, "head", 1, False),           # rows before the first key: empty
    ([130], [1500], 8, 2, 128, 64, "padded", 0, True),
    ([300, 1, 40], [300, 900, 777], 16, 4, 64, 16, "head", 0, False),
    ([257], [258], 5, 1, 128, 128, "token", 5, False),
    ([33, 2], [600, 129], 4, 2, 256, 16, "head", 0, False),
    ([12], [3000], 40, 8, 128, 1, "head", 0, False),
    ([200], [5000], 32, 8, 128, 16, "head", 0, False),
    ([16, 17], [1000, 1024], 7, 1, 64, 256, "head", 0, False),
]


@pytest.mark.parametrize("new,kv,Hq,Hkv,D,ps,order,tail,strided", SHAPES)
@pytest.mark.parametrize("dtype", ["BF16", "FP16"])
@pytest.mark.parametrize("variant", ["AUTO", "GENERIC"])
def test_paged_attention(S, new, kv, Hq, Hkv, D, ps, order, tail, strided, dtype, variant):
    dt = getattr(S, dtype)
    g = np.random.default_rng(len(kv) * 31 + D + ps)
    s, index, work = attn_scm(S, dt, Hq, Hkv, D, ps, getattr(S, "VARIANT_" + variant))
    b = R.batch(g, new, kv, Hq, Hkv, D, ps, dt, order, tail, strided)
    first = check_attn(S, b, Hq, Hkv, D, ps, dt, 1.0 / D ** 0.5, tail, s, index, work)
    b["out"].fill_(float("nan"))  # the workspace serves the next call, and the result is the same bits
    again = check_attn(S, b, Hq, Hkv, D, ps, dt, 1.0 / D ** 0.5, tail, s, index, work)
    assert torch.equal(first, again)
    s.close()


TILE_SHAPES = [  # enough rows and keys for the tile kernel; as above
    ([128], [900], 8, 1, 256, 16, "head", 0, False),             # heads of 256
    ([70, 90, 1], [1100, 800, 300], 16, 4, 256, 64, "token", 3, True),
    ([120, 200], [1600, 1024], 7, 1, 64, 256, "pair", 0, False),  # seven heads per group, pages longer than a tile
    ([500, 3, 64], [500, 2000, 3000], 8, 2, 128, 8, "padded", 1, False),
    ([400, 1, 1, 0, 90], [390, 600, 31, 0, 2111], 12, 2, 128, 32, "head", 0, False),  # ten rows before the first key
    ([129], [9000], 4, 1, 128, 16, "head", 0, False),            # one unit over all blocks: joined in groups
    ([40] * 20, [2000 + 13 * k for k in range(20)], 8, 1, 128, 16, "head", 0, False),
    ([1000], [1001], 64, 2, 64, 128, "head", 7, False),          # more units than blocks
]


@pytest.mark.parametrize("new,kv,Hq,Hkv,D,ps,order,tail,strided", TILE_SHAPES)
@pytest.mark.parametrize("dtype", ["BF16", "FP16"])
def test_paged_attention_many_rows(S, new, kv, Hq, Hkv, D, ps, order, tail, strided, dtype):
    test_paged_attention(S, new, kv, Hq, Hkv, D, ps, order, tail, strided, dtype, "AUTO")


def test_paged_attention_many_requests(S):
    """More requests than a block has threads, in both kernels."""
    g = np.random.default_rng(12)
    new, kv = [1] * 300, [int(x) for x in g.integers(0, 200, 300)]
    test_paged_attention(S, new, kv, 4, 1, 64, 16, "head", 0, False, "BF16", "AUTO")
    new = [30 if k % 3 else 1 for k in range(420)]
    test_paged_attention(S, new, [460 + k % 7 for k in range(420)], 8, 1, 128, 16, "head", 0, False, "FP16", "AUTO")


def test_paged_attention_without_requests_or_pages(S):
    Hq, Hkv, D, ps = 8, 2, 128, 16
    s, index, work = attn_scm(S, S.BF16, Hq, Hkv, D, ps, S.VARIANT_AUTO)
    g = np.random.default_rng(0)
    kc, vc = R.pool(g, 2, Hkv, ps, D, S.BF16, "head")
    q = torch.randn(400, Hq, D, device="cuda").bfloat16()
    for B, M in ((0, 4), (3, 0)):
        out, lse = torch.full_like(q, float("nan")), torch.zeros(400, Hq, device="cuda")
        cu = i32([0] * (B + 1) if B == 0 else [0, 100, 300, 400])
        args = S.make_args(S.OP_PAGED_ATTN, [q, kc, vc, torch.zeros(B, M, dtype=torch.int32, device="cuda"), cu,
                                             torch.zeros(B, dtype=torch.int32, device="cuda"), work, out, lse], scalar=1.0)
        assert s.invoke(args, stream()) == (S.OK, index), S.trident_scm_last_error()
        assert S.trident_scm_device_status(s.h, stream())[1] == 0
        assert (out == 0).all() and (lse == -float("inf")).all()
    s.close()


def test_paged_attention_workspace_is_checked(S):
    s, index, work = attn_scm(S, S.BF16, 8, 2, 128, 16, S.VARIANT_AUTO)
    b = R.batch(np.random.default_rng(0), [1], [40], 8, 2, 128, 16, S.BF16)
    ts = [b["q"], b["kc"], b["vc"], b["table"], b["cu"], b["kv"], work[:-1], b["out"], b["lse"]]
    assert s.invoke(S.make_args(S.OP_PAGED_ATTN, ts, scalar=1.0), stream())[0] == S.ERR_INVALID
    s.close()


def test_paged_attention_both_kernels_in_a_graph_and_on_two_streams(S):
    """A call that launches both kernels, captured and replayed; and two calls at once with a workspace each."""
    Hq, Hkv, D, ps = 16, 4, 128, 16
    s, index, work = attn_scm(S, S.BF16, Hq, Hkv, D, ps, S.VARIANT_AUTO)
    b = [R.batch(np.random.default_rng(k), [1, 300, 1, 4], [700, 900, 33, 1200], Hq, Hkv, D, ps, S.BF16) for k in range(2)]
    works = [work, torch.zeros_like(work)]
    refs = [R.attention(x["q"].cpu(), x["kc"].cpu(), x["vc"].cpu(), x["table"].cpu(), x["cu"].tolist(), x["kv"].tolist(), ps,
                        0.09) for x in b]
    args = [S.make_args(S.OP_PAGED_ATTN, [x["q"], x["kc"], x["vc"], x["table"], x["cu"], x["kv"], w, x["out"], x["lse"]],
                        scalar=0.09) for x, w in zip(b, works)]

    def check():
        torch.cuda.synchronize()
        assert S.trident_scm_device_status(s.h, stream())[1] == 0
        for x, (out, lse, wgt) in zip(b, refs):
            assert ((x["out"].cpu().double() - out).abs() <= R.attn_tolerance(out, wgt, S.BF16, 1200, 5.0)).all()
            x["out"].fill_(float("nan"))
        torch.cuda.synchronize()

    side = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for a, st in zip(args, side):
            assert s.invoke(a, st.cuda_stream) == (S.OK, index)
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side[0]):
        for _ in range(3):
            for a in args:
                assert s.invoke(a, torch.cuda.current_stream().cuda_stream) == (S.OK, index)
    for _ in range(2):
        graph.replay()
        check()
    s.close()


def test_paged_attention_reports_a_wait_that_ran_out(S):
    """The tile kernel's first wait for scores gives up at once: status bit, nothing written; with the workspace
    zeroed again the next call is right."""
    Hq, Hkv, D, ps = 8, 2, 128, 16
    b = R.batch(np.random.default_rng(6), [300], [2000], Hq, Hkv, D, ps, S.BF16)
    s = S.Scm(flags=S.OPT_TEST_WAIT_TIMEOUT)
    index = s.register(S.make_spec(S.OP_PAGED_ATTN, S.BF16, [Hq, Hkv, D, ps], 1, 1 << 20))
    work = torch.zeros(s.workspace(index), device="cuda")
    args = S.make_args(S.OP_PAGED_ATTN, [b["q"], b["kc"], b["vc"], b["table"], b["cu"], b["kv"], work, b["out"], b["lse"]],
                       scalar=0.1)
    assert s.invoke(args, stream()) == (S.OK, index)
    assert S.trident_scm_device_status(s.h, stream())[1] == S.DEVERR_TIMEOUT
    assert torch.isnan(b["out"]).all() and torch.isnan(b["lse"]).all()
    s.close()
    s, index, _ = attn_scm(S, S.BF16, Hq, Hkv, D, ps, S.VARIANT_AUTO)
    work.zero_()
    check_attn(S, b, Hq, Hkv, D, ps, S.BF16, 0.1, 0, s, index, work)
    s.close()


def far_pool(P, Hkv, ps, D):
    """k and v of one buffer whose pages start 2^28 elements apart, v's 2^27 behind k's."""
    base = torch.empty(P << 28, dtype=torch.bfloat16, device="cuda")
    return tuple(base.as_strided((P, Hkv, ps, D), (1 << 28, ps * D, D, 1), at) for at in (0, 1 << 27))


@pytest.mark.parametrize("variant", ["AUTO", "GENERIC"])
@pytest.mark.parametrize("new,kv,ps,row", [([1, 4], [700, 330], 64, 1 << 29), ([38], [21000], 2048, 1 << 26)])
def test_offsets_past_32_bits(S, new, kv, ps, row, variant):
    """Pages and rows of q beyond 2^31 elements: the same bits as from dense tensors, which are
    checked against the formula."""
    g = np.random.default_rng(77)
    Hq, Hkv, D, dt = 32, 2, 128, S.BF16
    s, index, work = attn_scm(S, dt, Hq, Hkv, D, ps, getattr(S, "VARIANT_" + variant))
    b = R.batch(g, new, kv, Hq, Hkv, D, ps, dt, spare=7)
    P, T = b["kc"].shape[0], b["q"].shape[0]
    dense = check_attn(S, b, Hq, Hkv, D, ps, dt, 1.0 / D ** 0.5, 0, s, index, work)
    far = dict(b, out=torch.full_like(b["out"], float("nan")))
    far["kc"], far["vc"] = far_pool(P, Hkv, ps, D)
    far["kc"].copy_(b["kc"])
    far["vc"].copy_(b["vc"])
    far["q"] = torch.empty(T * row, dtype=torch.bfloat16, device="cuda").as_strided((T, Hq, D), (row, D, 1))
    far["q"].copy_(b["q"])
    used = b["table"][b["table"] < P].max().item()
    assert used << 28 >= 1 << 31 and (T - 1) * row >= 1 << 31
    assert torch.equal(check_attn(S, far, Hq, Hkv, D, ps, dt, 1.0 / D ** 0.5, 0, s, index, work), dense)
    s.close()


@pytest.mark.parametrize("variant", ["AUTO", "GENERIC"])
def test_rope_paged_offsets_past_32_bits(S, variant):
    g = np.random.default_rng(78)
    T, Hq, Hkv, D, ps, P = 35, 4, 2, 128, 16, 18
    s = S.Scm()
    s.register(S.make_spec(S.OP_ROPE_PAGED_KV, S.BF16, [Hq, Hkv, D, D, ps], 1, 64, layout=S.LAYOUT_ANY,
                           variant=getattr(S, "VARIANT_" + variant)))
    q, k, v = (torch.from_numpy(g.standard_normal((T, h, D), dtype=np.float32)).bfloat16().cuda() for h in (Hq, Hkv, Hkv))
    far_q = torch.empty(T << 26, dtype=torch.bfloat16, device="cuda").as_strided((T, Hq, D), (1 << 26, D, 1))
    far_q.copy_(q)
    slots = g.permutation(P * ps)[:T]
    slots[0] = P * ps - 1  # the last row of the last page
    assert len(set(slots.tolist())) == T
    pos, freqs = i32(g.integers(0, 9000, T)), S.rope_freqs(10000.0, D)
    got = []
    for x, (kc, vc) in ((q, R.pool(g, P, Hkv, ps, D, S.BF16, "head")), (far_q, far_pool(P, Hkv, ps, D))):
        kc.fill_(0.0)
        vc.fill_(0.0)
        q_out = torch.full_like(q, float("nan"))
        args = S.make_args(S.OP_ROPE_PAGED_KV, [x, k, v, pos, i32(slots), freqs, q_out, kc, vc], scalar=1.0)
        assert s.invoke(args, stream()) == (S.OK, 0), S.trident_scm_last_error()
        assert S.trident_scm_device_status(s.h, stream())[1] == 0
        got.append((q_out.cpu(), kc.cpu(), vc.cpu()))
    want = R.rotate(k.cpu().double(), pos.cpu(), freqs.cpu().double().sum(1), 1.0, False)
    page, at = slots // ps, slots % ps
    tol = 2.0 ** -8 * want.abs() * 1.01 + 8e-6 * want.abs().amax(-1, keepdim=True) * 2 ** 0.5 + 2.0 ** -25
    assert ((got[0][1][page, :, at].double() - want).abs() <= tol).all()
    for near, far in zip(*got):
        assert torch.equal(near, far)
    s.close()


@pytest.mark.parametrize("D", [8, 40, 96, 512])
@pytest.mark.parametrize("dtype", ["BF16", "FP16"])
def test_paged_attention_other_head_sizes(S, D, dtype):
    dt = getattr(S, dtype)
    g = np.random.default_rng(D)
    s, index, work = attn_scm(S, dt, 6, 2, D, 16, S.VARIANT_AUTO)
    b = R.batch(g, [2, 9], [50, 9], 6, 2, D, 16, dt)
    check_attn(S, b, 6, 2, D, 16, dt, 0.3, 0, s, index, work)
    s.close()


@pytest.mark.parametrize("variant", ["AUTO", "GENERIC"])
def test_paged_attention_large_and_growing_scores(S, variant):
    """Scores that rise along the keys (the running maximum moves in every tile) and that differ by
    thousands (one key takes all)."""
    Hq, Hkv, D, ps = 8, 2, 128, 16
    g = np.random.default_rng(8)
    s, index, work = attn_scm(S, S.BF16, Hq, Hkv, D, ps, getattr(S, "VARIANT_" + variant))
    for new, kv, mode in (([1, 40], [2000, 900], "rise"), ([3, 300], [512, 800], "one"), ([5, 64], [333, 100], "fall")):
        b = R.batch(g, new, kv, Hq, Hkv, D, ps, S.BF16)
        b["q"].fill_(1.0)
        tab = b["table"].cpu().numpy()
        for r, L in enumerate(kv):
            for j in range(L):
                level = {"rise": j / 64, "fall": (L - j) / 64, "one": 40.0 * (j == L // 3)}[mode]
                b["kc"][int(tab[r, j // ps]), :, j % ps] = level
        check_attn(S, b, Hq, Hkv, D, ps, S.BF16, 1.0, 0, s, index, work)
    s.close()


@pytest.mark.parametrize("variant", ["AUTO", "GENERIC"])
@pytest.mark.parametrize("n", [1, 150])
def test_paged_attention_reports_bad_tables(S, variant, n):
    """Numbers out of range set the status bit; the other requests' results stay right."""
    Hq, Hkv, D, ps = 8, 2, 128, 16
    g = np.random.default_rng(4)
    s, index, work = attn_scm(S, S.BF16, Hq, Hkv, D, ps, getattr(S, "VARIANT_" + variant))
    for what in ("page", "negative page", "kv", "negative kv", "cu", "cu past T"):
        b = R.batch(g, [n, n, n], [400, 300, 200], Hq, Hkv, D, ps, S.BF16)
        good = [0, 2]
        out, lse, wgt = R.attention(b["q"].cpu(), b["kc"].cpu(), b["vc"].cpu(), b["table"].cpu(), b["cu"].tolist(),
                                    b["kv"].tolist(), ps, 0.1)
        b["kc"].nan_to_num_(0.0)
        b["vc"].nan_to_num_(0.0)
        rows = [t for r in good for t in range(r * n, (r + 1) * n)]
        if what == "page": b["table"][1, 3] = 10 ** 6
        if what == "negative page": b["table"][1, 0] = -2
        if what == "kv": b["kv"][1], b["table"][1, :] = 10 ** 6, 0
        if what == "negative kv": b["kv"][1] = -4
        if what == "cu": b["cu"][1], rows = n + n + 1, list(range(2 * n + 1, 3 * n)) if n > 1 else []
        if what == "cu past T": b["cu"][3], rows = 3 * n + 1, list(range(n))
        args = S.make_args(S.OP_PAGED_ATTN, [b["q"], b["kc"], b["vc"], b["table"], b["cu"], b["kv"], work, b["out"],
                                             b["lse"]], scalar=0.1)
        assert s.invoke(args, stream()) == (S.OK, index), S.trident_scm_last_error()
        assert S.trident_scm_device_status(s.h, stream())[1] == S.DEVERR_TABLE, what
        if what != "cu":
            tol = R.attn_tolerance(out, wgt, S.BF16, 400, 5.0)
            assert ((b["out"].cpu().double() - out).abs() <= tol)[rows].all(), what
    s.close()


def test_a_step_through_one_call_and_a_graph(S):
    """Page map, RoPE with append and attention of one step: one invoke_seq, on a stream of its own, and the
    same captured in a CUDA graph and replayed on new lengths."""
    g = np.random.default_rng(2)
    B, Hq, Hkv, D, ps, P, N = 6, 8, 2, 128, 16, 64, 24
    s = S.Scm(flags=S.OPT_PDL)
    s.register(S.make_spec(S.OP_PAGE_MAP, S.I32, [], 1, 64, align_bytes=4))
    s.register(S.make_spec(S.OP_ROPE_PAGED_KV, S.BF16, [Hq, Hkv, D, D, ps], 1, 64, layout=S.LAYOUT_ANY))
    s.register(S.make_spec(S.OP_PAGED_ATTN, S.BF16, [Hq, Hkv, D, ps], 1, 64, layout=S.LAYOUT_ANY))
    work = torch.zeros(s.workspace(2), device="cuda")
    z = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    ctx, new, free, head, tab = z(B), z(B), i32(g.permutation(P)), z(1), z(B, 8)
    cu, kv, pos, slot, head_out = z(B + 1), z(B), z(N), z(N), z(1)
    qkv = torch.zeros(N, Hq + 2 * Hkv, D, dtype=torch.bfloat16, device="cuda")
    q_out, out = (torch.zeros(N, Hq, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lse = torch.zeros(N, Hq, device="cuda")
    kc, vc = (torch.full((P, Hkv, ps, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    freqs = S.rope_freqs(500000.0, D)
    scale = D ** -0.5
    seq = (S.trident_args * 3)(
        S.make_args(S.OP_PAGE_MAP, [ctx, new, free, head, tab, cu, kv, pos, slot, head_out], scalar=ps),
        S.make_args(S.OP_ROPE_PAGED_KV, [qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], pos, slot, freqs, q_out, kc, vc],
                    scalar=1.0),
        S.make_args(S.OP_PAGED_ATTN, [q_out, kc, vc, tab, cu, kv, work, out, lse], scalar=scale))
    side = torch.cuda.Stream()
    keys = [torch.zeros(0, Hkv, D, dtype=torch.float64) for _ in range(B)]
    vals = [torch.zeros(0, Hkv, D, dtype=torch.float64) for _ in range(B)]
    graph = torch.cuda.CUDAGraph()
    f = freqs.cpu().double().sum(1)
    for step, lens in enumerate([[5, 0, 9, 1, 2, 3], [1, 1, 1, 1, 1, 1], [1, 7, 1, 0, 1, 8], [1] * 6, [2, 1, 1, 1, 1, 12]]):
        x = torch.from_numpy(g.standard_normal((N, Hq + 2 * Hkv, D), dtype=np.float32)).bfloat16()
        qkv.copy_(x)
        new.copy_(i32(lens))
        side.wait_stream(torch.cuda.current_stream())
        if step == 2:
            torch.cuda.synchronize()
            with torch.cuda.graph(graph, stream=side):
                st = s.invoke_seq(seq, torch.cuda.current_stream().cuda_stream)
            assert st == (S.OK, [0, 1, 2]), S.trident_scm_last_error()
        if step >= 2:
            graph.replay()
        else:
            assert s.invoke_seq(seq, side.cuda_stream) == (S.OK, [0, 1, 2]), S.trident_scm_last_error()
        torch.cuda.synchronize()
        assert S.trident_scm_device_status(s.h, stream())[1] == 0
        x64, at = x.double(), 0
        for b, n in enumerate(lens):
            c = keys[b].shape[0]
            p = torch.arange(c, c + n)
            qr = R.rotate(x64[at:at + n, :Hq], p, f, 1.0, False).bfloat16().double()
            kr = R.rotate(x64[at:at + n, Hq:Hq + Hkv], p, f, 1.0, False).bfloat16().double()
            keys[b] = torch.cat([keys[b], kr])
            vals[b] = torch.cat([vals[b], x64[at:at + n, Hq + Hkv:]])
            L, G = c + n, Hq // Hkv
            if n:
                s64 = torch.einsum("ihd,jhd->hij", qr, keys[b].repeat_interleave(G, 1)) * scale
                s64 = s64.masked_fill(torch.arange(L)[None] > (c + torch.arange(n))[:, None], -np.inf)
                w = torch.softmax(s64, -1)
                v = vals[b].repeat_interleave(G, 1)
                ref = torch.einsum("hij,jhd->ihd", w, v)
                mag = torch.einsum("hij,jhd->ihd", w, v.abs())
                # q and k may round the other way at a tie's edge: one step of one element moves a score by at
                # most scale * 2^-7 * 16 (|q|, |k| < 4), 1.1 %
                tol = R.attn_tolerance(ref, mag, S.BF16, L, 5.0) + 0.012 * 2 * mag
                assert ((out[at:at + n].cpu().double() - ref).abs() <= tol).all(), (step, b)
            at += n
        assert (out[at:] == 0).all() and torch.isinf(lse[at:]).all()
        ctx.copy_(kv)
        head.copy_(head_out)
    s.close()


def test_the_serving_example_runs(S):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, os.path.join(root, "examples", "paged_serving.py"), "3"], capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0 and r.stdout.count("device status 0") == 4, r.stdout + r.stderr
