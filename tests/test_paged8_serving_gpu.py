"""The ops over 8-bit caches as they are used together: page maps, the quantised append, attention, reading back; their
workspace, graphs, streams, and a wait that runs out."""
import math

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


def i32(x):
    return torch.tensor(np.asarray(x, np.int32)).cuda()


class Engine:
    """A serving step: PAGE_MAP, ROPE_PAGED_KV8, PAGED_ATTN8 through one invoke_seq over static buffers."""

    def __init__(self, S, Hq, Hkv, D, ps, bt, dt, reqs, rows, pool=96, width=12):
        self.S, self.shape = S, (Hq, Hkv, D, ps, bt)
        self.scm = S.Scm(flags=S.OPT_PDL)
        self.scm.register(S.make_spec(S.OP_PAGE_MAP, S.I32, [], 1, 4096, align_bytes=4))
        self.scm.register(S.make_spec(S.OP_ROPE_PAGED_KV8, dt, [Hq, Hkv, D, D, ps, bt], 1, 1 << 20, layout=S.LAYOUT_ANY))
        a = self.scm.register(S.make_spec(S.OP_PAGED_ATTN8, dt, [Hq, Hkv, D, ps, bt], 1, 1 << 20, layout=S.LAYOUT_ANY))
        self.scm.register(S.make_spec(S.OP_PAGED_READ8, dt, [Hkv, D, ps, bt], 1, 1 << 20, layout=S.LAYOUT_ANY))
        act = R.TORCH[dt]
        self.ctx, self.new, self.kv = (i32([0] * reqs) for _ in range(3))
        self.cu, self.head, self.head_out = i32([0] * (reqs + 1)), i32([0]), i32([0])
        self.free = i32(np.random.default_rng(0).permutation(pool))
        self.table = i32(np.zeros((reqs, width)))
        self.pos, self.slot = i32([0] * rows), i32([0] * rows)
        self.qkv = torch.zeros(rows, Hq + 2 * Hkv, D, dtype=act, device="cuda")
        self.q, self.out = (torch.zeros(rows, Hq, D, dtype=act, device="cuda") for _ in range(2))
        self.lse = torch.zeros(rows, Hq, device="cuda")
        # a pool in use before: stale codes, NaN among them, and stale scales
        g = torch.Generator(device="cuda").manual_seed(1)
        codes = lambda: torch.randint(0, 256, (pool, Hkv, ps, D), generator=g, device="cuda").to(torch.uint8)  # noqa: E731
        self.kc, self.vc = codes().view(Q.E4M3), codes().view(Q.E4M3)
        self.ks, self.vs = (torch.randint(0, 256, (pool, Hkv, ps // bt), generator=g, device="cuda").to(torch.uint8).view(Q.E8M0)
                            for _ in range(2))
        self.work = torch.zeros(self.scm.workspace(a), device="cuda")
        self.freqs = S.rope_freqs(1e4, D)
        q, k, v = self.qkv.split([Hq, Hkv, Hkv], 1)
        caches = [self.kc, self.vc, self.ks, self.vs]
        self.calls = (S.trident_args * 3)(
            S.make_args(S.OP_PAGE_MAP, [self.ctx, self.new, self.free, self.head, self.table, self.cu, self.kv, self.pos,
                                        self.slot, self.head_out], scalar=ps),
            S.make_args(S.OP_ROPE_PAGED_KV8, [q, k, v, self.pos, self.slot, self.freqs, self.q, *caches], scalar=1.0),
            S.make_args(S.OP_PAGED_ATTN8, [self.q, *caches, self.table, self.cu, self.kv, self.work, self.out, self.lse],
                        scalar=D ** -0.5))

    def launch(self):
        status, _ = self.scm.invoke_seq(self.calls, torch.cuda.current_stream().cuda_stream)
        assert status == self.S.OK, self.S.trident_scm_last_error()

    def advance(self):
        self.ctx.copy_(self.kv)
        self.head.copy_(self.head_out)

    def read(self, first, lens, dt):
        """Every request's tokens from `first` on, through PAGED_READ8."""
        S, (_, Hkv, D, _, _) = self.S, self.shape
        cu = i32(np.concatenate([[0], np.cumsum(lens)]))
        k, v = (torch.zeros(sum(lens), Hkv, D, dtype=R.TORCH[dt], device="cuda") for _ in range(2))
        args = S.make_args(S.OP_PAGED_READ8, [self.kc, self.vc, self.ks, self.vs, self.table, cu, i32(first), k, v])
        assert self.scm.invoke(args, torch.cuda.current_stream().cuda_stream) == (S.OK, 3)
        return k, v

    def status(self):
        return self.S.trident_scm_device_status(self.scm.h, torch.cuda.current_stream().cuda_stream)[1]


def plain_attention(eng, q, keys, values, new):
    Hq, Hkv, D, _, _ = eng.shape
    out, at = [], 0
    for b, n in enumerate(new):
        L = keys[b].shape[0]
        k, v = (x.double().repeat_interleave(Hq // Hkv, 1) for x in (keys[b], values[b]))
        s = torch.einsum("ihd,jhd->hij", q[at:at + n].double(), k) * D ** -0.5
        s = s.masked_fill(torch.arange(L, device="cuda")[None] > L - n + torch.arange(n, device="cuda")[:, None], -math.inf)
        out.append(torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), v))
        at += n
    return torch.cat(out)


@pytest.mark.parametrize("Hq,Hkv,D,ps,bt,dtype", [(8, 2, 128, 16, 16, "BF16"), (4, 4, 64, 32, 8, "FP16"), (6, 1, 256, 16, 4, "BF16"),
                                                  (14, 2, 64, 64, 64, "BF16"), (8, 2, 128, 8, 1, "FP16")])
def test_serving_loop(S, Hq, Hkv, D, ps, bt, dtype):
    """Prompts of unequal lengths and then single tokens: what is read back is within half a step of what was written (and
    of the growth of its block's scale), and the attention is that over the values read back."""
    dt, g = getattr(S, dtype), torch.Generator(device="cuda").manual_seed(3)
    prompts = [37, 1, 0, 90, 16]
    eng = Engine(S, Hq, Hkv, D, ps, bt, dt, len(prompts), 160)
    true_k, true_v = ([torch.zeros(0, Hkv, D, device="cuda", dtype=torch.float64) for _ in prompts] for _ in range(2))
    f = eng.freqs.double().sum(1).cpu()
    for step in range(7):
        new = prompts if step == 0 else [1, 1, 1, 0, 2] if step == 3 else [1] * 5
        T = sum(new)
        qkv = torch.randn(T, Hq + 2 * Hkv, D, generator=g, device="cuda") * (1 + 3 * step)  # scales that grow
        eng.new.copy_(i32(new))
        eng.qkv[:T] = qkv
        eng.launch()
        at = 0
        for b, n in enumerate(new):
            rows = eng.qkv[at:at + n].cpu().double()
            p = torch.arange(true_k[b].shape[0], true_k[b].shape[0] + n)
            true_k[b] = torch.cat([true_k[b], R.rotate(rows[:, Hq:Hq + Hkv], p, f, 1.0, False).cuda()])
            true_v[b] = torch.cat([true_v[b], rows[:, Hq + Hkv:].cuda()])
            at += n
        lens = [k.shape[0] for k in true_k]
        k, v = eng.read([0] * 5, lens, dt)
        at, keys, values = 0, [], []
        for b, L in enumerate(lens):
            for got, want, into in ((k[at:at + L], true_k[b], keys), (v[at:at + L], true_v[b], values)):
                # 2^-4 of a value at its rounding, 2^-10 of a scale (at most top / 224) below that; each growth of a block's
                # scale rounds its codes again: by powers of two, which is exact but where a code loses bits below the
                # smallest step (2^-10 of the larger scale) or, at most twice here, is brought below the normal numbers
                err, top = (got.double() - want).abs(), want.abs().max() if L else 0
                assert (err <= 2.0 ** -4 * 1.1 * want.abs() * min(step + 1, 3) + 2.0 ** -9 / 224 * top * (step + 1) + 1e-5).all()
                into.append(got)
            at += L
        ref = plain_attention(eng, eng.q[:T], keys, values, new)
        err = (eng.out[:T].double() - ref).norm() / ref.norm()
        assert err < 2 * R.UNIT[dt], (step, err.item())
        assert (eng.out[T:] == 0).all() and torch.isinf(eng.lse[T:]).all()
        assert eng.status() == 0
        eng.advance()
    eng.scm.close()


def test_read_a_span(S):
    """From the middle of a request's pages on, over their borders."""
    eng = Engine(S, 4, 2, 64, 16, 8, S.BF16, 2, 80)
    eng.new.copy_(i32([50, 23]))
    eng.qkv.copy_(torch.randn(80, 8, 64, device="cuda"))
    eng.launch()
    k, v = eng.read([0, 0], [50, 23], S.BF16)
    a, b = eng.read([15, 7], [34, 1], S.BF16)
    assert torch.equal(a, torch.cat([k[15:49], k[57:58]])) and torch.equal(b, torch.cat([v[15:49], v[57:58]]))
    eng.scm.close()


def test_captured_and_replayed(S):
    """A step captured into a graph and replayed with other lengths in its buffers equals the eager one."""
    a, b = (Engine(S, 8, 2, 128, 16, 16, S.BF16, 4, 64) for _ in range(2))
    for e in (a, b):
        e.launch()  # nothing new: the first call of each version is not in the capture
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        a.launch()
    torch.manual_seed(2)
    for new in ([9, 30, 1, 16], [1, 1, 1, 1], [0, 20, 0, 3], [1, 0, 1, 1]):
        x = torch.randn(64, 12, 128, device="cuda").bfloat16()
        for e in (a, b):
            e.new.copy_(i32(new))
            e.qkv.copy_(x)
        graph.replay()
        b.launch()
        T = sum(new)
        assert torch.equal(a.out[:T], b.out[:T]) and torch.equal(a.lse[:T], b.lse[:T])
        for name in ("kc", "vc", "ks", "vs"):
            assert torch.equal(getattr(a, name).view(torch.uint8), getattr(b, name).view(torch.uint8))
        for e in (a, b):
            e.advance()
    a.scm.close()
    b.scm.close()


def attention_call(S, scm, g, new, kv, D, bt, dt, work):
    b = Q.batch(g, new, kv, 8, 2, D, 16, bt, dt)
    args = S.make_args(S.OP_PAGED_ATTN8, [b["q"], b["kc"], b["vc"], b["ks"], b["vs"], b["table"], b["cu"], b["kv"], work, b["out"],
                                          b["lse"]], scalar=D ** -0.5)
    return dict(b, work=work), args  # the arguments hold addresses: every tensor is kept


def test_a_workspace_for_both_kinds_of_caches(S):
    """Calls in order share one, over 8-bit and 16-bit caches and heads of different sizes."""
    scm, g = S.Scm(flags=S.OPT_PDL), np.random.default_rng(4)
    specs = [(S.OP_PAGED_ATTN8, [8, 2, 128, 16, 16]), (S.OP_PAGED_ATTN8, [8, 2, 64, 16, 8]), (S.OP_PAGED_ATTN, [8, 2, 128, 16])]
    index = [scm.register(S.make_spec(op, S.BF16, fixed, 1, 1 << 20, layout=S.LAYOUT_ANY)) for op, fixed in specs]
    work = torch.zeros(max(scm.workspace(i) for i in index), device="cuda")
    new, kv = [1, 700, 1, 3], [900, 2500, 64, 3000]
    b8, a8 = attention_call(S, scm, g, new, kv, 128, 16, S.BF16, work)
    c8, d8 = attention_call(S, scm, g, new, kv, 64, 8, S.BF16, work)
    b16 = R.batch(g, new, kv, 8, 2, 128, 16, S.BF16)
    a16 = S.make_args(S.OP_PAGED_ATTN, [b16["q"], b16["kc"], b16["vc"], b16["table"], b16["cu"], b16["kv"], work, b16["out"],
                                        b16["lse"]], scalar=128 ** -0.5)
    stream = torch.cuda.current_stream().cuda_stream
    kept = []
    for args, b in ((a8, b8), (a16, b16), (d8, c8)):
        assert scm.invoke(args, stream)[0] == S.OK
        kept.append(b["out"].clone())
    for _ in range(3):
        for args in (a8, a16, d8, a16, a8):
            assert scm.invoke(args, stream)[0] == S.OK
    for b, out in zip((b8, b16, c8), kept):
        assert torch.equal(b["out"], out)
    assert S.trident_scm_device_status(scm.h, stream)[1] == 0
    scm.close()


def test_two_streams_two_workspaces(S):
    scm, g = S.Scm(flags=S.OPT_PDL), np.random.default_rng(6)
    i = scm.register(S.make_spec(S.OP_PAGED_ATTN8, S.BF16, [8, 2, 128, 16, 16], 1, 1 << 20, layout=S.LAYOUT_ANY))
    pairs = [attention_call(S, scm, g, new, kv, 128, 16, S.BF16, torch.zeros(scm.workspace(i), device="cuda"))
             for new, kv in (([1] * 30, [1500] * 30), ([600, 1, 9], [2200, 900, 64]))]
    alone = []
    for b, args in pairs:
        assert scm.invoke(args, torch.cuda.current_stream().cuda_stream)[0] == S.OK
        alone.append((b["out"].clone(), b["lse"].clone()))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in pairs]
    for _ in range(5):
        for (b, args), st in zip(pairs, streams):
            assert scm.invoke(args, st.cuda_stream)[0] == S.OK
    torch.cuda.synchronize()
    for (b, _), (out, lse) in zip(pairs, alone):
        assert torch.equal(b["out"], out) and torch.equal(b["lse"], lse)
    scm.close()


@pytest.mark.parametrize("D,dtype", [(64, "BF16"), (128, "BF16"), (128, "FP16"), (256, "BF16")])
def test_a_wait_that_runs_out(S, D, dtype):
    """The tile kernel gives up its first wait for scores, says so, and leaves the device usable; a zeroed workspace works."""
    dt, g = getattr(S, dtype), np.random.default_rng(7)
    scm = S.Scm(flags=S.OPT_TEST_WAIT_TIMEOUT)
    i = scm.register(S.make_spec(S.OP_PAGED_ATTN8, dt, [8, 2, D, 16, 16], 1, 1 << 20, layout=S.LAYOUT_ANY))
    work = torch.zeros(scm.workspace(i), device="cuda")
    b, args = attention_call(S, scm, g, [3000, 3000], [6000, 6000], D, 16, dt, work)
    stream = torch.cuda.current_stream().cuda_stream
    assert scm.invoke(args, stream)[0] == S.OK
    assert S.trident_scm_device_status(scm.h, stream)[1] & S.DEVERR_TIMEOUT
    scm.close()
    scm = S.Scm()
    scm.register(S.make_spec(S.OP_PAGED_ATTN8, dt, [8, 2, D, 16, 16], 1, 1 << 20, layout=S.LAYOUT_ANY))
    work.zero_()
    assert scm.invoke(args, stream)[0] == S.OK
    assert S.trident_scm_device_status(scm.h, stream)[1] == 0
    assert torch.isfinite(b["out"]).all() and torch.isfinite(b["lse"]).all()
    scm.close()


@pytest.mark.parametrize("new", [1, 300])
def test_attention_bad_tables(S, new):
    """Numbers out of range set the status bit, read nothing out of range, and leave other requests right."""
    g = np.random.default_rng(9)
    scm = S.Scm()
    i = scm.register(S.make_spec(S.OP_PAGED_ATTN8, S.BF16, [8, 2, 128, 16, 16], 1, 1 << 20, layout=S.LAYOUT_ANY))
    work = torch.zeros(scm.workspace(i), device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    for what in ("page", "kv"):
        b, args = attention_call(S, scm, g, [new, new], [3000, 3000], 128, 16, S.BF16, work)
        if what == "page":
            b["table"][1, 5] = -7
        else:
            b["kv"][1] = 1 << 30
        assert scm.invoke(args, stream)[0] == S.OK
        assert S.trident_scm_device_status(scm.h, stream)[1] == S.DEVERR_TABLE
        one = {k: v for k, v in b.items()}
        one.update(q=b["q"][:new], cu=b["cu"][:2], kv=b["kv"][:1], table=b["table"][:1])
        ref, want, wgt, level = Q.reference(one, 16, 128 ** -0.5)
        tol = Q.tolerance(ref, wgt, level, S.BF16, 3000)
        assert ((b["out"][:new].cpu().double() - ref).abs() <= tol).all()
        assert ((b["lse"][:new].cpu().double() - want).abs() <= R.LSE_TOLERANCE).all()
    scm.close()


def test_a_small_workspace_is_refused(S):
    g = np.random.default_rng(1)
    scm = S.Scm()
    i = scm.register(S.make_spec(S.OP_PAGED_ATTN8, S.BF16, [8, 2, 128, 16, 16], 1, 1 << 20, layout=S.LAYOUT_ANY))
    b, args = attention_call(S, scm, g, [1], [50], 128, 16, S.BF16, torch.zeros(scm.workspace(i) - 1, device="cuda"))
    assert scm.invoke(args, torch.cuda.current_stream().cuda_stream)[0] == S.ERR_INVALID
    assert torch.isnan(b["out"]).all()
    scm.close()


def test_through_a_recipe(S):
    """Codes and scales as leaves of a structured call."""
    g = np.random.default_rng(2)
    scm = S.Scm()
    b = Q.batch(g, [5, 3], [20, 9], 1, 2, 64, 16, 16, S.BF16)
    scm.register_tree(S.make_spec(S.OP_PAGED_READ8, S.BF16, [2, 64, 16, 16], 1, 64),
                      S.Recipe((S.Slot(0), S.Slot(2)), (S.Slot(1), S.Slot(3)), S.Slot(4), S.Slot(5), S.Slot(6), S.Slot(7), S.Slot(8)))
    k, v = (torch.zeros(8, 2, 64, device="cuda").bfloat16() for _ in range(2))
    status = scm.call((b["kc"], b["ks"]), (b["vc"], b["vs"]), b["table"], b["cu"], i32([15, 6]), k, v)
    assert (status[0] if isinstance(status, tuple) else status) == S.OK
    x = Q.values(b["vc"].view(torch.uint8), b["vs"])
    t = b["table"].cpu().long()
    want = torch.stack([x[t[r, j // 16], :, j % 16] for r, j in [(0, j) for j in range(15, 20)] + [(1, j) for j in range(6, 9)]])
    assert torch.equal(v.cpu(), want.bfloat16())
    scm.close()


@pytest.mark.parametrize("variant", ["VARIANT_AUTO", "VARIANT_GENERIC"])
@pytest.mark.parametrize("bt", [16, 32])
def test_pages_past_32_bits(S, variant, bt):
    """Pages whose first code lies past 2^32 bytes: every op does there what it does with the same pages at the beginning of
    a pool, bit for bit; and what lies 2^32 bytes before them is left as it was."""
    Hq, Hkv, D, ps, dt = 8, 2, 128, 32, S.BF16
    g = np.random.default_rng(11)
    new, kv = [1, 70, 150], [400, 90, 700]
    b = Q.batch(g, new, kv, Hq, Hkv, D, ps, bt, dt)
    P, T = b["kc"].shape[0], sum(new)
    off = 2 ** 32 // (Hkv * ps * D)
    names = ("kc", "vc", "ks", "vs")
    far = {}
    for n in names:
        big = torch.zeros(off + P, *b[n].shape[1:], dtype=torch.uint8, device="cuda")
        big[off:] = b[n].view(torch.uint8)
        far[n] = big.view(b[n].dtype)
    table = b["table"] + off * (b["table"] < P).int()
    act = R.TORCH[dt]
    q, k, v = (torch.from_numpy(g.standard_normal((T, h, D)) * 3).to(act).cuda() for h in (Hq, Hkv, Hkv))
    slot, pos = [], []
    for r, (n, L) in enumerate(zip(new, kv)):
        pos += range(L - n, L)
        slot += [int(b["table"][r, j // ps]) * ps + j % ps for j in range(L - n, L)]
    pos, slot = i32(pos), i32(slot)
    s = S.Scm()
    kw = dict(layout=S.LAYOUT_ANY, variant=getattr(S, variant))
    s.register(S.make_spec(S.OP_ROPE_PAGED_KV8, dt, [Hq, Hkv, D, D, ps, bt], 1, 1 << 20, **kw))
    a = s.register(S.make_spec(S.OP_PAGED_ATTN8, dt, [Hq, Hkv, D, ps, bt], 1, 1 << 20, **kw))
    s.register(S.make_spec(S.OP_PAGED_READ8, dt, [Hkv, D, ps, bt], 1, 1 << 20, **kw))
    work, freqs, st = torch.zeros(s.workspace(a), device="cuda"), S.rope_freqs(1e4, D), torch.cuda.current_stream().cuda_stream

    def serve(c, table, slot):
        caches = [c[n] for n in names]
        rot, out = (torch.zeros(T, Hq, D, dtype=act, device="cuda") for _ in range(2))
        lse = torch.zeros(T, Hq, device="cuda")
        ko, vo = (torch.zeros(T, Hkv, D, dtype=act, device="cuda") for _ in range(2))
        for args in (S.make_args(S.OP_ROPE_PAGED_KV8, [q, k, v, pos, slot, freqs, rot, *caches], scalar=1.0),
                     S.make_args(S.OP_PAGED_ATTN8, [rot, *caches, table, b["cu"], b["kv"], work, out, lse], scalar=D ** -0.5),
                     S.make_args(S.OP_PAGED_READ8, [*caches, table, b["cu"], b["kv"] - i32(new), ko, vo])):
            assert s.invoke(args, st)[0] == S.OK, S.trident_scm_last_error()
        assert S.trident_scm_device_status(s.h, st)[1] == 0
        return rot, out, lse, ko, vo

    want, got = serve(b, b["table"], slot), serve(far, table, slot + off * ps)
    for x, y in zip(want, got):
        assert torch.isfinite(x).all() and torch.equal(x, y)
    for n in names:
        assert torch.equal(far[n][off:].view(torch.uint8), b[n].view(torch.uint8))
        assert not far[n][:P].view(torch.uint8).any()
    s.close()
