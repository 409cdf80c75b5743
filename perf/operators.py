"""Timing cases of the paged-serving operators: a batch of requests of unequal lengths gets cache
pages (page_map), its new tokens' q and k are rotated and k, v written into the pages (rope), and
the new tokens attend to all of their request's pages (attn).

A case is one call of one operator on one batch, in the plain form (torch's elementary operations
in 32 bits) or, with `own`, through the library (paper_2609_37241_gb300.scm): one Scm for all
calls, and an argument tuple that is built on a state's first pass and kept, as an engine keeps it
for its static buffers.

Lengths come from the case alone ("lens"), values, page numbers and weights from the seed. Pages
are scattered over the pool in random order; the pool's unused slots hold stale values.
"""
import math
import random

import torch

own = False
TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-6


# ---------------------------------------------------------------- the cases
def _map(reqs, new, ctx, page, chunk=0, lens=1):
    return dict(op="page_map", reqs=reqs, new=new, ctx=ctx, page=page, chunk=chunk, lens=lens)


def _rope(tokens, q_heads, kv_heads, head, rot, page, dtype, pairs, qk_norm, scaled, order="head"):
    return dict(op="rope", tokens=tokens, q_heads=q_heads, kv_heads=kv_heads, head=head, rot=rot, page=page,
                dtype=dtype, pairs=pairs, qk_norm=qk_norm, scaled=scaled, order=order)


def _attn(reqs, new, ctx, q_heads, kv_heads, head, page, dtype, chunk=0, order="head", lens=1):
    """reqs requests of 1..new new tokens after ctx/8..ctx cached ones (new, ctx < 0: exactly -new,
    -ctx); the first one has `chunk` new tokens instead where chunk > 0."""
    return dict(op="attn", reqs=reqs, new=new, ctx=ctx, q_heads=q_heads, kv_heads=kv_heads, head=head, page=page,
                dtype=dtype, chunk=chunk, order=order, lens=lens)


def listed():
    return [
        # a decode step's bookkeeping: one new token for each of 64 requests
        dict(_map(64, -1, 8192, 16), name="map_64req_decode"),
        # admission of prompts into a large running batch: ragged chunks, one long
        dict(_map(512, 48, 4096, 32, chunk=8191), name="map_512req_chunks"),
        # a decode step's q/k norm, RoPE and append at the repository's second layer configuration
        dict(_rope(64, 32, 8, 128, 128, 16, "bf16", "half", True, False), name="rope_64tok_qk"),
        # a ragged prefill, interleaved pairs over half of the head, frequencies rescaled for a long
        # context, cache rows in token order
        dict(_rope(3333, 32, 8, 128, 64, 32, "fp16", "interleaved", False, True, "token"), name="rope_3333tok_partial"),
        # one long prompt's append
        dict(_rope(8192, 32, 8, 128, 128, 16, "bf16", "half", False, True), name="rope_8192tok"),
        # one token of one request: latency
        dict(_attn(1, -1, -1000, 32, 8, 128, 16, "bf16"), name="attn_1req_ctx1000"),
        # a decode step of 64 requests of ragged lengths
        dict(_attn(64, -1, 8192, 32, 8, 128, 16, "bf16"), name="attn_64req_decode"),
        # few requests with very long contexts: work split along the cache
        dict(_attn(3, -1, -131071, 32, 8, 128, 32, "fp16"), name="attn_3req_ctx131071"),
        # several drafted tokens for each request, heads of 64, seven q heads per kv head
        dict(_attn(48, 5, 3000, 28, 4, 64, 16, "fp16", order="token"), name="attn_48req_drafts_d64"),
        # a prompt's chunk that joins running decodes
        dict(_attn(17, -1, 4096, 32, 8, 128, 16, "bf16", chunk=1000), name="attn_17req_mixed"),
        # one chunk of a long prompt
        dict(_attn(1, -2048, -6144, 32, 8, 128, 16, "bf16"), name="attn_chunk2048_ctx6144"),
        # the largest: a whole prompt's second half
        dict(_attn(1, -8192, -8192, 32, 8, 128, 64, "bf16"), name="attn_chunk8192_ctx8192"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choices(["page_map", "rope", "attn"], [1, 2, 4])[0]
    page = rng.choice([8, 16, 16, 32, 64, 128])
    lens = rng.randint(2, 1 << 20)
    if op == "page_map":
        chunk = _log(rng, 64, 16384) if rng.random() < 0.5 else 0
        return _map(_log(rng, 1, 2048), rng.choice([-1, 5, 48]), _log(rng, 16, 8192), rng.choice([page, 1, 24]), chunk, lens)
    dtype, order = rng.choice(["bf16", "bf16", "fp16"]), rng.choice(["head", "head", "token"])
    head = rng.choice([128, 128, 64, 256])
    kv_heads = rng.choice([1, 2, 4, 8])
    q_heads = kv_heads * rng.choice([1, 2, 4, 4, 5, 7, 8])
    if op == "rope":
        rot = rng.choice([head, head, head // 2, head // 4])
        return _rope(_log(rng, 1, 8192), q_heads, kv_heads, head, rot, page, dtype,
                     rng.choice(["half", "interleaved"]), rng.random() < 0.4, rng.random() < 0.5, order)
    kind = rng.choices(["decode", "drafts", "chunk", "mixed"], [4, 2, 3, 2])[0]
    if kind == "decode":
        reqs = _log(rng, 1, 256)
        c = _attn(reqs, -1, _log(rng, 100, min(131072, 600000 // reqs)), q_heads, kv_heads, head, page, dtype, 0, order, lens)
    elif kind == "drafts":
        reqs = _log(rng, 1, 96)
        c = _attn(reqs, rng.randint(2, 9), _log(rng, 100, min(32768, 300000 // reqs)), q_heads, kv_heads, head, page,
                  dtype, 0, order, lens)
    elif kind == "chunk":
        c = _attn(1, -_log(rng, 16, 6000), -_log(rng, 1, 10000), q_heads, kv_heads, head, page, dtype, 0, order, lens)
    else:
        c = _attn(rng.randint(2, 24), rng.choice([-1, 4]), _log(rng, 200, 4096), q_heads, kv_heads, head, page, dtype,
                  _log(rng, 32, 1500), order, lens)
    top = work(listed()[-1])
    while work(c)["bytes"] > 2.5e9 or work(c)["flops"] > top["flops"]:
        c["ctx"] = -max(1, -c["ctx"] // 2) if c["ctx"] < 0 else max(8, c["ctx"] // 2)
        c["new"] = -max(1, -c["new"] * 3 // 4) if c["new"] < 0 else c["new"]
    return c


def _lengths(case):
    """(tokens cached, new tokens) of each request, by the case alone."""
    r, n = random.Random(case["lens"]), case["reqs"]
    new = [-case["new"] if case["new"] < 0 else r.randint(1, case["new"]) for _ in range(n)]
    ctx = [-case["ctx"] if case["ctx"] < 0 else r.randint(case["ctx"] // 8, case["ctx"]) for _ in range(n)]
    if case["chunk"]:
        new[0] = case["chunk"]
    return ctx, new


def work(case):
    """What one call has to read and write (each byte once) and compute."""
    if case["op"] == "page_map":
        ctx, new = _lengths(case)
        pages = sum(-(-(c + n) // case["page"]) + (-c // case["page"]) for c, n in zip(ctx, new))
        # the page that a request's first new token goes to is read where it is an old one
        return {"bytes": 4 * (2 * len(ctx) + 2 * pages + len(ctx) + 2 * len(ctx) + 1 + 2 * sum(new) + 2), "flops": 0}
    if case["op"] == "rope":
        heads, t = case["q_heads"] + 2 * case["kv_heads"], case["tokens"]
        rotated = (case["q_heads"] + case["kv_heads"]) * t
        return {"bytes": 2 * 2 * t * heads * case["head"] + 8 * t + 4 * case["rot"],
                "flops": rotated * (3 * case["rot"] + (4 * case["head"] if case["qk_norm"] else 0))}
    ctx, new = _lengths(case)
    seen = sum(n * c + n * (n + 1) // 2 for c, n in zip(ctx, new))
    kv = sum(c + n for c, n in zip(ctx, new))
    t = sum(new)
    return {"bytes": 2 * 2 * kv * case["kv_heads"] * case["head"] + 2 * 2 * t * case["q_heads"] * case["head"]
            + 4 * t * case["q_heads"] + 4 * sum(-(-(c + n) // case["page"]) for c, n in zip(ctx, new)) + 8 * len(ctx),
            "flops": 4 * seen * case["q_heads"] * case["head"]}


# ---------------------------------------------------------------- inputs
def _pool(shape, order, dtype, gen):
    """A cache [pages, kv heads, page, head size], its rows in head or in token order."""
    p, h, s, d = shape
    if order == "token":
        return torch.randn((p, s, h, d), generator=gen, device="cuda", dtype=dtype).transpose(1, 2)
    return torch.randn((p, h, s, d), generator=gen, device="cuda", dtype=dtype)


def _freqs(rot, scaled):
    """theta^(-2i/rot) as pairs (hi, lo) of 32 bits; scaled: the long wavelengths divided by 8 with a
    linear ramp between 1 and 32 rotations over 8192 positions."""
    f = [500000.0 ** (-2.0 * i / rot) for i in range(rot // 2)]
    if scaled:
        turns = [8192 * x / (2 * math.pi) for x in f]
        keep = [min(1.0, max(0.0, (n - 1.0) / 31.0)) for n in turns]
        f = [x * k + x / 8 * (1 - k) for x, k in zip(f, keep)]
    f = torch.tensor(f, dtype=torch.float64)
    hi = f.float()
    return torch.stack([hi, (f - hi.double()).float()], 1).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s = {"case": case}
    ps = case["page"]

    def perm(n):
        return torch.randperm(n, generator=gen, device="cuda").to(torch.int32)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    if case["op"] == "page_map":
        ctx, new = _lengths(case)
        need = [-(-(c + n) // ps) for c, n in zip(ctx, new)]
        have = [-(-c // ps) for c in ctx]
        pool = sum(need) + 100
        width = max(max(need), 1) + 3
        ids = perm(pool)
        held = sum(have)
        s.update(ctx=ints(ctx), new=ints(new), head=ints([7]), tokens=sum(new) + (-sum(new)) % 8)
        s["free"] = torch.cat([perm(7), ids[held:]])  # seven entries are taken already
        col = torch.arange(width, device="cuda")[None]
        at = torch.cumsum(ints(have), 0) - ints(have)
        s["table"] = torch.where(col < ints(have)[:, None], ids[(at[:, None] + col).clamp(max=pool - 1)], ids.new_full((), -1))
        return s
    dt = TORCH[case["dtype"]]
    hq, hk, d = case["q_heads"], case["kv_heads"], case["head"]
    if case["op"] == "rope":
        t = case["tokens"]
        pages = -(-t // ps) + 9
        qkv = torch.randn((t, hq + 2 * hk, d), generator=gen, device="cuda", dtype=dt)  # one projection's rows
        s.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hk], v=qkv[:, hq + hk:], freqs=_freqs(case["rot"], case["scaled"]).cuda())
        s["pos"] = torch.randint(0, 32768, (t,), generator=gen, device="cuda").to(torch.int32) if t <= 256 else \
            torch.arange(1000, 1000 + t, dtype=torch.int32, device="cuda")
        at = torch.arange(t, device="cuda")
        s["slots"] = (perm(pages)[at // ps] * ps + at % ps).to(torch.int32)
        s["magnitude"] = 1.0 + 0.1 * math.log(8) if case["scaled"] else 1.0
        for name in ("k_cache", "v_cache"):
            s[name] = _pool((pages, hk, ps, d), case["order"], dt, gen)
        for name in ("gamma_q", "gamma_k"):
            s[name] = torch.randn(d, generator=gen, device="cuda") * 0.1 + 1.0
        return s
    ctx, new = _lengths(case)
    need = [-(-(c + n) // ps) for c, n in zip(ctx, new)]
    pool, width = sum(need) + 5, max(need)
    ids = perm(pool)
    at = torch.cumsum(ints(need), 0) - ints(need)
    col = torch.arange(width, device="cuda")[None]
    s["table"] = torch.where(col < ints(need)[:, None], ids[(at[:, None] + col).clamp(max=pool - 1)], ids.new_zeros(()))
    s["cu"] = torch.nn.functional.pad(torch.cumsum(ints(new), 0), (1, 0)).to(torch.int32)
    s["kv"] = ints([c + n for c, n in zip(ctx, new)])
    s["q"] = torch.randn((sum(new), hq, d), generator=gen, device="cuda", dtype=dt)
    for name in ("k_cache", "v_cache"):
        s[name] = _pool((pool, hk, ps, d), case["order"], dt, gen)
    s.update(scale=1.0 / math.sqrt(d), max_new=max(new))
    return s


# ---------------------------------------------------------------- the plain forms
def _plain_map(s):
    ps, n, free = s["case"]["page"], s["tokens"], s["free"]
    ctx, new = s["ctx"].long(), s["new"].long()
    kv = ctx + new
    cu = torch.nn.functional.pad(torch.cumsum(new, 0), (1, 0))
    have, need = (ctx + ps - 1) // ps, (kv + ps - 1) // ps
    ends = torch.cumsum(need - have, 0)
    col = torch.arange(s["table"].shape[1], device=ctx.device)[None]
    j = col - have[:, None]
    idx = (s["head"].long() + (ends - (need - have))[:, None] + j).clamp(0, free.numel() - 1)
    table = torch.where((j >= 0) & (col < need[:, None]), free[idx], s["table"])
    tok = torch.arange(n, device=ctx.device)
    r = torch.searchsorted(cu[1:], tok, right=True).clamp(max=ctx.numel() - 1)
    real = tok < cu[-1]
    pos = torch.where(real, ctx[r] + tok - cu[r], 0)
    slot = torch.where(real, table[r, pos // ps].long() * ps + pos % ps, -1)
    i32 = torch.int32
    return [table, cu.to(i32), kv.to(i32), pos.to(i32), slot.to(i32), (s["head"] + ends[-1]).to(i32)]


def _rotate(x, cos, sin, rot, interleaved):
    y, a = x.clone(), x[..., :rot]
    lo, hi = (a[..., 0::2], a[..., 1::2]) if interleaved else (a[..., :rot // 2], a[..., rot // 2:])
    p, q = lo * cos - hi * sin, hi * cos + lo * sin
    y[..., :rot] = torch.stack([p, q], -1).flatten(-2) if interleaved else torch.cat([p, q], -1)
    return y


def _plain_rope(s):
    c, dt = s["case"], s["q"].dtype
    q, k = s["q"].float(), s["k"].float()
    if c["qk_norm"]:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + EPS) * s["gamma_q"]
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + EPS) * s["gamma_k"]
    pos = s["pos"].float()[:, None]
    angle = pos * s["freqs"][None, :, 0] + pos * s["freqs"][None, :, 1]
    cos, sin = torch.cos(angle)[:, None] * s["magnitude"], torch.sin(angle)[:, None] * s["magnitude"]
    inter = c["pairs"] == "interleaved"
    page, at = s["slots"].long() // c["page"], s["slots"].long() % c["page"]
    s["k_cache"][page, :, at] = _rotate(k, cos, sin, c["rot"], inter).to(dt)
    s["v_cache"][page, :, at] = s["v"]
    return [_rotate(q, cos, sin, c["rot"], inter).to(dt), s["k_cache"], s["v_cache"]]


def _plain_attn(s):
    c, q = s["case"], s["q"]
    hk, d, ps, n = c["kv_heads"], c["head"], c["page"], s["max_new"]
    g = c["q_heads"] // hk
    cu, kv = s["cu"].long(), s["kv"].long()
    b, width = s["table"].shape
    new = cu[1:] - cu[:-1]
    i = torch.arange(n, device=q.device)
    rows = (cu[:-1, None] + i).clamp(max=q.shape[0] - 1)                           # [b, n]
    x = q[rows].float().view(b, n, hk, g, d).permute(0, 2, 3, 1, 4).reshape(b, hk, g * n, d)
    tab = s["table"].long()
    k = s["k_cache"][tab].float().transpose(1, 2).reshape(b, hk, width * ps, d)
    v = s["v_cache"][tab].float().transpose(1, 2).reshape(b, hk, width * ps, d)
    j = torch.arange(width * ps, device=q.device)
    seen = j <= (kv - new)[:, None, None] + i[:, None]                             # [b, n, keys]
    p = torch.matmul(x, k.transpose(2, 3)).view(b, hk, g, n, width * ps)
    p.mul_(s["scale"]).masked_fill_(~seen[:, None, None], -math.inf)
    top = p.amax(-1, keepdim=True)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(b, hk, g * n, width * ps), v).view(b, hk, g, n, d) / total
    lse = (top + torch.log(total))[..., 0]
    # back to one row per token
    t = torch.arange(q.shape[0], device=q.device)
    r = torch.searchsorted(cu[1:], t, right=True)
    o = out.permute(0, 3, 1, 2, 4).reshape(b, n, hk * g, d)[r, t - cu[r]]
    return [o.to(q.dtype), lse.permute(0, 3, 1, 2).reshape(b, n, hk * g)[r, t - cu[r]].contiguous()]


# ---------------------------------------------------------------- the library's calls
_lib = {}


def _version(S, op, dtype, fixed, **kw):
    """The process's Scm and its version for (op, dtype, fixed), registered at its first use."""
    if "scm" not in _lib:
        _lib["scm"] = S.Scm(device=torch.cuda.current_device(), flags=S.OPT_PDL)
    key = (op, dtype, tuple(fixed))
    if key not in _lib:
        _lib[key] = _lib["scm"].register(S.make_spec(op, dtype, fixed, 1, 1 << 30, device=torch.cuda.current_device(), **kw))
    return _lib["scm"], _lib[key]


def _bind(s):
    """The argument tuple of a state's call and its output tensors (made once, kept with the state)."""
    from paper_2609_37241_gb300 import scm as S
    c = s["case"]
    new = lambda shape, dt: torch.empty(shape, dtype=dt, device="cuda")  # noqa: E731
    i32 = torch.int32
    if c["op"] == "page_map":
        b = c["reqs"]
        scm, _ = _version(S, S.OP_PAGE_MAP, S.I32, [], rank=1, align_bytes=4)
        table = s["table"].clone()
        out = [table, new(b + 1, i32), new(b, i32), new(s["tokens"], i32), new(s["tokens"], i32), new(1, i32)]
        args = S.make_args(S.OP_PAGE_MAP, [s["ctx"], s["new"], s["free"], s["head"], *out], scalar=c["page"])
        return scm, args, out
    dt = {"bf16": S.BF16, "fp16": S.FP16}[c["dtype"]]
    hq, hk, d, ps = c["q_heads"], c["kv_heads"], c["head"], c["page"]
    if c["op"] == "rope":
        op = {("half", False): S.OP_ROPE_PAGED_KV, ("interleaved", False): S.OP_ROPE_PAGED_KV_INTERLEAVED,
              ("half", True): S.OP_QKNORM_ROPE_PAGED_KV,
              ("interleaved", True): S.OP_QKNORM_ROPE_PAGED_KV_INTERLEAVED}[c["pairs"], c["qk_norm"]]
        scm, _ = _version(S, op, dt, [hq, hk, d, c["rot"], ps], layout=S.LAYOUT_ANY)
        q_out = new((c["tokens"], hq, d), s["q"].dtype)
        ts = [s["q"], s["k"], s["v"], s["pos"], s["slots"], s["freqs"], q_out, s["k_cache"], s["v_cache"]]
        if c["qk_norm"]:
            ts += [s["gamma_q"], s["gamma_k"]]
        return scm, S.make_args(op, ts, eps=EPS, scalar=s["magnitude"]), [q_out, s["k_cache"], s["v_cache"]]
    scm, index = _version(S, S.OP_PAGED_ATTN, dt, [hq, hk, d, ps], layout=S.LAYOUT_ANY)
    if ("work", index) not in _lib:  # a workspace per stream, zeros before its first use
        _lib["work", index] = torch.zeros(scm.workspace(index), dtype=torch.float32, device="cuda")
    out, lse = new(tuple(s["q"].shape), s["q"].dtype), new((s["q"].shape[0], hq), torch.float32)
    args = S.make_args(S.OP_PAGED_ATTN, [s["q"], s["k_cache"], s["v_cache"], s["table"], s["cu"], s["kv"],
                                         _lib["work", index], out, lse], scalar=s["scale"])
    return scm, args, [out, lse]


def run(state):
    if not own:
        return {"page_map": _plain_map, "rope": _plain_rope, "attn": _plain_attn}[state["case"]["op"]](state)
    if "call" not in state:
        state["call"] = _bind(state)
    scm, args, out = state["call"]
    status, _ = scm.invoke(args, torch.cuda.current_stream().cuda_stream)
    if status != 0:
        from paper_2609_37241_gb300 import scm as S
        raise S.ScmError(status, state["case"]["op"])
    return out


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "page_map":
        return None
    if case["op"] == "rope":
        rot, inter, ps = case["rot"], case["pairs"] == "interleaved", case["page"]
        i = torch.arange(rot // 2, device="cuda")
        first, second = (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)
        w = s["freqs"].to(f64).sum(1)
        turn = torch.polar(torch.full((), s["magnitude"], dtype=f64, device="cuda"), s["pos"].to(f64)[:, None] * w)[:, None]

        def side(x, gamma):
            y = x.to(f64)
            if case["qk_norm"]:
                y = y / torch.sqrt(y.pow(2).sum(-1, keepdim=True) / case["head"] + EPS) * gamma.to(f64)
            z = torch.complex(y[..., first], y[..., second]) * turn
            y = y.clone()
            y[..., first], y[..., second] = z.real, z.imag
            return y

        kc, vc = s["k_cache"].to(f64), s["v_cache"].to(f64)
        slots = s["slots"].long()
        kc[slots // ps, :, slots % ps] = side(s["k"], s["gamma_k"])
        vc[slots // ps, :, slots % ps] = s["v"].to(f64)
        return [side(s["q"], s["gamma_q"]), kc, vc]
    if work(case)["flops"] > 4e12:
        return None
    ctx, new = _lengths(case)
    hq, hk = case["q_heads"], case["kv_heads"]
    out = torch.empty(s["q"].shape, dtype=f64, device="cuda")
    lse = torch.empty(s["q"].shape[:2], dtype=f64, device="cuda")
    first = 0
    for b, (c, n) in enumerate(zip(ctx, new)):
        pages = s["table"][b, :-(-(c + n) // case["page"])].long()
        last = c + torch.arange(n, device="cuda")
        for h in range(hk):
            k, v = (s[name][pages, h].reshape(-1, case["head"])[:c + n].to(f64) for name in ("k_cache", "v_cache"))
            for a in range(h * (hq // hk), (h + 1) * (hq // hk)):
                z = (s["q"][first:first + n, a].to(f64) @ k.T) * s["scale"]
                z = z.masked_fill(torch.arange(c + n, device="cuda") > last[:, None], -math.inf)
                lse[first:first + n, a] = torch.logsumexp(z, 1)
                out[first:first + n, a] = torch.softmax(z, 1) @ v
        first += n
    return [out, lse]
