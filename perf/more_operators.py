"""Timing cases of paged serving over a cache held in 8 bits: e4m3 codes with a power-of-two scale for
each block of tokens and head. A batch's new tokens are rotated and quantised into the pages as they
are written (write), the new tokens attend to all of their request's pages (attn), and spans of a
request are read back in the activation type (read).

A block is `block` consecutive rows of a page, one head; its scale is 2^e with the smallest e in
[-32, 32] for which its largest value is at most 448 * 2^e. A call that writes a block's first row
begins it anew; one that goes on with it raises e where its own rows need it, and the rows that the
block held are rounded to the new scale.

A case is one call of one operator on one batch, in the plain form (torch's elementary operations
in 32 bits) or, with `own`, through the library (paper_2609_37241_gb300.scm): one Scm for all
calls, and an argument tuple that is built on a state's first pass and kept, as an engine keeps it
for its static buffers.

Lengths come from the case alone ("lens"), values, page numbers and weights from the seed. Pages
are scattered over the pool in random order; the pool's unused slots hold stale values. Keys have
a few channels that are larger than the others, and tokens differ in size.
"""
import math
import random

import torch

own = False
TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16}
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
EPS = 1e-6
E_MIN, E_MAX = -32, 32


# ---------------------------------------------------------------- the cases
def _write(tokens, reqs, q_heads, kv_heads, head, rot, page, block, dtype, pairs, qk_norm, scaled, order="head", lens=1):
    """tokens new tokens of reqs requests, each going on somewhere behind what it has in the cache."""
    return dict(op="write", tokens=tokens, reqs=reqs, q_heads=q_heads, kv_heads=kv_heads, head=head, rot=rot, page=page,
                block=block, dtype=dtype, pairs=pairs, qk_norm=qk_norm, scaled=scaled, order=order, lens=lens)


def _read(reqs, span, kv_heads, head, page, block, dtype, order="head", lens=1):
    """span/8..span tokens (span < 0: exactly -span) of each of reqs requests, from anywhere."""
    return dict(op="read", reqs=reqs, span=span, kv_heads=kv_heads, head=head, page=page, block=block, dtype=dtype,
                order=order, lens=lens)


def _attn(reqs, new, ctx, q_heads, kv_heads, head, page, block, dtype, chunk=0, order="head", lens=1):
    """reqs requests of 1..new new tokens after ctx/8..ctx cached ones (new, ctx < 0: exactly -new,
    -ctx); the first one has `chunk` new tokens instead where chunk > 0."""
    return dict(op="attn", reqs=reqs, new=new, ctx=ctx, q_heads=q_heads, kv_heads=kv_heads, head=head, page=page,
                block=block, dtype=dtype, chunk=chunk, order=order, lens=lens)


def listed():
    return [
        # a decode step's q/k norm, RoPE and quantised append: one token each, inside blocks that are begun
        dict(_write(64, 64, 32, 8, 128, 128, 16, 16, "bf16", "half", True, False), name="write_64tok_qk"),
        # a ragged prefill, interleaved pairs over half of the head, frequencies rescaled for a long
        # context, cache rows in token order, two blocks to a page
        dict(_write(3333, 11, 32, 8, 128, 64, 64, 32, "fp16", "interleaved", False, True, "token"), name="write_3333tok_partial"),
        # one long prompt's append
        dict(_write(8192, 1, 32, 8, 128, 128, 16, 16, "bf16", "half", False, True), name="write_8192tok"),
        # a short prefix handed to another engine: latency
        dict(_read(1, -500, 8, 128, 16, 16, "bf16"), name="read_1req_500"),
        # the contexts of a batch that moves to a cache in the activation type
        dict(_read(24, 8192, 8, 128, 32, 16, "fp16", "token"), name="read_24req_ragged"),
        # one token of one request: latency
        dict(_attn(1, -1, -1000, 32, 8, 128, 16, 16, "bf16"), name="attn_1req_ctx1000"),
        # a decode step of 64 requests of ragged lengths
        dict(_attn(64, -1, 8192, 32, 8, 128, 16, 16, "bf16"), name="attn_64req_decode"),
        # few requests with very long contexts, a scale for each token: work split along the cache
        dict(_attn(3, -1, -131071, 32, 8, 128, 32, 1, "fp16"), name="attn_3req_ctx131071"),
        # several drafted tokens for each request, heads of 64, seven q heads per kv head
        dict(_attn(48, 5, 3000, 28, 4, 64, 16, 8, "fp16", order="token"), name="attn_48req_drafts_d64"),
        # a prompt's chunk that joins running decodes
        dict(_attn(17, -1, 4096, 32, 8, 128, 16, 16, "bf16", chunk=1000), name="attn_17req_mixed"),
        # one chunk of a long prompt
        dict(_attn(1, -2048, -6144, 32, 8, 128, 16, 16, "bf16"), name="attn_chunk2048_ctx6144"),
        # the largest: a whole prompt's second half
        dict(_attn(1, -8192, -8192, 32, 8, 128, 64, 64, "bf16"), name="attn_chunk8192_ctx8192"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choices(["write", "read", "attn"], [2, 1, 4])[0]
    page = rng.choice([8, 16, 16, 32, 64, 128])
    block = rng.choice([b for b in (1, 8, 16, 16, 32, page, page) if page % b == 0])
    lens = rng.randint(2, 1 << 20)
    dtype, order = rng.choice(["bf16", "bf16", "fp16"]), rng.choice(["head", "head", "token"])
    head = rng.choice([128, 128, 64, 256])
    kv_heads = rng.choice([1, 2, 4, 8])
    q_heads = kv_heads * rng.choice([1, 2, 4, 4, 5, 7, 8])
    if op == "write":
        rot = rng.choice([head, head, head // 2, head // 4])
        tokens = _log(rng, 1, 8192)
        reqs = tokens if tokens <= 256 and rng.random() < 0.6 else rng.randint(1, min(16, tokens))
        return _write(tokens, reqs, q_heads, kv_heads, head, rot, page, block, dtype, rng.choice(["half", "interleaved"]),
                      rng.random() < 0.4, rng.random() < 0.5, order, lens)
    if op == "read":
        reqs = _log(rng, 1, 128)
        return _read(reqs, _log(rng, 1, min(65536, 400000 // reqs)), kv_heads, head, page, block, dtype, order, lens)
    kind = rng.choices(["decode", "drafts", "chunk", "mixed"], [4, 2, 3, 2])[0]
    if kind == "decode":
        reqs = _log(rng, 1, 256)
        c = _attn(reqs, -1, _log(rng, 100, min(131072, 600000 // reqs)), q_heads, kv_heads, head, page, block, dtype, 0,
                  order, lens)
    elif kind == "drafts":
        reqs = _log(rng, 1, 96)
        c = _attn(reqs, rng.randint(2, 9), _log(rng, 100, min(32768, 300000 // reqs)), q_heads, kv_heads, head, page,
                  block, dtype, 0, order, lens)
    elif kind == "chunk":
        c = _attn(1, -_log(rng, 16, 6000), -_log(rng, 1, 10000), q_heads, kv_heads, head, page, block, dtype, 0, order, lens)
    else:
        c = _attn(rng.randint(2, 24), rng.choice([-1, 4]), _log(rng, 200, 4096), q_heads, kv_heads, head, page, block,
                  dtype, _log(rng, 32, 1500), order, lens)
    top = work(listed()[-1])
    while work(c)["bytes"] > 1.25e9 or work(c)["flops"] > top["flops"]:
        c["ctx"] = -max(1, -c["ctx"] // 2) if c["ctx"] < 0 else max(8, c["ctx"] // 2)
        c["new"] = -max(1, -c["new"] * 3 // 4) if c["new"] < 0 else c["new"]
    return c


def _lengths(case):
    """(tokens before, tokens of the call) of each request, by the case alone."""
    r, n = random.Random(case["lens"]), case["reqs"]
    if case["op"] == "write":  # cuts of the tokens; what is before ends anywhere in a page
        cuts = sorted(r.sample(range(1, case["tokens"]), n - 1)) if n > 1 else []
        new = [b - a for a, b in zip([0] + cuts, cuts + [case["tokens"]])]
        return [r.randint(0, 3 * case["page"]) for _ in range(n)], new
    if case["op"] == "read":
        span = case["span"]
        new = [-span if span < 0 else r.randint(max(1, span // 8), span) for _ in range(n)]
        return [r.randint(0, 200) for _ in range(n)], new
    new = [-case["new"] if case["new"] < 0 else r.randint(1, case["new"]) for _ in range(n)]
    ctx = [-case["ctx"] if case["ctx"] < 0 else r.randint(case["ctx"] // 8, case["ctx"]) for _ in range(n)]
    if case["chunk"]:
        new[0] = case["chunk"]
    return ctx, new


def work(case):
    """What one call has to read and write (each byte once) and compute."""
    ctx, new = _lengths(case)
    hk, d, bt, t = case["kv_heads"], case["head"], case["block"], sum(new)
    blocks = sum(-(-(c + n) // bt) - c // bt for c, n in zip(ctx, new))  # that the call's tokens lie in
    if case["op"] == "write":
        hq = case["q_heads"]
        return {"bytes": 2 * t * (hq + 2 * hk) * d + 2 * t * hq * d + 2 * t * hk * d + 2 * blocks * hk + 8 * t + 4 * case["rot"],
                "flops": (hq + hk) * t * (3 * case["rot"] + (4 * d if case["qk_norm"] else 0)) + 4 * t * hk * d}
    pages = sum(-(-(c + n) // case["page"]) for c, n in zip(ctx, new))
    if case["op"] == "read":
        pages -= sum(c // case["page"] for c in ctx)
        return {"bytes": 2 * t * hk * d + 2 * blocks * hk + 2 * 2 * t * hk * d + 4 * pages + 8 * len(ctx), "flops": 2 * t * hk * d}
    hq = case["q_heads"]
    seen = sum(n * c + n * (n + 1) // 2 for c, n in zip(ctx, new))
    kv = sum(c + n for c, n in zip(ctx, new))
    blocks = sum(-(-(c + n) // bt) for c, n in zip(ctx, new))
    return {"bytes": 2 * kv * hk * d + 2 * blocks * hk + 2 * 2 * t * hq * d + 4 * t * hq + 4 * pages + 8 * len(ctx),
            "flops": 4 * seen * hq * d}


# ---------------------------------------------------------------- inputs
def _exponent(top):
    """The smallest e in [E_MIN, E_MAX] with top <= 448 * 2^e = 1.75 * 2^(e + 8)."""
    m, x = torch.frexp(top)
    e = (x - 9 + (m > 0.875)).clamp(E_MIN, E_MAX)
    return torch.where(top == 0, E_MIN, e).to(torch.int32)


def _scales(e):
    return (e + 127).to(torch.uint8).view(E8M0)


def _pool(shape, block, order, channels, gen):
    """A cache [pages, kv heads, page, head size] of codes, its rows in head or in token order, and its
    scales [pages, kv heads, page / block]."""
    p, h, s, d = shape
    out, top = torch.empty((p, s, h, d) if order == "token" else (p, h, s, d), dtype=E4M3, device="cuda"), []
    for a in range(0, p, 4096):  # a part of the pages at a time
        n = min(4096, p - a)
        x = torch.randn((n, h, s, d), generator=gen, device="cuda")
        x *= channels * torch.exp(0.3 * torch.randn((n, h, s, 1), generator=gen, device="cuda"))
        e = _exponent(x.view(n, h, s // block, block * d).abs().amax(-1))
        x = torch.ldexp(x.view(n, h, s // block, block, d), -e[..., None, None]).view(n, h, s, d).to(E4M3)
        (out.transpose(1, 2) if order == "token" else out)[a:a + n].copy_(x)
        top.append(e)
    return out.transpose(1, 2) if order == "token" else out, _scales(torch.cat(top))


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
    ps, hk, d, dt = case["page"], case["kv_heads"], case["head"], TORCH[case["dtype"]]
    ctx, new = _lengths(case)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    need = [-(-(c + n) // ps) for c, n in zip(ctx, new)]
    pool, width = sum(need) + 5, max(need)
    ids = torch.randperm(pool, generator=gen, device="cuda").to(torch.int32)
    at = torch.cumsum(ints(need), 0) - ints(need)
    col = torch.arange(width, device="cuda")[None]
    table = torch.where(col < ints(need)[:, None], ids[(at[:, None] + col).clamp(max=pool - 1)], ids.new_zeros(()))
    cu = torch.nn.functional.pad(torch.cumsum(ints(new), 0), (1, 0)).to(torch.int32)
    loud = torch.rand((hk, 1, d), generator=gen, device="cuda") < 1 / 16  # key channels, by head
    channels = 0.8 + 2.4 * loud
    s = {"case": case, "table": table, "cu": cu, "total": sum(new)}
    s["k_cache"], s["k_scale"] = _pool((pool, hk, ps, d), case["block"], case["order"], channels, gen)
    s["v_cache"], s["v_scale"] = _pool((pool, hk, ps, d), case["block"], case["order"], 0.3 + 0.0 * channels, gen)
    if case["op"] == "read":
        s["first"], s["kv"] = ints(ctx), ints([c + n for c, n in zip(ctx, new)])
        return s
    hq, t = case["q_heads"], sum(new)
    if case["op"] == "attn":
        s["kv"] = ints([c + n for c, n in zip(ctx, new)])
        s["q"] = torch.randn((t, hq, d), generator=gen, device="cuda", dtype=dt)
        s.update(scale=1.0 / math.sqrt(d), max_new=max(new))
        return s
    qkv = torch.randn((t, hq + 2 * hk, d), generator=gen, device="cuda")  # one projection's rows
    qkv *= torch.exp(0.3 * torch.randn((t, hq + 2 * hk, 1), generator=gen, device="cuda"))
    qkv[:, hq:hq + hk] *= channels.transpose(0, 1)
    qkv = qkv.to(dt)
    s.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hk], v=qkv[:, hq + hk:], freqs=_freqs(case["rot"], case["scaled"]).cuda())
    tok = torch.arange(t, device="cuda")
    r = torch.searchsorted(cu[1:].long(), tok, right=True)
    place = ints(ctx).long()[r] + tok - cu.long()[r]
    s["slots"] = (table[r, place // ps].long() * ps + place % ps).to(torch.int32)
    s["pos"] = (place + torch.randint(0, 16000, (len(ctx),), generator=gen, device="cuda")[r]).to(torch.int32)
    s["magnitude"] = 1.0 + 0.1 * math.log(8) if case["scaled"] else 1.0
    for name in ("gamma_q", "gamma_k"):
        s[name] = torch.randn(d, generator=gen, device="cuda") * 0.1 + 1.0
    return s


# ---------------------------------------------------------------- the plain forms
def _rotate(x, cos, sin, rot, interleaved):
    y, a = x.clone(), x[..., :rot]
    lo, hi = (a[..., 0::2], a[..., 1::2]) if interleaved else (a[..., :rot // 2], a[..., rot // 2:])
    p, q = lo * cos - hi * sin, hi * cos + lo * sin
    y[..., :rot] = torch.stack([p, q], -1).flatten(-2) if interleaved else torch.cat([p, q], -1)
    return y


def _codes(x, e):
    return torch.ldexp(x, -e).clamp(-448.0, 448.0).to(E4M3).view(torch.uint8)


def _append(cache, scale, x, slots, block):
    """Quantises x [T, Hkv, D] into the cache at the slots, in place."""
    p, h, ps, d = cache.shape
    nb, t = ps // block, x.shape[0]
    slots = slots.long()
    of = slots // block                                                    # block of the token, over all pages
    top = torch.zeros((p * nb, h), device=x.device)
    top.scatter_reduce_(0, of[:, None].expand(t, h), x.abs().amax(-1), "amax")
    hit = torch.zeros(p * ps, dtype=torch.bool, device=x.device)
    hit[slots] = True
    rows = hit.view(p * nb, block)
    touched, begun = rows.any(1)[:, None], rows[:, 0, None]
    old = scale.view(torch.uint8).to(torch.int32).transpose(1, 2).reshape(p * nb, h) - 127
    fresh = _exponent(top)
    e = torch.where(touched, torch.where(begun, fresh, torch.maximum(old, fresh)), old)
    # rows that a block held, to its new scale
    grown = (touched & ~begun & (e > old)).view(p, nb, h).permute(0, 2, 1)[..., None, None]
    shift = (e - old).view(p, nb, h).permute(0, 2, 1)[..., None, None].expand(p, h, nb, block, 1)
    was = cache.reshape(p, h, nb, block, d)
    now = torch.where(grown, _codes(was.float(), shift), was.view(torch.uint8))
    cache.view(torch.uint8).copy_(now.view(p, h, ps, d))
    cache.view(torch.uint8)[slots // ps, :, slots % ps] = _codes(x, e[of][..., None])
    scale.view(torch.uint8).copy_((e + 127).to(torch.uint8).view(p, nb, h).transpose(1, 2))


def _plain_write(s):
    c, dt = s["case"], s["q"].dtype
    q, k = s["q"].float(), s["k"].float()
    if c["qk_norm"]:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + EPS) * s["gamma_q"]
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + EPS) * s["gamma_k"]
    angle = s["pos"].double()[:, None] * s["freqs"].double().sum(1)  # far positions: the angle in 64 bits
    cos, sin = (torch.cos(angle) * s["magnitude"]).float()[:, None], (torch.sin(angle) * s["magnitude"]).float()[:, None]
    inter = c["pairs"] == "interleaved"
    _append(s["k_cache"], s["k_scale"], _rotate(k, cos, sin, c["rot"], inter), s["slots"], c["block"])
    _append(s["v_cache"], s["v_scale"], s["v"].float(), s["slots"], c["block"])
    return [_rotate(q, cos, sin, c["rot"], inter).to(dt), s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]]


def _plain_read(s):
    c, dt = s["case"], TORCH[s["case"]["dtype"]]
    tok = torch.arange(s["total"], device="cuda")
    cu = s["cu"].long()
    r = torch.searchsorted(cu[1:], tok, right=True)
    place = s["first"].long()[r] + tok - cu[r]
    page, at = s["table"].long()[r, place // c["page"]], place % c["page"]
    k = s["k_cache"].view(torch.uint8)[page, :, at].view(E4M3).float() * \
        s["k_scale"].view(torch.uint8)[page, :, at // c["block"]].view(E8M0).float()[..., None]
    v = s["v_cache"].view(torch.uint8)[page, :, at].view(E4M3).float() * \
        s["v_scale"].view(torch.uint8)[page, :, at // c["block"]].view(E8M0).float()[..., None]
    return [k.to(dt), v.to(dt)]


def _values(s, name, tab):
    """The cache's pages [b, pages, ...] as numbers in 32 bits, [b, kv heads, keys, head size]."""
    cache, scale = s[name + "_cache"].view(torch.uint8)[tab], s[name + "_scale"].view(torch.uint8)[tab]
    b, width, hk, ps, d = cache.shape
    x = cache.view(E4M3).float().reshape(b, width, hk, scale.shape[-1], -1, d)
    return (x * scale.view(E8M0).float()[..., None, None]).view(b, width, hk, ps, d).transpose(1, 2).reshape(b, hk, width * ps, d)


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
    k, v = _values(s, "k", tab), _values(s, "v", tab)
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
# Kept for the process, whose passes all go to one stream of one device, one after the other. (Calls that may overlap
# on the GPU need a workspace each.)
_lib = {}


def _version(S, op, dtype, fixed, **kw):
    """The process's Scm and its version for (op, dtype, fixed), registered at its first use."""
    if "scm" not in _lib:
        _lib["scm"] = S.Scm(device=torch.cuda.current_device(), flags=S.OPT_PDL)
    key = (op, dtype, tuple(fixed))
    if key not in _lib:
        _lib[key] = _lib["scm"].register(S.make_spec(op, dtype, fixed, 1, 1 << 30, device=torch.cuda.current_device(),
                                                     layout=S.LAYOUT_ANY, **kw))
    return _lib["scm"], _lib[key]


def _bind(s):
    """The argument tuple of a state's call and its output tensors (made once, kept with the state)."""
    from paper_2609_37241_gb300 import scm as S
    c = s["case"]
    new = lambda shape, dt: torch.empty(shape, dtype=dt, device="cuda")  # noqa: E731
    dt = {"bf16": S.BF16, "fp16": S.FP16}[c["dtype"]]
    hk, d, ps, bt = c["kv_heads"], c["head"], c["page"], c["block"]
    cache = [s[name] for name in ("k_cache", "v_cache", "k_scale", "v_scale")]
    if c["op"] == "read":
        scm, _ = _version(S, S.OP_PAGED_READ8, dt, [hk, d, ps, bt])
        out = [new((s["total"], hk, d), TORCH[c["dtype"]]) for _ in range(2)]
        return scm, S.make_args(S.OP_PAGED_READ8, [*cache, s["table"], s["cu"], s["first"], *out]), out
    hq = c["q_heads"]
    if c["op"] == "write":
        op = {("half", False): S.OP_ROPE_PAGED_KV8, ("interleaved", False): S.OP_ROPE_PAGED_KV8_INTERLEAVED,
              ("half", True): S.OP_QKNORM_ROPE_PAGED_KV8,
              ("interleaved", True): S.OP_QKNORM_ROPE_PAGED_KV8_INTERLEAVED}[c["pairs"], c["qk_norm"]]
        scm, _ = _version(S, op, dt, [hq, hk, d, c["rot"], ps, bt])
        q_out = new((c["tokens"], hq, d), s["q"].dtype)
        ts = [s["q"], s["k"], s["v"], s["pos"], s["slots"], s["freqs"], q_out, *cache]
        if c["qk_norm"]:
            ts += [s["gamma_q"], s["gamma_k"]]
        return scm, S.make_args(op, ts, eps=EPS, scalar=s["magnitude"]), [q_out, *cache]
    scm, index = _version(S, S.OP_PAGED_ATTN8, dt, [hq, hk, d, ps, bt])
    if ("work", index) not in _lib:  # one for all of the version's calls, zeros before its first use
        _lib["work", index] = torch.zeros(scm.workspace(index), dtype=torch.float32, device="cuda")
    out, lse = new(tuple(s["q"].shape), s["q"].dtype), new((s["q"].shape[0], hq), torch.float32)
    args = S.make_args(S.OP_PAGED_ATTN8, [s["q"], *cache, s["table"], s["cu"], s["kv"], _lib["work", index], out, lse],
                       scalar=s["scale"])
    return scm, args, [out, lse]


def run(state):
    if not own:
        return {"write": _plain_write, "read": _plain_read, "attn": _plain_attn}[state["case"]["op"]](state)
    if "call" not in state:
        state["call"] = _bind(state)
    scm, args, out = state["call"]
    status, _ = scm.invoke(args, torch.cuda.current_stream().cuda_stream)
    if status != 0:
        from paper_2609_37241_gb300 import scm as S
        raise S.ScmError(status, state["case"]["op"])
    return out


# ---------------------------------------------------------------- the definitions in 64 bits
def _numbers(s, name):
    """A cache in 64 bits: its codes' values and its scales."""
    return s[name + "_cache"].to(torch.float64), s[name + "_scale"].to(torch.float64)


def _exact_write(case, s):
    f64 = torch.float64
    rot, inter, ps, bt = case["rot"], case["pairs"] == "interleaved", case["page"], case["block"]
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

    def stored(name, x):
        codes, scales = _numbers(s, name)
        p, hk, _, d = codes.shape
        slots = s["slots"].long()
        block, member = torch.unique(slots // bt, return_inverse=True)
        rows = torch.zeros((block.numel(), bt), dtype=torch.bool, device="cuda")
        rows[member, slots % bt] = True
        most = torch.zeros((block.numel(), hk), dtype=f64, device="cuda")
        most.index_reduce_(0, member, x.abs().amax(-1), "amax")
        near = torch.round(torch.log2(most.clamp(min=1e-300) / 448))  # the smallest of three that holds it
        want = torch.exp2((near - 1 + sum((most > 448 * torch.exp2(near - i)).to(f64) for i in (1, 0))).clamp(E_MIN, E_MAX))
        page, part = block // (ps // bt), block % (ps // bt)
        held = scales[page, :, part]
        now = torch.where(rows[:, :1], want, torch.maximum(want, held))
        scales[page, :, part] = now
        cells = codes.view(p, hk, ps // bt, bt, d) if codes.is_contiguous() else codes.contiguous().view(p, hk, ps // bt, bt, d)
        # rows that a block held stand for the same numbers; where it is begun anew they are left as they were
        cells[page, :, part] *= torch.where(rows[:, :1], torch.ones_like(now), held / now)[..., None, None]
        codes = cells.view(p, hk, ps, d)
        codes[slots // ps, :, slots % ps] = x / now[member][..., None]
        return codes, scales

    k, ke = stored("k", side(s["k"], s["gamma_k"]))
    v, ve = stored("v", s["v"].to(f64))
    return [side(s["q"], s["gamma_q"]), k, v, ke, ve]


def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "write":
        return _exact_write(case, s)
    ctx, new = _lengths(case)
    ps, bt, hk, d = case["page"], case["block"], case["kv_heads"], case["head"]

    def keys(name, b, h, n):
        """The first n keys of request b, head h."""
        pages = s["table"][b, :-(-n // ps)].long()
        codes = s[name + "_cache"].view(torch.uint8)[pages, h].view(E4M3).to(f64).reshape(-1, bt, d)
        return (codes * s[name + "_scale"].view(torch.uint8)[pages, h].view(E8M0).to(f64).reshape(-1, 1, 1)).reshape(-1, d)[:n]

    if case["op"] == "read":
        out = [torch.empty((sum(new), hk, d), dtype=f64, device="cuda") for _ in range(2)]
        at = 0
        for b, (c, n) in enumerate(zip(ctx, new)):
            for h in range(hk):
                for o, name in zip(out, ("k", "v")):
                    o[at:at + n, h] = keys(name, b, h, c + n)[c:]
            at += n
        return out
    if work(case)["flops"] > 4e12:
        return None
    hq = case["q_heads"]
    out = torch.empty(s["q"].shape, dtype=f64, device="cuda")
    lse = torch.empty(s["q"].shape[:2], dtype=f64, device="cuda")
    first = 0
    for b, (c, n) in enumerate(zip(ctx, new)):
        last = c + torch.arange(n, device="cuda")
        for h in range(hk):
            k, v = keys("k", b, h, c + n), keys("v", b, h, c + n)
            for a in range(h * (hq // hk), (h + 1) * (hq // hk)):
                z = (s["q"][first:first + n, a].to(f64) @ k.T) * s["scale"]
                z = z.masked_fill(torch.arange(c + n, device="cuda") > last[:, None], -math.inf)
                lse[first:first + n, a] = torch.logsumexp(z, 1)
                out[first:first + n, a] = torch.softmax(z, 1) @ v
        first += n
    return [out, lse]
