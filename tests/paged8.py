"""The paged ops over caches held in 8 bits, in 64 bits on the CPU, for their tests."""
import numpy as np
import torch

from tests import paged as R

E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
LO, HI = -32, 32


def exponent(top):
    """The smallest e in [LO, HI] with top <= 448 * 2^e, by trying them."""
    for e in range(LO, HI):
        if top <= 448.0 * 2.0 ** e:
            return e
    return HI


def scale_bytes(e):
    return torch.as_tensor(e + 127, dtype=torch.uint8).view(E8M0)


def values(codes, scales):
    """A cache [P,H,ps,D] of codes with scales [P,H,nb] as numbers."""
    p, h, ps, d = codes.shape
    nb = scales.shape[2]
    e = (scales.cpu().view(torch.uint8).double() - 127).clamp(LO, HI)
    x = codes.cpu().contiguous().view(E4M3).to(torch.float64).reshape(p, h, nb, ps // nb, d)
    return (x * torch.exp2(e)[..., None, None]).reshape(p, h, ps, d)


def rounded(x):
    """The nearest e4m3 value of x (fp64), ties to even, +-448 beyond the range: the grid's steps are 2^(floor(log2) - 3)."""
    a = np.abs(x)
    with np.errstate(divide="ignore"):
        step = np.exp2(np.maximum(np.floor(np.log2(np.where(a == 0, 1, a))), -6) - 3)
    return np.copysign(np.minimum(np.where(np.isfinite(x), np.round(a / np.where(np.isfinite(step), step, 1)) * step, np.inf), 448.0), x)


def codes_of(x):
    return torch.from_numpy(rounded(x)).to(torch.float32).to(E4M3).view(torch.uint8).numpy()


def append(codes, exps, x, slots, skip, bt):
    """Writes rows x [T,H,D] (fp64) into codes [P,H,ps,D] (uint8) with exponents exps [P,H,nb] (int) at the slots, in
    place. skip: tokens dropped for their position."""
    P, H, ps, D = codes.shape
    nb = ps // bt
    rows = {}
    for t, s in enumerate(slots):
        if 0 <= s < P * ps:
            rows.setdefault(s // bt, []).append((s % bt, t))
    for block, members in rows.items():
        p, part = block // nb, block % nb
        begun = any(r == 0 for r, _ in members)
        live = [(r, t) for r, t in members if not skip[t]]
        for h in range(H):
            tops = [np.abs(x[t, h][~np.isnan(x[t, h])]).max(initial=0.0) for _, t in live]
            e, old = exponent(max(tops, default=0.0)), int(exps[p, h, part])
            lo = part * bt
            if not begun:
                e = max(e, old)
                if e > old:
                    others = [r for r in range(bt) if r not in {m for m, _ in members}]
                    was = torch.from_numpy(codes[p, h, lo:lo + bt][others]).view(E4M3).to(torch.float64).numpy()
                    codes[p, h, lo + np.array(others, int)] = codes_of(was * 2.0 ** (old - e)) if others else 0
            exps[p, h, part] = e
            for r, t in live:
                codes[p, h, lo + r] = codes_of(x[t, h] * 2.0 ** -e)


def pool(g, P, Hkv, ps, D, bt, order, size=1.0):
    """Codes and scales of a k and a v cache on the GPU, of random values: order as paged.pool."""
    def one(pad):
        x = g.standard_normal((P, Hkv, ps // bt, bt, D)) * size * np.exp(g.standard_normal((P, Hkv, ps // bt, 1, 1)))
        top = np.abs(x).max((3, 4))
        e = np.vectorize(exponent)(top)
        c = torch.from_numpy(codes_of(x * np.exp2(-e.astype(float))[..., None, None])).view(P, Hkv, ps, D)
        return c, torch.from_numpy(e)
    (kc, ke), (vc, ve) = one(0), one(0)
    if order == "token":
        kc, vc = (x.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3) for x in (kc, vc))
    elif order == "pair":
        kv = torch.stack([kc, vc], 1).cuda()
        kc, vc = kv[:, 0], kv[:, 1]
    elif order == "padded":
        big = [torch.zeros(P, Hkv, ps, D + n, dtype=torch.uint8, device="cuda") for n in (16, 32)]
        for b, x in zip(big, (kc, vc)):
            b[..., :D] = x.cuda()
        kc, vc = (b[..., :D] for b in big)
    elif order == "record":  # a page's k, v and their scales behind one another
        n, m = Hkv * ps * D, Hkv * (ps // bt)
        rec = torch.zeros(P, -(-(2 * n + 2 * m) // 16) * 16, dtype=torch.uint8, device="cuda")
        parts = []
        for i, x in enumerate((kc, vc)):
            y = rec[:, i * n:(i + 1) * n].view(P, Hkv, ps, D)
            y.copy_(x.cuda())
            parts.append(y)
        for i, e in enumerate((ke, ve)):
            y = rec[:, 2 * n + i * m:2 * n + (i + 1) * m].view(P, Hkv, ps // bt)
            y.copy_((e + 127).to(torch.uint8).cuda())
            parts.append(y)
        return [parts[0].view(E4M3), parts[1].view(E4M3), parts[2].view(E8M0), parts[3].view(E8M0)]
    else:
        kc, vc = kc.cuda(), vc.cuda()
    ks, vs = (scale_bytes(e).cuda() for e in (ke, ve))
    if order == "token":  # a block's heads side by side
        ks, vs = (s.view(torch.uint8).permute(0, 2, 1).contiguous().permute(0, 2, 1).view(E8M0) for s in (ks, vs))
    return [kc.view(E4M3), vc.view(E4M3), ks, vs]


def batch(g, new, kv, Hq, Hkv, D, ps, bt, dtype, order="head", tail=0, strided=False, spare=3, size=1.0):
    """As paged.batch: requests with scattered pages; every cache row that no request owns holds NaN codes, and every
    scale without such a row the NaN byte."""
    need = [-(-L // ps) for L in kv]
    P, M = sum(need) + spare, max(max(need, default=0), 1) + 1
    kc, vc, ks, vs = pool(g, P, Hkv, ps, D, bt, order, size)
    ids = g.permutation(P)
    table = np.full((len(kv), M), 2 ** 30, np.int32)
    used = torch.zeros(P, ps, dtype=torch.bool)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        for j in range(n):
            used[int(ids[at + j]), :min(ps, kv[b] - j * ps)] = True
        at += n
    dead = (~used).cuda()[:, None, :, None]
    for c in (kc, vc):
        c.view(torch.uint8).masked_fill_(dead, 0x7f)
    empty = (~used.view(P, ps // bt, bt).any(2)).cuda()[:, None]
    for s in (ks, vs):
        s.view(torch.uint8).masked_fill_(empty, 255)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = int(cu[-1]) + tail
    q = torch.from_numpy(g.standard_normal((T, Hq, D), dtype=np.float32)).to(R.TORCH[dtype]).cuda()
    out = torch.full_like(q, float("nan"))
    if strided:
        big = torch.zeros(T, Hq + 2, D, dtype=R.TORCH[dtype], device="cuda")
        big[:, 1:Hq + 1] = q
        q = big[:, 1:Hq + 1]
        out = torch.full((T, Hq + 1, D), float("nan"), dtype=R.TORCH[dtype], device="cuda")[:, :Hq]
    i32 = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()  # noqa: E731
    return dict(q=q, kc=kc, vc=vc, ks=ks, vs=vs, table=i32(table), cu=i32(cu), kv=i32(kv), out=out,
                lse=torch.full((T, Hq), float("nan"), device="cuda"))


def attention(q, k, v, e, table, cu, kv, ps, scale):
    """(out, lse, weight, level) in fp64 of k and v [P,H,ps,D] with v's exponents e [P,H,ps]: weight = sum_j softmax_j |v_j|,
    level = max_j softmax_j 2^e_j, the size of the largest numerator."""
    T, Hq, D = q.shape
    G = Hq // k.shape[1]
    out, lse = torch.zeros(T, Hq, D, dtype=torch.float64), torch.full((T, Hq), -np.inf, dtype=torch.float64)
    wgt, level = torch.zeros_like(out), torch.zeros(T, Hq, 1, dtype=torch.float64)
    for b in range(len(kv)):
        n, L = cu[b + 1] - cu[b], kv[b]
        if n == 0 or L == 0:
            continue
        pages = table[b, :-(-L // ps)].long()
        kb, vb = (x[pages].transpose(1, 2).reshape(-1, x.shape[1], D)[:L].repeat_interleave(G, 1) for x in (k, v))
        eb = e[pages].transpose(1, 2).reshape(-1, e.shape[1])[:L].repeat_interleave(G, 1)
        s = torch.einsum("ihd,jhd->hij", q[cu[b]:cu[b + 1]].double(), kb) * scale
        seen = torch.arange(L)[None] <= (L - n + torch.arange(n))[:, None]
        s = s.masked_fill(~seen, -np.inf)
        any_ = seen.any(1)
        p = torch.zeros_like(s)
        p[:, any_] = torch.softmax(s[:, any_], -1)
        rows = slice(cu[b], cu[b + 1])
        out[rows] = torch.einsum("hij,jhd->ihd", p, vb)
        wgt[rows] = torch.einsum("hij,jhd->ihd", p, vb.abs())
        level[rows] = (p * torch.exp2(eb).T[:, None]).amax(-1).T[..., None]
        lse[rows] = torch.logsumexp(s, -1).T
    return out, lse, wgt, level


def reference(b, ps, scale):
    """attention() of a batch."""
    k, v = (torch.nan_to_num(values(b[c].view(torch.uint8), b[s]), nan=0.0) for c, s in (("kc", "ks"), ("vc", "vs")))
    e = (b["vs"].cpu().view(torch.uint8).double() - 127).clamp(LO, HI)
    e = e.repeat_interleave(ps // e.shape[2], 2)
    return attention(b["q"].cpu(), k, v, e, b["table"].cpu(), b["cu"].tolist(), b["kv"].tolist(), ps, scale)


def tolerance(ref, wgt, level, dtype, n_keys):
    """|out - ref| bound: the output's rounding; the numerators' rounding to fp16, 2^-11 of each, and below fp16's normal
    numbers half of 2^-24 where the largest is at least 2^7 (2^-32 of the largest, times codes up to 448, n_keys times);
    the scores' error, below 2^-13 for inputs as these (D products in fp32; q held within 2^-21 of its row's largest
    element), so 2^-12 of the weights."""
    return 1.01 * R.UNIT[dtype] * ref.abs() + (1.05 * 2.0 ** -11 + 2.0 ** -12) * wgt + n_keys * 2.0 ** -32 * 448 * level
