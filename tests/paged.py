"""The paged ops in 64 bits (numpy / torch on the CPU), and random paged batches, for their tests."""
import numpy as np
import torch

from paper_2609_37241_gb300 import scm as S

TORCH = {S.BF16: torch.bfloat16, S.FP16: torch.float16}
UNIT = {S.BF16: 2.0 ** -8, S.FP16: 2.0 ** -11}  # half a step relative to the value


def page_map(ctx, new, free, head, table, ps, N):
    """PAGE_MAP's outputs (cu, kv, pos, slot, head, table, ok) as plain Python integers."""
    B, M = len(ctx), table.shape[1]
    table = table.copy()
    need = [-(-(c + n) // ps) for c, n in zip(ctx, new)]
    have = [-(-c // ps) for c in ctx]
    taken = sum(need) - sum(have)
    ok = (min(ctx, default=0) >= 0 and min(new, default=0) >= 0 and sum(new) <= N and max(need, default=0) <= M
          and 0 <= head <= len(free) and taken <= len(free) - head)
    pos, slot = [0] * N, [-1] * N
    if not ok:
        return [0] * (B + 1), list(ctx), pos, slot, head, table, False
    cu, at = [0], head
    for b in range(B):
        for j in range(have[b], need[b]):
            table[b, j] = free[at]
            at += 1
        for i in range(new[b]):
            p = ctx[b] + i
            pos[cu[b] + i] = p
            s = int(table[b, p // ps]) * ps + p % ps
            slot[cu[b] + i] = s if 0 <= s < 2 ** 31 else -1
        cu.append(cu[b] + new[b])
    return cu, [c + n for c, n in zip(ctx, new)], pos, slot, at, table, True


def rotate(x, pos, freqs, mag, inter, gamma=None, eps=0.0):
    """RoPE of x [T,H,D] (fp64) by freqs [R/2] (fp64), optionally after RMSNorm."""
    if gamma is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gamma
    R = 2 * freqs.numel()
    a = pos.double()[:, None] * freqs
    c, s = (mag * torch.cos(a))[:, None], (mag * torch.sin(a))[:, None]
    i = torch.arange(R // 2)
    u, v = (2 * i, 2 * i + 1) if inter else (i, i + R // 2)
    y = x.clone()
    y[..., u] = x[..., u] * c - x[..., v] * s
    y[..., v] = x[..., v] * c + x[..., u] * s
    return y


def attention(q, kc, vc, table, cu, kv, ps, scale):
    """(out, lse, weight) in fp64: weight = sum_j softmax_j |v_j|, the scale of out's rounding errors."""
    T, Hq, D = q.shape
    G = Hq // kc.shape[1]
    out, lse = torch.zeros(T, Hq, D, dtype=torch.float64), torch.full((T, Hq), -np.inf, dtype=torch.float64)
    wgt = torch.zeros(T, Hq, D, dtype=torch.float64)
    for b in range(len(kv)):
        n, L = cu[b + 1] - cu[b], kv[b]
        if n == 0 or L == 0:
            continue
        pages = table[b, :-(-L // ps)].long()
        k = kc[pages].transpose(1, 2).reshape(-1, kc.shape[1], D)[:L].double()
        v = vc[pages].transpose(1, 2).reshape(-1, kc.shape[1], D)[:L].double()
        k, v = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
        s = torch.einsum("ihd,jhd->hij", q[cu[b]:cu[b + 1]].double(), k) * scale
        seen = torch.arange(L)[None] <= (L - n + torch.arange(n))[:, None]
        s = s.masked_fill(~seen, -np.inf)
        any_ = seen.any(1)
        p = torch.zeros_like(s)
        p[:, any_] = torch.softmax(s[:, any_], -1)
        out[cu[b]:cu[b + 1]] = torch.einsum("hij,jhd->ihd", p, v)
        wgt[cu[b]:cu[b + 1]] = torch.einsum("hij,jhd->ihd", p, v.abs())
        lse[cu[b]:cu[b + 1]] = torch.logsumexp(s, -1).T
    return out, lse, wgt


def pool(g, P, Hkv, ps, D, dtype, order):
    """A cache [P,Hkv,ps,D] on the GPU, by `order`: head (dense), token (row-major tokens), pair (k
    and v of one buffer: returns both), padded (rows longer than D)."""
    def rand(*shape):
        return torch.from_numpy(g.standard_normal(shape, dtype=np.float32)).to(TORCH[dtype]).cuda()
    if order == "head":
        return rand(P, Hkv, ps, D), rand(P, Hkv, ps, D)
    if order == "token":
        return rand(P, ps, Hkv, D).transpose(1, 2), rand(P, ps, Hkv, D).transpose(1, 2)
    if order == "pair":
        kv = rand(P, 2, Hkv, ps, D)
        return kv[:, 0], kv[:, 1]
    return rand(P, Hkv, ps, D + 8)[..., :D], rand(P, Hkv, ps, D + 16)[..., :D]


def batch(g, new, kv, Hq, Hkv, D, ps, dtype, order="head", tail=0, strided=False, spare=3):
    """A batch of requests with scattered pages; every cache row that no request owns is NaN."""
    need = [-(-L // ps) for L in kv]
    P, M = sum(need) + spare, max(max(need, default=0), 1) + 1
    kc, vc = pool(g, P, Hkv, ps, D, dtype, order)
    ids = g.permutation(P)
    table = np.full((len(kv), M), 2 ** 30, np.int32)  # entries past a request's pages are never read
    used = torch.zeros(P, ps, dtype=torch.bool)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        for j in range(n):
            used[int(ids[at + j]), :min(ps, kv[b] - j * ps)] = True
        at += n
    dead = (~used).cuda()[:, None, :, None]
    kc.masked_fill_(dead, float("nan"))
    vc.masked_fill_(dead, float("nan"))
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = int(cu[-1]) + tail
    q = torch.from_numpy(g.standard_normal((T, Hq, D), dtype=np.float32)).to(TORCH[dtype]).cuda()
    out = torch.full_like(q, float("nan"))
    if strided:
        big = torch.zeros(T, Hq + 2, D, dtype=TORCH[dtype], device="cuda")
        big[:, 1:Hq + 1] = q
        q = big[:, 1:Hq + 1]
        out = torch.full((T, Hq + 1, D), float("nan"), dtype=TORCH[dtype], device="cuda")[:, :Hq]
    i32 = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()  # noqa: E731
    return dict(q=q, kc=kc, vc=vc, table=i32(table), cu=i32(cu), kv=i32(kv), out=out,
                lse=torch.full((T, Hq), float("nan"), device="cuda"))


def attn_tolerance(ref, wgt, dtype, n_keys, vmax):
    """|out - ref| bound: the output's rounding, the numerators' rounding (each within UNIT of itself, so
    within UNIT * wgt in all, also through the denominators where they are those of the rounded ones), the
    scores' fp32 error (D products, below 2^-13 for the inputs here), and for fp16 numerators below the
    smallest step, 2^-25 each against a denominator of at least 1."""
    u = UNIT[dtype]
    return u * ref.abs() * (1 + u) + (1.05 * u + 2.0 ** -12) * wgt + (n_keys * 2.0 ** -25 * vmax if dtype == S.FP16 else 0.0)


# the scores' error, 2^-13 at most for N(0, 1) inputs, and 2^-22 of the exponentials and the sum (and, where
# the scores are large, their own roundings: a few 2^-24 of them)
LSE_TOLERANCE = 2e-4
