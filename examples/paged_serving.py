"""A small serving loop on the paged operators: requests of unequal lengths share a pool of cache
pages; each step hands pages to the new tokens (PAGE_MAP), rotates q and k and appends k, v to the
pages (ROPE_PAGED_KV) and attends to all of a request's pages (PAGED_ATTN), through one invoke_seq.

    python examples/paged_serving.py [steps]

The first step takes the prompts, the next ones a token per request; after every step the output
is compared with a plain computation over each request's own tokens. Random data and one layer: the
projections before and after, which would make q, k, v and use the output, are left out.
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_37241_gb300 import scm as S  # noqa: E402

HQ, HKV, D, PAGE, POOL, WIDTH = 32, 8, 128, 16, 1024, 64  # WIDTH: pages of a request at most
THETA, CONTEXT, FACTOR = 500000.0, 8192, 8.0                # positions rescaled to 8 times the trained context


class Engine:
    def __init__(self, requests, rows):
        """rows: new tokens of a step at most."""
        dev = torch.cuda.current_device()
        self.scm = S.Scm(device=dev, flags=S.OPT_PDL)
        self.scm.register(S.make_spec(S.OP_PAGE_MAP, S.I32, [], 1, 4096, align_bytes=4, device=dev))
        self.scm.register(S.make_spec(S.OP_ROPE_PAGED_KV, S.BF16, [HQ, HKV, D, D, PAGE], 1, 1 << 20, layout=S.LAYOUT_ANY,
                                      device=dev))
        attn = self.scm.register(S.make_spec(S.OP_PAGED_ATTN, S.BF16, [HQ, HKV, D, PAGE], 1, 1 << 20,
                                             layout=S.LAYOUT_ANY, device=dev))
        i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
        bf = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.ctx, self.new, self.kv, self.cu = i32(requests), i32(requests), i32(requests), i32(requests + 1)
        self.free, self.head, self.head_out = torch.randperm(POOL, device="cuda").to(torch.int32), i32(1), i32(1)
        self.table = i32(requests, WIDTH)
        self.pos, self.slot = i32(rows), i32(rows)
        self.qkv = bf(rows, HQ + 2 * HKV, D)
        self.q_rot, self.out, self.lse = bf(rows, HQ, D), bf(rows, HQ, D), torch.zeros(rows, HQ, device="cuda")
        self.k_cache, self.v_cache = bf(POOL, HKV, PAGE, D), bf(POOL, HKV, PAGE, D)
        self.work = torch.zeros(self.scm.workspace(attn), device="cuda")
        self.freqs = S.rope_freqs(THETA, D, S.ROPE_PARTS, FACTOR, CONTEXT)
        self.magnitude, self.scale = 1.0 + 0.1 * math.log(FACTOR), 1.0 / math.sqrt(D)
        q, k, v = self.qkv.split([HQ, HKV, HKV], 1)
        # One argument array for all steps: the buffers stay, their contents change. It holds addresses, not
        # tensors, so the engine keeps every buffer.
        self.calls = (S.trident_args * 3)(
            S.make_args(S.OP_PAGE_MAP, [self.ctx, self.new, self.free, self.head, self.table, self.cu, self.kv, self.pos,
                                        self.slot, self.head_out], scalar=PAGE),
            S.make_args(S.OP_ROPE_PAGED_KV, [q, k, v, self.pos, self.slot, self.freqs, self.q_rot, self.k_cache,
                                               self.v_cache], scalar=self.magnitude),
            S.make_args(S.OP_PAGED_ATTN, [self.q_rot, self.k_cache, self.v_cache, self.table, self.cu, self.kv, self.work,
                                         self.out, self.lse], scalar=self.scale))

    def step(self, new, qkv):
        """new: tokens of each request; qkv [sum(new), HQ + 2 HKV, D]. Returns the attention's output."""
        self.new.copy_(torch.tensor(new, dtype=torch.int32))
        self.qkv[:qkv.shape[0]] = qkv
        status, _ = self.scm.invoke_seq(self.calls, torch.cuda.current_stream().cuda_stream)
        if status != S.OK:
            raise S.ScmError(status, "invoke_seq")
        self.ctx.copy_(self.kv)
        self.head.copy_(self.head_out)
        return self.out[:qkv.shape[0]]


def rotate(x, pos, freqs, magnitude):
    a = pos.double()[:, None, None] * freqs
    c, s = magnitude * torch.cos(a), magnitude * torch.sin(a)
    lo, hi = x[..., :D // 2].double(), x[..., D // 2:].double()
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)


def main(steps):
    torch.manual_seed(0)
    prompts = [500, 3, 77, 240, 1]
    engine = Engine(len(prompts), 1024)
    freqs = engine.freqs.double().sum(1)
    keys = [torch.zeros(0, HKV, D, dtype=torch.float64, device="cuda") for _ in prompts]
    values = [k.clone() for k in keys]
    for step in range(steps + 1):
        new = prompts if step == 0 else [1] * len(prompts)
        qkv = torch.randn(sum(new), HQ + 2 * HKV, D, device="cuda").bfloat16()
        out, worst = engine.step(new, qkv), 0.0
        at = 0
        for b, n in enumerate(new):
            c = keys[b].shape[0]
            pos = torch.arange(c, c + n, device="cuda")
            q, k, v = qkv[at:at + n].split([HQ, HKV, HKV], 1)
            q, k = (rotate(x, pos, freqs, engine.magnitude).bfloat16().double() for x in (q, k))
            keys[b], values[b] = torch.cat([keys[b], k]), torch.cat([values[b], v.double()])
            g = HQ // HKV
            s = torch.einsum("ihd,jhd->hij", q, keys[b].repeat_interleave(g, 1)) * engine.scale
            s = s.masked_fill(torch.arange(c + n, device="cuda") > pos[:, None], -math.inf)
            ref = torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), values[b].repeat_interleave(g, 1))
            worst = max(worst, ((out[at:at + n].double() - ref).norm() / ref.norm()).item())
            at += n
        status = S.trident_scm_device_status(engine.scm.h, torch.cuda.current_stream().cuda_stream)[1]
        print(f"step {step}: {sum(new)} new tokens, {int(engine.head)} pages taken, device status {status}, "
              f"relative error {worst:.1e}")
        assert status == 0 and worst < 1e-2
    engine.scm.close()


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 20)
