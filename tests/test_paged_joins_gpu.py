"""Paged attention whose units are cut and joined at every block, many times over: the same bits each time."""
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


def reference(b, Hq, Hkv, ps, scale):
    """(out, lse, weight) of R.attention, a head at a time on the GPU."""
    T, _, D = b["q"].shape
    out, wgt = (torch.zeros(T, Hq, D, dtype=torch.float64, device="cuda") for _ in range(2))
    lse = torch.full((T, Hq), -np.inf, dtype=torch.float64, device="cuda")
    cu = b["cu"].tolist()
    for r, L in enumerate(b["kv"].tolist()):
        n, rows = cu[r + 1] - cu[r], slice(cu[r], cu[r + 1])
        if n == 0 or L == 0:
            continue
        pages = b["table"][r, :-(-L // ps)].long()
        seen = torch.arange(L, device="cuda")[None] <= (L - n + torch.arange(n, device="cuda"))[:, None]
        for h in range(Hq):
            k, v = (b[c][pages, h * Hkv // Hq].reshape(-1, D)[:L].double() for c in ("kc", "vc"))
            s = (b["q"][rows, h].double() @ k.T * scale).masked_fill(~seen, -np.inf)
            p = torch.softmax(s, -1).masked_fill(~seen.any(1, keepdim=True), 0.0)
            out[rows, h], wgt[rows, h], lse[rows, h] = p @ v, p @ v.abs(), torch.logsumexp(s, -1)
    return out, lse, wgt


def call(S, s, index, b, work, scale):
    args = S.make_args(S.OP_PAGED_ATTN, [b["q"], b["kc"], b["vc"], b["table"], b["cu"], b["kv"], work, b["out"], b["lse"]],
                       scalar=scale)
    assert s.invoke(args, stream()) == (S.OK, index), S.trident_scm_last_error()


def check(b, ref, dt, n_keys):
    out, lse, wgt = ref
    assert ((b["out"].double() - out).abs() <= R.attn_tolerance(out, wgt, dt, n_keys, 5.0)).all()
    none = torch.isinf(lse)
    assert torch.equal(torch.isinf(b["lse"]), none) and (b["out"][none] == 0).all()
    assert ((b["lse"].double() - lse).abs() <= R.LSE_TOLERANCE + 2.0 ** -21 * lse.abs())[~none].all()


@pytest.mark.parametrize("new,kv,Hq,Hkv,D", [
    ([1] * 37, [2500] * 37, 32, 8, 128),        # few rows: 296 units a little longer than a block's run
    ([2] * 9, [300 + k for k in range(9)], 28, 4, 64),
    ([1] * 40, [333] * 40, 8, 2, 256),
    ([100], [8000], 160, 160, 64),              # many rows: 160 units of 100 over 152 blocks
])
def test_cut_units_many_times(S, new, kv, Hq, Hkv, D):
    ps, scale = 16, 1.0 / D ** 0.5
    s = S.Scm(flags=S.OPT_PDL)
    index = s.register(S.make_spec(S.OP_PAGED_ATTN, S.BF16, [Hq, Hkv, D, ps], 1, 1 << 20, layout=S.LAYOUT_ANY))
    work = torch.zeros(s.workspace(index), device="cuda")
    b = R.batch(np.random.default_rng(D), new, kv, Hq, Hkv, D, ps, S.BF16)
    call(S, s, index, b, work, scale)
    check(b, reference(b, Hq, Hkv, ps, scale), S.BF16, max(kv))
    first, differ = (b["out"].clone(), b["lse"].clone()), torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(300):
        b["out"].fill_(float("nan"))
        b["lse"].fill_(float("nan"))
        call(S, s, index, b, work, scale)
        differ += (b["out"] != first[0]).sum() + (b["lse"] != first[1]).sum()
    assert differ.item() == 0
    assert S.trident_scm_device_status(s.h, stream())[1] == 0
    s.close()


@pytest.mark.parametrize("D", [64, 128, 256])
def test_both_kernels_while_another_stream_holds_the_sms(S, D):
    """A call that launches both kernels, the tile kernel's work cut over every block, beside long chunks of a
    second stream, at several distances in time: the second kernel's blocks start when those leave the SMs,
    some after the others have ended. Then the same call alone on the same workspace."""
    ps, Hq, Hkv, scale = 16, 32, 8, 1.0 / D ** 0.5
    s = S.Scm(flags=S.OPT_PDL)
    index = s.register(S.make_spec(S.OP_PAGED_ATTN, S.BF16, [Hq, Hkv, D, ps], 1, 1 << 20, layout=S.LAYOUT_ANY))
    new, kv = [1, 64, 1, 64, 1], [700, 9728, 3000, 9728, 33]
    g = np.random.default_rng(9)
    b = R.batch(g, new, kv, Hq, Hkv, D, ps, S.BF16)
    long = R.batch(g, [2048], [8192], Hq, Hkv, D, ps, S.BF16)
    work, long_work = (torch.zeros(s.workspace(index), device="cuda") for _ in range(2))
    call(S, s, index, b, work, scale)
    check(b, reference(b, Hq, Hkv, ps, scale), S.BF16, max(kv))
    call(S, s, index, long, long_work, scale)
    alone, long_alone = (b["out"].clone(), b["lse"].clone()), long["out"].clone()
    side, main = torch.cuda.Stream(), torch.cuda.current_stream()
    for trial in range(48):
        for x in (b["out"], b["lse"], long["out"]):
            x.fill_(float("nan"))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(6):
                call(S, s, index, long, long_work, scale)
        torch.cuda._sleep(1 + trial * 30000)  # one thread, up to 0.7 ms
        for _ in range(3):
            call(S, s, index, b, work, scale)
        torch.cuda.synchronize()
        assert torch.equal(b["out"], alone[0]) and torch.equal(b["lse"], alone[1]), trial
        assert torch.equal(long["out"], long_alone), trial
        b["out"].fill_(float("nan"))
        call(S, s, index, b, work, scale)
        assert torch.equal(b["out"], alone[0]), trial
        assert S.trident_scm_device_status(s.h, main.cuda_stream)[1] == 0
    s.close()


def test_versions_of_different_head_sizes_share_a_workspace(S):
    """Heads of 128, 64 and 256 in turn on one workspace, each call with cut units of both kernels: each
    leaves partial results where it may, and what the next one counts with at zero."""
    Hq, Hkv, ps = 32, 8, 16
    s = S.Scm(flags=S.OPT_PDL)
    heads = (128, 64, 256)
    index = {D: s.register(S.make_spec(S.OP_PAGED_ATTN, S.BF16, [Hq, Hkv, D, ps], 1, 1 << 20, layout=S.LAYOUT_ANY))
             for D in heads}
    work = torch.zeros(max(s.workspace(i) for i in index.values()), device="cuda")
    cases = {}
    for D in heads:
        b = R.batch(np.random.default_rng(D + 1), [1, 64, 1, 64], [2700, 9728, 3000, 9728], Hq, Hkv, D, ps, S.BF16)
        cases[D] = b, reference(b, Hq, Hkv, ps, 1.0 / D ** 0.5)
    for D in heads + heads[::-1] + heads:
        b, ref = cases[D]
        b["out"].fill_(float("nan"))
        b["lse"].fill_(float("nan"))
        call(S, s, index[D], b, work, 1.0 / D ** 0.5)
        check(b, ref, S.BF16, 9728)
    assert S.trident_scm_device_status(s.h, stream())[1] == 0
    s.close()
