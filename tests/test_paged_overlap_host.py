"""Which pairs of caches the launch precondition takes: k and v may lie in one buffer, interleaved in any
dimension, as long as no element has bytes of both (no GPU)."""
import random

import pytest

from tests.test_paged_host import BASE, rope_args

H, D, PS, P = 2, 64, 16, 8


@pytest.fixture(scope="module")
def S(built_lib):
    from paper_2609_37241_gb300 import scm
    return scm


@pytest.fixture(scope="module")
def scm(S):
    s = S.Scm(flags=S.OPT_DRY_RUN)
    s.register(S.make_spec(S.OP_ROPE_PAGED_KV, S.BF16, [4, 2, 64, 32, 16], 1, 64, layout=S.LAYOUT_ANY))
    yield s
    s.close()


def invoke(S, scm, pages, strides, offset):
    """k at BASE * 16, v `offset` elements behind it, both [pages, H, PS, D] with these strides."""
    t, kw = rope_args(S, P=pages)
    t[7] = dict(t[7], addr=16 * BASE, stride=tuple(strides) + (1,))
    t[8] = dict(t[7], addr=16 * BASE + 2 * offset)
    return scm.invoke(S.make_args(S.OP_ROPE_PAGED_KV, t, **kw))[0]


@pytest.mark.parametrize("strides,offset", [  # of pages, heads, rows; v's offset
    ((2 * H * PS * D, PS * D, D), H * PS * D),           # [P, 2, H, ps, D]
    ((2 * H * PS * D, 2 * PS * D, D), PS * D),           # [P, H, 2, ps, D]
    ((2 * H * PS * D, 2 * PS * D, 2 * D), D),            # [P, H, ps, 2, D]
    ((2 * H * PS * D, D, 2 * H * D), H * D),             # [P, ps, 2, H, D]
    ((2 * H * PS * D, 2 * D, 2 * H * D), D),             # [P, ps, H, 2, D]
    ((PS * D, 2 * P * PS * D, D), P * PS * D),           # [H, 2, P, ps, D]
    ((2 * PS * D, 2 * P * PS * D, D), PS * D),           # [H, P, 2, ps, D]
])
def test_k_and_v_of_one_buffer(S, scm, strides, offset):
    assert invoke(S, scm, P, strides, offset) == S.OK
    for wrong in (0, 8, D // 2, offset - 8, offset + 8):  # no longer between k's elements
        assert invoke(S, scm, P, strides, wrong) == S.ERR_INVALID, wrong


def test_against_the_sets_of_elements(S, scm):
    r = random.Random(5)
    seen = {True: 0, False: 0}
    for _ in range(400):
        dims = [r.choice([1, 2, 3]), H, PS]   # pages, heads, rows
        strides, span = [0, 0, 0], D
        for k in r.sample(range(3), 3):       # in any order, each past the span of those before it
            strides[k] = (span + 7) // 8 * 8 + 8 * r.choice([0, 0, 8, 8, 16, 40])
            span += (dims[k] - 1) * strides[k]
        offset = 8 * r.randrange(0, span // 8 + 8) if r.random() < 0.5 else \
            sum(r.randrange(0, 2) * s for s in strides) + 8 * r.choice([0, 8, 8, 16])
        first = {p * strides[0] + h * strides[1] + t * strides[2] for p in range(dims[0]) for h in range(H) for t in range(PS)}
        shared = any(a + offset + e in first for a in first for e in range(-D + 1, D))
        want = S.ERR_INVALID if shared else S.OK
        assert invoke(S, scm, dims[0], strides, offset) == want, (dims, strides, offset)
        seen[shared] += 1
    assert min(seen.values()) > 40
