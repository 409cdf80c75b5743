"""The binding beside a torch without the 8-bit float types: the ops that do not take them work as ever."""
import subprocess
import sys

import pytest

CHILD = """
import torch
for name in {missing}:
    delattr(torch, name)
from paper_2609_37241_gb300 import scm as S
x, out = (torch.zeros(4, 64, dtype=torch.bfloat16) for _ in range(2))
s = S.Scm(flags=S.OPT_DRY_RUN)
a = S.make_args(S.OP_SILU, [x, out])
assert [a.t[i].dtype for i in range(2)] == [S.BF16, S.BF16]
seen = []
s.set_tree_hook(lambda scm, nodes, nargs, nnodes, stream: seen.append([nodes[i].t.dtype for i in range(nargs)]))
status = s.call(x, torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.bool))
assert status == S.MISS_HANDLED and seen == [[S.BF16, S.I32, S.U8]], (status, seen)
if hasattr(torch, "float8_e4m3fn"):  # a type that is there is taken still
    status = s.call(torch.zeros(4, dtype=torch.uint8).view(torch.float8_e4m3fn))
    assert status == S.MISS_HANDLED and seen[-1] == [S.E4M3], (status, seen)
try:
    s.call(torch.zeros(2, dtype=torch.complex64))
    raise SystemExit("an unknown type was taken")
except (TypeError, KeyError):
    pass
s.close()
print("fine", S.fastcall() is not None)
"""


@pytest.mark.parametrize("missing", [[], ["float8_e8m0fnu"], ["float8_e4m3fn", "float8_e8m0fnu"]])
def test_ops_without_8_bit_types_need_none(built_lib, missing):
    pytest.importorskip("torch")
    r = subprocess.run([sys.executable, "-c", CHILD.format(missing=missing)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.startswith("fine"), r.stderr[-2000:]
