"""The tile kernels' loads from tensor memory: registers count as loaded behind a wait, so the wait names them. Where it does not,
nothing but the order of the statements keeps a use of them behind it, and a compiler may change that order."""
import os
import re

import pytest

from paper_2609_37241_gb300 import build


@pytest.mark.parametrize("name", ["attn_tile.cuh", "attn_tile.cu", "attn_tile8.cu"])
def test_every_load_is_waited_for_by_its_registers(name):
    text = open(os.path.join(build.CSRC, name)).read()
    calls = re.findall(r"(?<!void )\btc_(ld32|wait_ld)(?:<\w+>)?\(([^;]*)\);", text)
    assert calls
    open_loads = set()
    for what, args in calls:
        names = re.findall(r"\b[a-z]\w*", args.split(",")[-1])  # a load's last argument, the wait's only one
        if what == "ld32":
            open_loads.add(names[0])
        else:
            assert names and open_loads == {names[0]}, (name, args, open_loads)
            open_loads.clear()
    assert not open_loads
