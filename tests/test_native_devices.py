"""Each tensor of the calls of 8-bit pages, weights and eviction has to lie on the context's device.  Tensors that say they are on a device but have no
memory stand for the GPUs' (no device is needed for one); a call that looks at their memory instead of refusing them raises another error.  In a process
of its own, so that a crash is a failure and not the end of the run."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SCRIPT = """
import sys
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
from paper_2608_19662_b200 import binding

binding.load_library()
I, F, B, H, E = torch.int32, torch.float32, torch.uint8, torch.bfloat16, torch.float8_e4m3fn


class Context:
    _shape, _ws = (8, 2, 128, 64, 0), None


POOL, TABLE, ITEMS = ((9, 64, 128), H), ((6, 3), I), ((6,), I)
Q8 = [((4, 64, 128), E)] * 2 + [((4,), F)] * 2
NEW = [((3, 2, 128), H)] * 2
CALLS = {
    "compact_q8": [((2, 50, 128), H)] * 2 + [((50,), B), ((2,), I), ((1,), I), ((1,), I), ((2, 1), B), ((3,), I), ((60,), I)] + Q8 + [((2, 2), I), ((4,), I), ((2,), I), ((1 << 16,), B)],
    "decode_q8": [((3, 8, 128), H), ((3,), I)] + Q8 + [TABLE, ITEMS, POOL, POOL, TABLE, ITEMS] + NEW + [((9, 64), F)] * 2 + [((3, 8, 128), H), None, ((1 << 24,), B)],
    "decode_weighted": [((3, 8, 128), H), ((3,), I), POOL, POOL, TABLE, ITEMS, TABLE, ITEMS] + [((9, 64), F)] * 2 + NEW + [((3, 8, 128), H), None, ((1 << 24,), B)],
    "evict": [POOL, POOL, ((9, 64), F), TABLE, ITEMS, 70, 3, ((4,), I), ((6, 2), I), ITEMS, ((6, 70), I)],
}
call = sys.argv[1]
with FakeTensorMode():
    def made(x, device):
        return torch.empty(x[0], dtype=x[1], device=device) if isinstance(x, tuple) else x

    for other in [None] + [i for i, x in enumerate(CALLS[call]) if isinstance(x, tuple)]:
        args = [made(x, "cuda:1" if i == other else "cuda:0") for i, x in enumerate(CALLS[call])]
        try:
            getattr(binding._native, call)(Context(), None, binding.BF16, *args)
        except Exception as e:
            print(other, "here" if "another device" in str(e) else "memory" if isinstance(e, RuntimeError) else repr(e))
"""
TENSORS = {"compact_q8": 17, "decode_q8": 18, "decode_weighted": 14, "evict": 9}


@pytest.mark.parametrize("call", sorted(TENSORS))
def test_a_tensor_on_another_device_is_refused(call):
    run = subprocess.run([sys.executable, "-c", SCRIPT, call], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr[-2000:]
    lines = run.stdout.splitlines()
    assert len(lines) == TENSORS[call] + 1 and lines[0] == "None memory", lines
    assert all(line.endswith(" here") for line in lines[1:]), lines
