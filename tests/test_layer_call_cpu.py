"""The native calls of csrc/layer_call.cpp on tensors without storage, as torch.func's transforms hand them on: torch refuses their address, and
that has to reach the caller as an exception, whether or not the interpreter's lock has been given back by then."""
import os
import subprocess
import sys

import pytest

from paper_2603_24517_amd import build as B

HERE = os.path.dirname(os.path.abspath(__file__))

# (a process of its own: the module answers for the runtime, and a mistake here ends the process)
PROGRAM = """
import ctypes, importlib.util, sys
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

spec = importlib.util.spec_from_file_location("_layer_call", sys.argv[1])
module = importlib.util.module_from_spec(spec)
spec.loader.exec_module(module)
calls = []
C = ctypes.CFUNCTYPE
entries = [C(ctypes.c_int)(lambda: calls.append("entry") or 0), C(ctypes.c_longlong)(lambda: 0)]
order = [entries[0], entries[1], entries[0], entries[0], entries[1]]
module.bind(*(ctypes.cast(f, ctypes.c_void_p).value for f in order))

with FakeTensorMode() as mode:
    do, q, k, v, o = (torch.empty(1, 4, 2, 128, device="cuda", dtype=torch.bfloat16) for _ in range(5))
    lse, cos, w = torch.empty(1, 2, 4, device="cuda"), torch.empty(4, 64, device="cuda"), torch.empty(128, device="cuda")
do, q, k, v, o, lse, cos, w = (torch._to_functional_tensor(t) for t in (do, q, k, v, o, lse, cos, w))
results = {}


def backward(x):
    assert type(x) is torch.Tensor
    with mode:          # (results of the call: fake tensors, as there is no device)
        results["backward"] = module.backward(do, x, k, v, o, lse, False, None, None)
    return x.float().sum()


def rope(x):
    with mode:
        results["rope"] = module.rope(x, k, w, w, cos, cos, None, 1e-6, False, None, None)
        results["rope_backward"] = module.rope_backward(x, k, q, k, w, w, cos, cos, None, 1e-6, False, None, None)
    return x.float().sum()


for f in (backward, rope):
    try:
        torch.func.grad(f)(q)
    except Exception as e:      # (what torch makes of the number behind the call does not matter here)
        print(type(e).__name__, str(e)[:100])
assert results == dict.fromkeys(("backward", "rope", "rope_backward")), results      # left to the general form
assert calls == []
print("done")
"""


@pytest.fixture(scope="module")
def native(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("layer_call") / "_layer_call.so")
    cmd = B.call_command(os.path.join(HERE, "layer_call_shim.cpp"), so)
    subprocess.run(cmd + ["-Wl,-Bsymbolic"], check=True)
    return so


def test_address_that_torch_refuses_leaves_the_call_to_the_general_form(native):
    run = subprocess.run([sys.executable, "-c", PROGRAM, native], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and run.stdout.endswith("done\n"), (run.returncode, run.stdout, run.stderr[-2000:])
