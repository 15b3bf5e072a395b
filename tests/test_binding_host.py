"""CPU-only tests of the Python binding itself."""
import subprocess
import sys

import torch

from paper_2512_12990_amd import binding as B


def test_loads_with_a_torch_without_gpu_support():
    """Such a torch lacks the symbols of the device runtime; the host-only calls have to work all the same, and the stream comes from the public call."""
    code = """
import torch
for name in [n for n in dir(torch._C) if n.startswith("_cuda_getCurrentRawStream")]:
    delattr(torch._C, name)
from paper_2512_12990_amd import binding as B
assert B.smoe_topn_slices(__import__("numpy").ones((1, 2), "uint32"), 3).tolist() == [0, 2, 1]
class S:
    cuda_stream = 1234
torch.cuda.current_stream = lambda device: S if device == 1 else None
assert B._stream_now(1) == 1234
print("fine")
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "fine", r.stderr


def test_tensors_of_a_call():
    """Every tensor that a call is given has to be found, whatever the pair of an Mx arrives in: it is kept from reuse while another stream works on it."""
    a, b, c, d, e = (torch.zeros(1) for _ in range(5))
    got = list(B._tensors((a, B.Mx(b, c), 3, None, [d, e], "x")))
    assert [id(t) for t in got] == [id(t) for t in (a, b, c, d, e)]
