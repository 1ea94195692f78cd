"""The binding on a torch without CUDA's private entry points: it imports, and takes the stream the public way."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
import types
import torch
for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
    if hasattr(torch._C, name):
        delattr(torch._C, name)
from paper_2512_15176_b200 import binding
torch.cuda.current_stream = lambda: types.SimpleNamespace(cuda_stream=4711)
assert binding._stream(None) == 4711
assert binding._stream(7) == 7
print("imported")
"""


def test_import_without_the_private_stream_calls():
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "imported" in r.stdout, r.stderr
