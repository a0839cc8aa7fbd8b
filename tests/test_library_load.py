"""The binding loads and refuses bad arguments on a torch without GPU support (no GPU needed)."""
import os
import subprocess
import sys

import pytest

import paper_2604_09603_amd as pkg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

WITHOUT = """
import torch
if hasattr(torch._C, "_cuda_getCurrentRawStream"):
    del torch._C._cuda_getCurrentRawStream
import paper_2604_09603_amd as pkg
lib = pkg.load()
assert lib.echo_store_kv_q8(*[None] * 2, 0, 0, None, -1, 1, 128, 0, *[None] * 4, 1, 32, None, None) == pkg.ERR_INVALID_ARG
assert pkg.tree_verify_attn_paged_q8_workspace_size(0, 1, 8, 8, 1) == 0
class Stream:
    cuda_stream = 7
assert pkg._stream(Stream()) == 7
class Cuda:  # what torch offers without the raw handle
    current_stream = staticmethod(lambda: Stream())
torch.cuda.current_stream = Cuda.current_stream
assert pkg._stream(None) == 7
print("loaded")
"""


def test_load_without_the_raw_stream_handle():
    if not os.path.exists(pkg.LIB_PATH):
        pytest.skip("libecho.so not built")
    run = subprocess.run([sys.executable, "-c", WITHOUT], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip() == "loaded", run.stderr[-2000:]
