"""What the paged 4-bit cache's entry points say and the binding needs without a GPU."""
import ctypes
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def kv4():
    from paper_2502_01941_amd import build, kv4, shotkv
    if not os.path.exists(shotkv.LIB_PATH):
        build.build(force=True)
    kv4.load_library()
    return kv4


def workspace(kv4, heads, kv_heads, requests, tokens, most, page=64, max_pages=16):
    cfg = kv4._heads(heads, kv_heads, 128, torch.bfloat16)
    return kv4.load_library().shotkv_kv4_attention_workspace_bytes(ctypes.byref(cfg), requests, tokens, most, page, max_pages)


@pytest.mark.parametrize("heads,kv_heads", [(64, 8), (32, 8), (8, 1), (4, 4)])
def test_limits_of_the_header(kv4, heads, kv_heads):
    """2^29 rows of queries in a request, 2^28 tokens in a batch, 65535 requests, 2^30 tokens in a row of the table."""
    most = min(2**29 // heads, 2**28)
    assert workspace(kv4, heads, kv_heads, 1, most, most) > 0
    assert workspace(kv4, heads, kv_heads, 1, most, 2**28) > 0          # no more tokens than the batch has
    assert workspace(kv4, heads, kv_heads, 1, most + 1, most + 1) == 0
    assert workspace(kv4, heads, kv_heads, 2, 2**28, 2**28 // 64) > 0 and workspace(kv4, heads, kv_heads, 2, 2**28 + 1, 1) == 0
    assert workspace(kv4, heads, kv_heads, 65535, 65535, 1) > 0 and workspace(kv4, heads, kv_heads, 65536, 65536, 1) == 0
    assert workspace(kv4, heads, kv_heads, 1, 1, 1, 32, 2**25) > 0 and workspace(kv4, heads, kv_heads, 1, 1, 1, 32, 2**25 + 1) == 0


def test_the_binding_does_not_need_names_that_torch_keeps_to_itself():
    """A torch built without GPUs has no _cuda_* names: the module can be imported, and streams come from the public interface."""
    import subprocess
    import sys
    code = ("import sys, torch; sys.path.insert(0, %r)\n"
            "for name in [n for n in dir(torch._C) if n.startswith('_cuda_')]: delattr(torch._C, name)\n"
            "from paper_2502_01941_amd import kv4, shotkv\n"
            "class Stream: cuda_stream = 1234\n"
            "torch.cuda.current_stream = Stream\n"
            "assert kv4._stream() == shotkv._stream() == 1234\n") % ROOT
    out = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr
