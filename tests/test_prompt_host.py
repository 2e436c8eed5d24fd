"""Host side of the prompt's and the shared prefix's calls, without a GPU: what is refused before any CUDA call, and that a tensor
without storage raises in Python instead of ending the process."""
import ctypes
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
E_NULL = -1


@pytest.fixture(scope="module")
def lib():
    from paper_2509_15235_b200 import binding, build
    build.build()
    return binding.load()


def test_a_null_context_is_refused(lib):
    z = ctypes.c_void_p(0)
    n = ctypes.c_size_t()
    assert lib.vispec_rope_axes_rows(z, z, 0, z, 0, z, 0, None, z, 0, z, 0, z) == E_NULL
    assert lib.vispec_kv_append(z, 0, z, 0, z, 0, z, 0, z, None, z, z, 0, 0, z, 0, z, z) == E_NULL
    assert lib.vispec_kv_append_paged(z, 0, z, 0, z, 0, z, 0, z, None, z, z, z, 0, 0, 0, z, 0, z, z) == E_NULL
    assert lib.vispec_tree_verify_attn_prefix_paged(z, 0, z, z, z, 1, 0, z, 1, 1, 1.0, z, 0, z, z, z) == E_NULL
    assert lib.vispec_prefix_scratch_bytes(z, 1, 1, ctypes.byref(n)) == E_NULL


def test_rope_axes_holds_the_c_struct(lib):
    from paper_2509_15235_b200 import binding
    ax = binding.RopeAxes((16, 24, 24), 1e6, True)
    c = binding._RopeAxes.from_address(ax._addr)
    assert (c.n_axes, list(c.sections), c.interleaved, c.theta) == (3, [16, 24, 24, 0], 1, 1e6)
    assert ctypes.sizeof(binding._RopeAxes) == 28
    for bad in ((), (8,) * 5):
        with pytest.raises(ValueError):
            binding.RopeAxes(bad, 1e4)


@pytest.mark.parametrize("call", [
    "rope_axes_rows(0, 4, 2, 128, rows, None, pos, ax._addr, rows, None)",
    "kv_append(0, 2, 4, 128, 0, None, rows, rows, pos, ax._addr, ints, ints, None, None)",
    "kv_append_paged(0, 2, 4, 128, 0, None, rows, rows, pos, ax._addr, ints, ints, pos, None, None)",
    "tree_verify_attn_prefix_paged(0, 4, 2, 128, 0, tree, ints, pos, 0, ints, 1.0, ints, tree, None)",
])
def test_a_tensor_without_storage_raises_in_python(lib, call):
    code = f"""
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
from paper_2509_15235_b200 import binding
binding.load()
ax = binding.RopeAxes((64,), 1e4)
with FakeTensorMode():
    rows = torch.empty(1, 4, 128, device="cuda", dtype=torch.bfloat16)
    tree = torch.empty(1, 1, 4, 128, device="cuda", dtype=torch.bfloat16)
    pos = torch.empty(1, 1, device="cuda", dtype=torch.int32)
    ints = torch.empty(1, device="cuda", dtype=torch.int32)
try:
    binding._native.{call}
except (RuntimeError, ValueError) as e:
    print("raised", type(e).__name__)
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=ROOT, timeout=300)
    assert r.returncode == 0 and "raised" in r.stdout, (r.returncode, r.stderr[-500:])
