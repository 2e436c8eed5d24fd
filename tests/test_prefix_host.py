"""What the shared-prefix attention and the prompt's calls promise that shows without a GPU: in their sources, and in what the binding refuses."""
import glob
import os
import re
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2509_15235_b200", "csrc")


def test_barriers_are_arrived_at_with_release():
    """The products that overwrite an accumulator start behind the arrivals of the threads that have read it: arrivals that order nothing
    (.relaxed) would leave that to the hardware."""
    sources = glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh"))
    assert sources
    for path in sources:
        assert not re.search(r"mbarrier\.arrive[.\w]*\.relaxed", open(path).read()), path


@pytest.fixture(scope="module")
def lib():
    from paper_2509_15235_b200 import binding, build
    build.build()
    return binding.load()


# every tensor of the type and shape that the call takes
CALLS = [
    "rope_axes_rows(0, 4, 2, 128, q, None, pos, ax._addr, q, None)",
    "rope_axes_rows(0, 4, 2, 128, None, k, pos, ax._addr, None, k)",
    "kv_append(0, 4, 2, 128, 0, q, k, k, pos, ax._addr, cu, kv, q, kv)",
    "kv_append_paged(0, 4, 2, 128, 0, q, k, k, pos, ax._addr, cu, kv, table, q, kv)",
    "tree_verify_attn_prefix_paged(0, 4, 2, 128, 0, tree, kv, table, 0, mask, 1.0, scratch, tree, lse)",
]


def test_tensors_without_storage_are_refused(lib):
    """A fake CUDA tensor has no memory: whichever the binding meets first it names, before anything asks for a device, and instead of
    passing on an address of zero (which an optional argument would take for "not given")."""
    code = f"""
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
from paper_2509_15235_b200 import binding
binding.load()
ax = binding.RopeAxes((64,), 1e4)
with FakeTensorMode():
    t = lambda *shape, dtype=torch.bfloat16: torch.empty(*shape, device="cuda", dtype=dtype)
    q, k, tree, pos = t(1, 4, 128), t(1, 2, 128), t(1, 1, 4, 128), t(1, 1, dtype=torch.int32)
    cu, kv, table = t(2, dtype=torch.int32), t(1, dtype=torch.int32), t(1, 8, dtype=torch.int32)
    mask, scratch, lse = t(1, 1, 1, dtype=torch.int64), t(64, dtype=torch.uint8), t(1, 4, 1, dtype=torch.float32)
for call in {CALLS!r}:
    try:
        eval("binding._native." + call)
        print("nothing raised", call)
    except RuntimeError as e:
        print("raised", str(e).splitlines()[0])
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=ROOT, timeout=300)
    said = r.stdout.splitlines()
    assert r.returncode == 0 and len(said) == len(CALLS), (r.returncode, r.stderr[-500:])
    assert all(s.startswith("raised") and "storage" in s for s in said), said


@pytest.mark.parametrize("call", ["tree_verify_attn_prefix_paged(0, 4, 2, 128, {}, None, None, None, 0, None, 1.0, None, None, None)",
                                  "kv_append(0, 4, 2, 128, {}, None, None, None, None, 0, None, None, None, None)",
                                  "rope_axes_rows(0, {}, 2, 128, None, None, None, 0, None, None)",
                                  "tree_verify_attn(0, {}, None, None, None, None, None, None, 1.0, None, None)"])
@pytest.mark.parametrize("value", [2 ** 31, 2 ** 32, 2 ** 63 - 1, 2 ** 64, -2 ** 31 - 1])
def test_integers_beyond_an_int_are_refused(lib, call, value):
    """2^32 is not layer 0."""
    from paper_2509_15235_b200 import binding
    with pytest.raises(OverflowError):
        eval("binding._native." + call.format(value))
