"""What the native binding of the paged calls makes of the library's status: a call that was refused before anything was
enqueued goes back to paged.py's own checks, any other failure is raised at once and the call not made again (a copy that failed
behind the tables' rewrite would find nothing left to copy).

Without the binding's library the same calls go through paged.py alone.

In processes of their own, without a GPU: tensors of one aligned block of host memory that claim to be on device 0, and a
library whose calls only count themselves and give the status that they are told to."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CALLS = ["sd2_paged_append", "sd2_paged_append_scaled", "sd2_paged_attn_window", "sd2_paged_attn_scaled", "sd2_pages_fork",
         "sd2_pages_slide", "sd2_pages_reserve"]
STUB = ("#include <stddef.h>\nint calls, status;\n" + "".join(f"int {c}() {{ calls++; return status; }}\n" for c in CALLS)
        + "".join(f"size_t {c}_workspace_bytes() {{ return 256; }}\n" for c in CALLS if "attn" in c))

SETUP = r'''
import ctypes, sys
stub = ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL)  # its symbols come before those of libsd2.so
import torch
from paper_2511_09844_amd import binding as B
from paper_2511_09844_amd import paged

calls, status = (ctypes.c_int.in_dll(stub, x) for x in ("calls", "status"))
block = ctypes.create_string_buffer(1 << 20)
at = (ctypes.addressof(block) + 255) // 256 * 256
device = torch.device("cuda", 0)


def claimed(shape, dtype):
    strides = [1]
    for n in reversed(shape[1:]):
        strides.insert(0, strides[0] * max(n, 1))
    storage = torch._C._construct_storage_from_data_pointer(at, device, strides[0] * max(shape[0], 1) * dtype.itemsize)
    return torch._C._construct_CUDA_Tensor_From_Storage_And_Metadata(
        dict(dtype=dtype, device=device, size=tuple(shape), stride=tuple(strides), storage_offset=0), storage)


lib = torch.library.Library("aten", "IMPL")
lib.impl("empty.memory_format", lambda size, dtype=None, layout=None, device=None, pin_memory=None, memory_format=None: claimed(size, dtype), "CUDA")

torch.empty_like = lambda t, **kw: claimed(tuple(t.shape), t.dtype)
torch.cuda._lazy_init, torch.cuda.current_device = (lambda: None), (lambda: 0)
paged._device, paged._stream_of = (lambda: 0), (lambda i: 0)
i32 = torch.int32


def cache_of(held):
    pool = (4, 1, 2, 16, 32)
    scales = claimed((4, 1, 2, 1, 2), torch.float8_e8m0fnu) if held == paged.HELD8 else None
    return paged.PagedCache(claimed(pool, held), claimed(pool, held), claimed((3, 4), i32), claimed((4,), i32), scales)


q, kv, lens = claimed((3, 2, 32), torch.float32), claimed((3, 2, 32), torch.float32), claimed((3,), i32)
at += 1 << 16
out = claimed((3, 2, 32), torch.float32)
ways = {
    "append": ("sd2_paged_append", lambda c: c.append(kv, kv, lens)),
    "attend": ("sd2_paged_attn", lambda c: c.attend(q, lens)),
    "attend into": ("sd2_paged_attn", lambda c: c.attend(q, lens, out=out, window=5)),
    "fork": ("sd2_pages_fork", lambda c: c.fork([0], [1])),
    "slide": ("sd2_pages_slide", lambda c: c.slide(lens, 5)),
    "reserve": ("sd2_pages_reserve", lambda c: c.reserve(lens, lens)),
}
'''

STATUS = r'''
CALLS = sys.argv[2].split(",")
caches = {}
for held in (torch.float32, torch.float8_e4m3fn):
    caches[held] = c = cache_of(held)

    class Again:  # paged.py's own way to the library
        def __init__(self, lib):
            self.real = lib

        def __getattr__(self, name):
            return again if name in CALLS + ["sd2_paged_attn"] else getattr(self.real, name)

    def again(*args):
        raise AssertionError("called again")
    c.lib = Again(c.lib)
for held, c in caches.items():
    for name, (what, call) in ways.items():
        calls.value, status.value = 0, 0
        call(c)
        assert calls.value == 1, (held, name)
        for failed in (-4, -5, -2):
            calls.value, status.value = 0, failed
            try:
                call(c)
                raise SystemExit(f"{held} {name}: status {failed} was not raised")
            except B.Sd2Error as e:
                assert what in str(e) and f"({failed})" in str(e), e
            assert calls.value == 1, (held, name)
        # refused: paged.py's own way follows
        calls.value, status.value = 0, -1
        try:
            call(c)
            raise SystemExit(f"{held} {name}: a refused call did not go on to the checks")
        except AssertionError as e:
            assert str(e) == "called again", e
        assert calls.value == 1
print("every status")
'''


MISSING = r'''
import warnings
B.TORCH_SO = sys.argv[1] + ".missing"
for held in (torch.float32, torch.float8_e4m3fn):
    with warnings.catch_warnings(record=True) as told:
        warnings.simplefilter("always")
        c = cache_of(held)
    assert [w.category for w in told] == [RuntimeWarning] and "not built" in str(told[0].message), told
    for name, (what, call) in ways.items():
        try:  # as far as the library, which finds no device
            call(c)
            raise SystemExit(f"{held} {name}: no call")
        except B.Sd2Error as e:
            assert what in str(e), e
print("every call")
'''


def run(program, tmp_path):
    from paper_2511_09844_amd import binding
    binding.load_torch_paged()
    stub = tmp_path / "libstub.so"
    (tmp_path / "stub.c").write_text(STUB)
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-o", str(stub), str(tmp_path / "stub.c")])
    res = subprocess.run([sys.executable, "-c", SETUP + program, str(stub), ",".join(CALLS)], capture_output=True, text=True,
                         env=dict(os.environ, PYTHONPATH=ROOT, HIP_VISIBLE_DEVICES=""), timeout=300)
    assert res.returncode == 0, res.stdout[-2000:] + res.stderr[-4000:]
    return res.stdout


def test_a_failed_call_is_raised_and_not_made_again(tmp_path):
    assert "every status" in run(STATUS, tmp_path)


def test_without_the_binding_calls_go_the_long_way(tmp_path):
    assert "every call" in run(MISSING, tmp_path)
