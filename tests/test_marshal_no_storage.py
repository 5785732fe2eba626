"""A tensor without memory of its own (as function transforms hand to what they call) is left to the checks in Python, which raise:
in a process of its own, for the native checks once went on without the interpreter's lock there."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r'''
import ctypes
import torch
import paper_2407_11550_amd as adakv
from paper_2407_11550_amd import binding
from torch._C._functorch import _grad_decrement_nesting, _grad_increment_nesting, _wrap_for_grad

BF = torch.bfloat16
memory = ctypes.create_string_buffer(1 << 20)


def device(*shape):                              # says that it is on the GPU; nobody looks at its memory here
    st = torch._C._construct_storage_from_data_pointer(ctypes.addressof(memory), torch.device("cuda:0"), 1 << 20)
    stride = [1]
    for n in reversed(shape[1:]):
        stride.insert(0, stride[0] * n)
    return torch._C._construct_CUDA_Tensor_From_Storage_And_Metadata(
        dict(size=shape, stride=stride, dtype=BF, storage_offset=0, device=torch.device("cuda:0")), st)


layer = adakv.Layer(BF, 8, 2, 64, 4, 3, 0.2, [128], [40])
K, V, q, out = device(132, 2, 64), device(132, 2, 64), device(132, 8, 64), device(132, 8, 64)
calls = []
P, I, L = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
fn = ctypes.CFUNCTYPE(ctypes.c_int, P, P, L, L, P, P, I, I, P, P, P)(lambda *given: calls.append(given) or 0)


def native(q, K, V, out):
    return binding._marshal.window_attn(0, ctypes.cast(fn, P).value, layer._address, 132, False, False, q, K, V, 9, 1, out, None, 7)


assert native(q, K, V, out) == 0 and len(calls) == 1
assert calls[0][1:4] == (q.data_ptr(), 8 * 64, 64) and calls[0][6:8] == (9, 1)
level = _grad_increment_nesting()
for i in range(4):
    a = [q, K, V, out]
    a[i] = _wrap_for_grad(a[i], level)
    assert type(a[i]) is torch.Tensor and a[i].is_cuda
    assert native(*a) is None, i
_grad_decrement_nesting()
assert len(calls) == 1
print("left to Python")
'''


def test_a_tensor_without_memory_is_left_to_python(lib):
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "left to Python" in r.stdout, (r.returncode, r.stdout, r.stderr)
