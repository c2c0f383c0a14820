"""Tensors that say they are on a GPU, over host memory, in a process whose CUDA runtime says that cuda:0 is current (two
functions in front of the runtime's): what the binding does with its arguments shows on a machine without a GPU.  Nothing
can be launched or allocated there: a call that gets past the checks ends with torch's or the library's error."""
import os
import subprocess
import sys

from fake_runtime import ensure_built

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PRELUDE = """
import ctypes, torch
import paper_2603_04359_gb300 as cat

cat._raw_device = lambda: 0                   # (torch's own wants a driver first)
kept = []

def on(device, dtype, *shape, stride=None):
    if stride is None:
        stride = [1] * len(shape)
        for i in range(len(shape) - 2, -1, -1):
            stride[i] = stride[i + 1] * shape[i + 1]
    n = (1 + sum((a - 1) * b for a, b in zip(shape, stride)) if all(shape) else 0) * dtype.itemsize
    kept.append((ctypes.c_char * (max(n, 16) + 64))())
    at = -(-ctypes.addressof(kept[-1]) // 64) * 64
    s = torch._C._construct_storage_from_data_pointer(at, torch.device("cuda", device), n)
    return torch._C._construct_CUDA_Tensor_From_Storage_And_Metadata(
        dict(size=shape, stride=tuple(stride), dtype=dtype, storage_offset=0), s)

f, b, u, i, h, l = torch.float32, torch.bfloat16, torch.uint8, torch.int32, torch.float16, torch.int64

def outcome(call):
    try:
        r = call()
    except BaseException as e:
        return type(e).__name__ + " | " + str(e).splitlines()[0]
    return "returned | " + ("None" if r is None else type(r).__name__)
"""


def run(script, folder):
    """The script's lines, split at '|'."""
    ensure_built()
    lib, source = os.path.join(str(folder), "current.so"), os.path.join(str(folder), "current.c")
    with open(source, "w") as f:
        f.write("int cudaGetDevice(int* d) { *d = 0; return 0; }\nint cudaGetDeviceCount(int* n) { *n = 0; return 0; }\n")
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", lib, source], check=True)
    p = subprocess.run([sys.executable, "-c", PRELUDE + script], cwd=ROOT, capture_output=True, text=True,
                       env=dict(os.environ, LD_PRELOAD=lib, CUDA_VISIBLE_DEVICES=""))
    assert p.returncode == 0, p.stdout[-2000:] + p.stderr[-2000:]
    return [[part.strip() for part in line.split("|")] for line in p.stdout.splitlines()]
