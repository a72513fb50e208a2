"""The AdamW step's table and roots, apart from the step itself."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2408_06995_b200 as fpq
from paper_2408_06995_b200 import build as fpq_build

F32, BF = torch.float32, torch.bfloat16


class Memory:
    """Stands in for a tensor on the GPU: the table looks at a tensor's place and type alone."""
    is_cuda = True

    def __init__(self, at, n, dtype=F32):
        self.at, self.n, self.dtype = at, n, dtype

    def data_ptr(self):
        return self.at

    def numel(self):
        return self.n

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True


def memory_table(codes=False, **changed):
    """Two tensors of 64 and 40 elements, every buffer directly behind another; {name: tensor 0's or 1's} are put elsewhere."""
    at, given = 1 << 20, {}
    state = torch.uint8 if codes else F32
    for name, dtype, unit in (("params", F32, 1), ("grads", BF, 1), ("m", state, 1), ("v", state, 1), ("m_scale", torch.uint8, 32), ("v_scale", torch.uint8, 32),
                              ("copies", BF, 1)):
        given[name] = []
        for n in (64, 40):
            given[name].append(Memory(at, -(-n // unit), dtype))
            at += given[name][-1].numel() * dtype.itemsize
    for name, (i, place) in changed.items():
        given[name][i] = Memory(place(given), given[name][i].n, given[name][i].dtype)
    if not codes:
        given["m_scale"] = given["v_scale"] = None
    return fpq.fpq_adamw_table(**given)


@pytest.mark.parametrize("codes", [False, True])
def test_the_table_takes_buffers_side_by_side(codes):
    memory_table(codes)
    memory_table(codes, grads=(1, lambda t: t["grads"][0].at))         # gradients are only read: two may be one
    memory_table(codes, grads=(1, lambda t: t["grads"][0].at + 2))


@pytest.mark.parametrize("codes,changed", [
    (False, {"grads": (0, lambda t: t["copies"][0].at)}), (False, {"grads": (1, lambda t: t["copies"][0].at + 100)}), (True, {"grads": (0, lambda t: t["copies"][1].at - 126)}),
    (False, {"grads": (0, lambda t: t["params"][0].at)}), (True, {"grads": (1, lambda t: t["params"][1].at + 158)}), (False, {"grads": (1, lambda t: t["v"][0].at + 16)}),
    (True, {"grads": (1, lambda t: t["v_scale"][0].at)}), (False, {"params": (1, lambda t: t["params"][0].at + 252)}), (False, {"m": (0, lambda t: t["m"][1].at - 252)}),
    (False, {"copies": (1, lambda t: t["params"][0].at + 4)}), (True, {"m": (0, lambda t: t["v"][0].at + 8)}), (True, {"m_scale": (0, lambda t: t["v_scale"][0].at + 1)}),
    (True, {"m_scale": (1, lambda t: t["m"][0].at + 63)}), (False, {"params": (1, lambda t: t["params"][0].at)})])
def test_the_table_refuses_memory_in_two_roles(codes, changed):
    with pytest.raises(AssertionError, match="overlap|twice"):
        memory_table(codes, **changed)


ROOTS = r"""#include <stdint.h>

#include "fpq_roots.cuh"

// Counts the numbers of [first, last) (as bits) whose roots are not those rounded to nearest, and keeps the smallest of them.
__global__ void compare(uint32_t first, uint32_t last, unsigned long long* wrong, unsigned* smallest)
{
    for (uint64_t i = first + 2ull * (blockIdx.x * blockDim.x + threadIdx.x); i < last; i += 2ull * gridDim.x * blockDim.x) {
        const float2 v = make_float2(__uint_as_float((uint32_t)i), __uint_as_float(i + 1 < last ? (uint32_t)i + 1 : first));
        const float2 r = fpq::roots_of(v);
        if (__float_as_uint(r.x) != __float_as_uint(__fsqrt_rn(v.x)) || __float_as_uint(r.y) != __float_as_uint(__fsqrt_rn(v.y))) {
            atomicAdd(wrong, 1ull);
            atomicMin(smallest, (unsigned)i);
        }
    }
}

extern "C" int roots(uint32_t first, uint32_t last, unsigned long long* wrong, unsigned* smallest, void* stream)
{
    compare<<<148 * 8, 256, 0, (cudaStream_t)stream>>>(first, last, wrong, smallest);
    return (int)cudaGetLastError();
}
"""


@pytest.mark.gpu
def test_roots_are_rounded_to_nearest(tmp_path):
    """Every FP32 number from 2^-96 to the largest, and zero: what the step uses without a branch."""
    (tmp_path / "roots.cu").write_text(ROOTS)
    so = tmp_path / "roots.so"
    subprocess.run([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-shared",
                    "-Xcompiler", "-fPIC", "-cudart", "static", "-I", fpq_build.CSRC, str(tmp_path / "roots.cu"), "-o", str(so)], check=True)
    f = ctypes.CDLL(str(so)).roots
    f.argtypes = [ctypes.c_uint32, ctypes.c_uint32] + [ctypes.c_void_p] * 3
    for first, last in ((0, 1), ((127 - 96) << 23, 0x7F800000)):
        wrong, smallest = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.full((1,), 0x7FFFFFFF, dtype=torch.int32, device="cuda")
        assert f(first, last, wrong.data_ptr(), smallest.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
        assert int(wrong) == 0, f"{int(wrong)} wrong, from bits {int(smallest):#x} on"
