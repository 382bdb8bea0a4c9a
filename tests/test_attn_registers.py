"""Attention's warps exchange registers, which works with the number that the kernels are launched with and no other:
this compiler gives it, and a build where it does not refuses attention alone."""
import os
import re
import shutil
import subprocess
import sys

import pytest

from paper_2606_26472_gb300 import build as B

# A stand-in for the CUDA runtime that records launches: no GPU is needed, and none is used.
_RUNTIME = r"""
#include <cuda_runtime_api.h>
#include <stdlib.h>
#include <string.h>
int launches = 0;
cudaError_t cudaFuncGetAttributes(struct cudaFuncAttributes* a, const void* f) {
  memset(a, 0, sizeof(*a));
  a->numRegs = atoi(getenv("TEST_REGISTERS"));
  return cudaSuccess;
}
cudaError_t cudaFuncSetAttribute(const void* f, enum cudaFuncAttribute a, int v) { return cudaSuccess; }
cudaError_t cudaMemsetAsync(void* p, int v, size_t n, cudaStream_t s) { return cudaSuccess; }
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void* f, void** a) { ++launches; return cudaSuccess; }
cudaError_t cudaGetLastError(void) { return cudaSuccess; }
"""

_CALLS = r"""
import ctypes as C, sys
from paper_2606_26472_gb300 import epikv as E
count = C.c_int.in_dll(C.CDLL(sys.argv[1]), "launches")
P = 1 << 20                       # an address that nothing reads
cfg = E.make_attn_config(max_seqs=2, max_cache_tokens=64, max_new_tokens=2, num_layers=1, num_heads=4, num_kv_heads=2,
                         head_dim=128, cache_format=E.EPIKV_CACHE_E2M1)
units = 2 * 72
view = E.kv_view(P, P, layout=E.EPIKV_LAYOUT_CONTIGUOUS, stride_layer=0, stride_seq=64 * units, stride_token=units)
q, k = E.epikv_rows(P, 4 * 128, 128, E.EPIKV_TYPE_BF16), E.epikv_rows(P, 2 * 128, 128, E.EPIKV_TYPE_BF16)
rope = E.epikv_rope_view(P, 100, 128, E.EPIKV_ROPE_HALF)
ctx = E.epikv_attn_init(cfg, P, E.epikv_attn_workspace_bytes(cfg), stream=0)
E.epikv_rope(ctx, 2, 4, q, q, P, rope, stream=0)
E.epikv_append(ctx, 0, 1, P, P, 1, P, P, q, q, k, k, rope, view, stream=0)
E.epikv_cache_read(ctx, 0, 1, P, P, k, None, view, stream=0)
print(count.value, end=" ")
try:
    E.epikv_attention(ctx, 0, 1, P, P, 1, P, q, q, view, stream=0)
    print(count.value, "taken")
except E.EpikvError as e:
    print(count.value, "refused" if e.status == E.EPIKV_ECUDA else e.status)
"""


@pytest.fixture(scope="module")
def runtime(tmp_path_factory):
    B.build()
    include = os.path.join(os.path.dirname(B._cuda_lib_dir()), "include")
    out = str(tmp_path_factory.mktemp("runtime") / "runtime.so")
    r = subprocess.run([shutil.which("gcc") or "cc", "-shared", "-fPIC", "-I" + include, "-x", "c", "-", "-o", out],
                       input=_RUNTIME, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return out


@pytest.mark.parametrize("registers,said", [(168, "3 5 taken"), (160, "3 3 refused"), (128, "3 3 refused")])
def test_other_operators_do_not_depend_on_it(runtime, registers, said):
    r = subprocess.run([sys.executable, "-c", _CALLS, runtime], capture_output=True, text=True, cwd=B.ROOT,
                       env={**os.environ, "LD_PRELOAD": runtime, "TEST_REGISTERS": str(registers)})
    assert r.returncode == 0, r.stderr
    assert r.stdout.strip() == said


def test_this_compiler_gives_it(tmp_path):
    r = subprocess.run([B._nvcc(), *B.NVFLAGS, "-Xptxas", "-v", "-I" + B.INCLUDE, "-I" + B.CSRC, "-c",
                        os.path.join(B.CSRC, "attention.cu"), "-o", str(tmp_path / "attention.o")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    used = re.findall(r"entry function '(\w*attention_kernelILi(\d+)\w*)'.*?Used (\d+) registers", r.stdout + r.stderr, re.S)
    assert len(used) >= 10
    assert {(d, n) for _, d, n in used if d != "256"} == {("64", "168"), ("128", "168")}
