"""Prompt calls of several host threads, without a GPU: what the extension holds while the interpreter is unlocked, and in which order launches are made."""
import ctypes as C
import importlib.machinery
import importlib.util
import os
import shutil
import subprocess
import weakref

import numpy as np
import pytest

from paper_2608_23599_b200 import binding as B
from paper_2608_23599_b200 import build as _build


class Rows:
    """What the extension asks of a tensor."""
    dtype = "bf16"

    def __init__(self, *shape):
        self.shape = shape

    def get_device(self):
        return 0

    def stride(self):
        return tuple(int(np.prod(self.shape[i + 1:])) for i in range(len(self.shape)))

    def data_ptr(self):
        return 1 << 20


@pytest.fixture
def extension(tmp_path):
    """A second copy of the extension, to be bound to fakes."""
    B.load()
    path = shutil.copy(_build.CALL_LIB, tmp_path)
    spec = importlib.util.spec_from_file_location("_gkv_call", path, loader=importlib.machinery.ExtensionFileLoader("_gkv_call", path))
    return importlib.util.module_from_spec(spec)


def test_a_streams_workspace_is_held_until_the_launches_are_made(extension):
    """Another thread replaces the stream's workspace while this one is inside the library."""
    class Memory:
        pass

    spaces, seen = {}, []
    memory = Memory()
    alive = weakref.ref(memory)
    spaces[64 * 0x77] = (1 << 24, 4096, memory)
    del memory

    def bytes_needed(_, need):
        need[0] = 4096
        return 0

    def attn(d, q, k, v, out, lse, ws, n, st):
        spaces.clear()
        seen.append((ws, n, alive() is not None))
        return 0

    vp = C.c_void_p
    fakes = [C.CFUNCTYPE(C.c_int, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp)(attn), C.CFUNCTYPE(C.c_int, vp, C.POINTER(C.c_size_t))(bytes_needed)]
    a, b = (C.cast(f, vp).value for f in fakes)
    extension.bind_rows(a, b, 0, 0, Rows, Rows.dtype, "f32", lambda: 0, lambda d: 0x77, lambda: False)
    q, k, off = Rows(5, 8, 128), Rows(5, 2, 128), np.array([0, 5], dtype=np.int32)
    assert extension.prompt_attn(q, k, k, q, off, None, 0.0, spaces) == 0
    assert seen == [(1 << 24, 4096, True)]
    assert alive() is None                           # (and given back behind them)


FAKE = r"""
#include <chrono>
#include <cstdio>
#include <cstring>
#include <mutex>
#include <thread>
#include <vector>
#include "../../include/gkv.h"
#include <cuda.h>
#include "gkv_internal.h"

namespace gkv {
extern bool (*make_map)(CUtensorMap*, const void*, int, const uint64_t*, const uint64_t*, const uint32_t*);
}

static std::mutex mu;
static std::vector<int> order;                                   // threads in the order of their launches
static thread_local int me = 0;

extern "C" {
cudaError_t cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t*, const void*, void**) {
  {
    std::lock_guard<std::mutex> lock(mu);
    order.push_back(me);
  }
  std::this_thread::sleep_for(std::chrono::milliseconds(30));    // (long enough for the other thread's)
  return cudaSuccess;
}
cudaError_t cudaLaunchKernel(const void*, dim3, dim3, void**, size_t, cudaStream_t) { return cudaErrorInvalidValue; }
unsigned __cudaPushCallConfiguration(dim3, dim3, size_t, cudaStream_t) { return 1; }
cudaError_t __cudaPopCallConfiguration(dim3*, dim3*, size_t*, void*) { return cudaErrorInvalidValue; }
void** __cudaRegisterFatBinary(void*) { static void* h; return &h; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
void __cudaRegisterFunction(void**, const char*, char*, const char*, int, uint3*, uint3*, dim3*, dim3*, int*) {}
}

int main() {
  gkv::on_current_device = [](std::initializer_list<const void*>) { return true; };
  gkv::make_map = [](CUtensorMap*, const void*, int, const uint64_t*, const uint64_t*, const uint32_t*) { return true; };
  const int32_t offsets[2] = {0, 2500};
  gkv_prompt d{};
  d.struct_size = sizeof(d);
  d.abi_version = GKV_ABI_VERSION;
  d.n_seqs = 1;
  d.n_q_heads = 8;
  d.n_kv_heads = 2;
  d.head_dim = 128;
  d.offsets = offsets;
  size_t need = 0;
  int bad = gkv_prompt_workspace_bytes(&d, &need) != GKV_OK || need == 0;
  char* const rows = reinterpret_cast<char*>(1 << 20);
  auto call = [&](int id, char* workspace) {
    me = id;
    for (int i = 0; i < 3; ++i) bad += gkv_prompt_attn(&d, rows, rows, rows, rows, nullptr, workspace, need, nullptr) != GKV_OK;
  };
  std::thread a([&] { call(1, rows); }), b([&] { call(2, rows); });
  a.join();
  b.join();
  for (int id : order) std::printf("%d", id);
  std::printf("\n");
  if (order.size() != 12) ++bad;
  for (size_t i = 0; i + 1 < order.size(); i += 2) bad += order[i] != order[i + 1];      // a call's parts are merged before the next call's are made
  return bad != 0;
}
"""


def test_the_launches_of_calls_that_share_a_workspace_do_not_mix(tmp_path):
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    if not os.path.exists(os.path.join(cuda, "bin", "nvcc")) or not shutil.which("g++"):
        pytest.skip("no compiler")
    src, obj, exe = tmp_path / "fake.cpp", tmp_path / "gkv_prompt.o", tmp_path / "fake"
    src.write_text(FAKE)
    subprocess.run([os.path.join(cuda, "bin", "nvcc"), *_build.NVCC_FLAGS, "-c", os.path.join(_build.CSRC, "gkv_prompt.cu"), "-o", str(obj)],
                   check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    subprocess.run(["g++", "-std=c++17", "-I", _build.CSRC, "-I", os.path.join(cuda, "include"), str(src), str(obj), "-o", str(exe), "-lpthread"], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr
