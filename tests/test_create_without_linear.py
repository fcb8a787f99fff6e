"""A context is created although the linear gradient's kernels cannot be made ready: only the calls that need them fail.  Host
code alone, on a fake of the CUDA runtime calls that it makes; no GPU."""
import os
import subprocess

from paper_2010_16248_b200 import build

FAKES = r"""
#include <cuda_runtime_api.h>

#include <cstring>

// The runtime's calls of acc_create: device memory is host memory, and every kernel was compiled with 32 registers.
int memory_calls = 0, asked = 0;
extern "C" {
cudaError_t cudaMemcpy(void* to, const void* from, size_t bytes, cudaMemcpyKind) {
  ++memory_calls;
  memcpy(to, from, bytes);
  return cudaSuccess;
}
cudaError_t cudaMemset(void* to, int value, size_t bytes) {
  ++memory_calls;
  memset(to, value, bytes);
  return cudaSuccess;
}
cudaError_t cudaMemsetAsync(void* to, int value, size_t bytes, cudaStream_t) { return cudaMemset(to, value, bytes); }
cudaError_t cudaGetDevice(int* device) { *device = 0; return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* value, cudaDeviceAttr, int) { *value = 148; return cudaSuccess; }
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaFuncGetAttributes(cudaFuncAttributes* a, const void*) {
  ++asked;
  memset(a, 0, sizeof *a);
  a->numRegs = 32;
  return cudaSuccess;
}
cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }
}
"""

PROGRAM = r"""
#include "acc_api.cu"
#include "acc_linear.cu"

#include <cstdlib>

extern int memory_calls, asked;
namespace acc {
cudaError_t prepare_powersgd() { return cudaSuccess; }
cudaError_t prepare_topk(acc_ctx*) { return cudaSuccess; }
cudaError_t prepare_adamw(acc_ctx*) { return cudaSuccess; }
}

int main() {
  acc_layer_desc layer{};
  layer.offset = 0;
  layer.rows = 2600;
  layer.cols = 650;
  layer.kind = ACC_MATRIX;
  acc_config cfg{};
  cfg.n_workers = 1;
  cfg.n_layers = 1;
  cfg.layers = &layer;
  cfg.worker_stride = 2600 * 650;
  cfg.rank_low = 2;
  cfg.rank_high = 1;
  cfg.topk_low_bp = 1000;
  cfg.topk_high_bp = 100;
  cfg.eta = 0.5f;
  cfg.gs_eps = 1e-8f;
  size_t bytes = 0;
  if (acc_workspace_bytes(&cfg, &bytes) != ACC_OK) return 10;
  acc_ctx* ctx = nullptr;
  void* ws = std::aligned_alloc(256, (bytes + 255) / 256 * 256);
  const int status = acc_create(&cfg, ws, bytes, &ctx);
  std::printf("acc_create %d, kernels asked about %d\n", status, asked);
  if (status != ACC_OK || !ctx || memory_calls == 0) return 1;
  // the call that needs them says so, before it starts anything
  const long long n = 700;
  size_t need = 0;
  if (acc_linear_grad_workspace_bytes(ctx, 0, n, &need) != ACC_OK) return 11;
  float* grads = static_cast<float*>(std::aligned_alloc(256, sizeof(float) * 2600 * 650));
  void* scratch = std::aligned_alloc(256, (need + 255) / 256 * 256);
  uint8_t* code = static_cast<uint8_t*>(std::aligned_alloc(256, n * 672));
  const int grad = acc_linear_grad(ctx, 0, grads, ACC_BF16, n, 2600, 2600 * n, 1.f, code, code, grads, 0, scratch, need, nullptr);
  std::printf("acc_linear_grad %d, launches %d\n", grad, acc_last_launch_count(ctx));
  if (grad != ACC_ECUDA || acc_last_launch_count(ctx) != 0 || asked == 0) return 2;
  // no tokens need no kernel
  grads[5] = 1.f;
  if (acc_linear_grad(ctx, 0, nullptr, ACC_BF16, 0, 2600, 2600, 1.f, nullptr, nullptr, grads, 0, scratch, need, nullptr) != ACC_OK) return 3;
  return grads[5] == 0.f ? 0 : 4;
}
"""


def test_create_without_the_linear_kernels(tmp_path):
    source, fakes, binary = tmp_path / "create.cu", tmp_path / "fakes.cpp", tmp_path / "create"
    source.write_text(PROGRAM)
    fakes.write_text(FAKES)
    # (device code is not run: PTX will do; the launches of the other files are never reached)
    subprocess.run([build._nvcc(), "-gencode", "arch=compute_100a,code=compute_100a", "-std=c++17", "-O1", "-cudart", "shared", "-I",
                    os.path.join(build.ROOT, "include"), "-I", build.CSRC, str(source), str(fakes), "-Xlinker", "--unresolved-symbols=ignore-all",
                    "-o", str(binary)], check=True, capture_output=True, text=True)
    libs = os.path.join(os.path.dirname(os.path.dirname(build._nvcc())), "lib64")
    env = {**os.environ, "LD_LIBRARY_PATH": libs + ":" + os.environ.get("LD_LIBRARY_PATH", "")}
    done = subprocess.run([str(binary)], capture_output=True, text=True, timeout=120, env=env)
    assert done.returncode == 0, (done.returncode, done.stdout, done.stderr)
