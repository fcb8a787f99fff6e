"""Host side of the linear gradient's workspace query, without a GPU: a small program builds a context by hand and asks the library
from several threads at once."""
import os
import subprocess

import pytest

from paper_2010_16248_b200 import build

PROGRAM = r"""
#include <atomic>
#include <cstdio>
#include <thread>

#include "acc_internal.cuh"

// A checkpoint's rows have 2^30 columns at most, and so have the layers of a gradient from one.
static int columns() {
  static acc_ctx ctx;
  ctx.cfg.n_workers = ctx.cfg.n_layers = 1;
  ctx.plan.layers.emplace_back();
  acc::DevLayer& l = ctx.plan.layers[0];
  l.rows = 1; l.kind = ACC_MATRIX;
  size_t bytes = 0;
  l.cols = 1 << 30;
  if (acc_linear_grad_workspace_bytes(&ctx, 0, 1, &bytes) != ACC_OK || bytes < (2ull << 30)) return 3;
  l.cols = (1 << 30) + 1;
  if (acc_linear_grad_workspace_bytes(&ctx, 0, 1, &bytes) != ACC_EINVAL) return 4;
  alignas(256) static float here[64];  // (an address; the call is refused before anything is read)
  uint8_t* const code = reinterpret_cast<uint8_t*>(here);
  return acc_linear_grad(&ctx, 0, here, ACC_BF16, 1, 1, 1, 1.f, code, code, here, 0, here, ~(size_t)0, nullptr) == ACC_EINVAL ? 0 : 5;
}

int main(int argc, char**) {
  if (argc > 1) return columns();
  static acc_ctx ctx;
  ctx.cfg.n_workers = 4;
  const int shapes[][2] = {{33278, 650}, {2600, 650}, {40, 24}, {70000, 33}};
  for (auto& s : shapes) {
    acc::DevLayer l{};
    l.rows = s[0]; l.cols = s[1]; l.kind = ACC_MATRIX;
    ctx.plan.layers.push_back(l);
  }
  ctx.cfg.n_layers = (int)ctx.plan.layers.size();
  const long long tokens[] = {35, 700, 4096, 65};
  size_t want[4][4];
  for (int l = 0; l < 4; ++l)
    for (int k = 0; k < 4; ++k)
      if (acc_linear_grad_workspace_bytes(&ctx, l, tokens[k], &want[l][k]) != ACC_OK) return 2;
  std::atomic<long long> wrong{0};
  auto ask = [&](unsigned seed) {
    for (int i = 0; i < 150000; ++i) {
      seed = seed * 1664525u + 1013904223u;
      const int l = seed >> 30, k = (seed >> 28) & 3;
      size_t bytes = 0;
      if (acc_linear_grad_workspace_bytes(&ctx, l, tokens[k], &bytes) != ACC_OK || bytes != want[l][k]) ++wrong;
    }
  };
  std::thread threads[] = {std::thread(ask, 1u), std::thread(ask, 2u), std::thread(ask, 3u), std::thread(ask, 4u)};
  for (auto& t : threads) t.join();
  std::printf("%lld wrong answers\n", wrong.load());
  return wrong.load() ? 1 : 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    lib = build.build_library()
    folder = tmp_path_factory.mktemp("query")
    source, binary = folder / "query.cu", folder / "query"
    source.write_text(PROGRAM)
    subprocess.run([build._nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-O1", "-I", os.path.join(build.ROOT, "include"),
                    "-I", build.CSRC, str(source), lib, "-Xlinker", "-rpath", "-Xlinker", os.path.dirname(lib), "-o", str(binary)],
                   check=True, capture_output=True, text=True)
    return str(binary)


def test_threads_that_ask_at_once_get_their_own_answers(program):
    done = subprocess.run([program], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stdout + done.stderr


def test_most_columns(program):
    assert subprocess.run([program, "columns"], timeout=60).returncode == 0
