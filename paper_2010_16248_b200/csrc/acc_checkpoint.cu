// Activation checkpoints in 8 bits: e4m3 codes with a power of two for each 32 columns of a row, written and read back.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <type_traits>

#include "acc_internal.cuh"

namespace acc {

constexpr int kBlock = ACC_CHECKPOINT_BLOCK;  // columns that share a scale
static_assert(kBlock == 32, "two lanes of sixteen columns hold a block");

// The larger magnitudes of two pairs of bf16, NaN when one is (a of magnitudes); one instruction, where the integer maximum of
// two halves takes several.
__device__ __forceinline__ unsigned max_abs2(unsigned a, unsigned b) {
  unsigned y;
  asm("{\n  .reg .b32 m;\n  abs.bf16x2 m, %2;\n  max.NaN.bf16x2 %0, %1, m;\n}\n" : "=r"(y) : "r"(a), "r"(b));
  return y;
}
__device__ __forceinline__ unsigned as_bits(float x) { return __float_as_uint(x); }
__device__ __forceinline__ unsigned as_bits(__nv_bfloat16 x) { return __bfloat16_as_ushort(x); }

struct CkptArgs {
  void* x;              // [n] rows of ld elements
  long long n, ld;
  int cols;
  const void* tokens;   // nullptr, or one per row: rows of negative tokens are zeros and not read
  int token64;
  uint8_t* code;        // [n][32 blocks]
  uint8_t* scale;       // [n][blocks]
  int blocks;           // of a row
  int units;            // of a row
  float inv_units;
  bool narrow;          // all units' numbers fit 32 bits (a division of 64 is a hundred instructions)
  const char *first, *end;  // the rows' bytes
};

// Where a thread's k-th unit lies: units count through the rows, a block of threads takes a stretch of them.  The first of the
// stretch in 64 bits, the way from there in fp32 (below 2^22, and half a unit away from the next whole number).
struct CkptPlace {
  long long row;
  int unit;
  template <int UNITS> __device__ __forceinline__ static CkptPlace of(const CkptArgs& a, int k) {
    const long long base = (long long)blockIdx.x * (blockDim.x * UNITS);
    const long long row0 = a.narrow ? (long long)((unsigned)base / (unsigned)a.units) : base / a.units;
    const int from = (int)(base - row0 * a.units), way = k * (int)blockDim.x + (int)threadIdx.x;
    int at = from + way;
    CkptPlace p;
    p.row = row0;
    if (a.units < (1 << 20)) {
      const int rows = (int)(((float)at + 0.5f) * a.inv_units);
      p.row += rows;
      at -= rows * a.units;
    } else if (at >= a.units) {  // (a stretch is shorter than such a row)
      p.row += 1;
      at -= a.units;
    }
    p.unit = at;
    return p;
  }
};

constexpr int kCkptThreads = 256;
// Units a thread has under way, at least 64 bytes of x.
template <typename T> constexpr int kStoreUnits = 4 / (int)sizeof(T);
constexpr int kLoadUnits = 4;

// The bits of sixteen neighbouring values of a row, columns behind the row zeros: the 16-byte pieces that hold them, moved (rows
// that do not start on 16 bytes: !ROWS16) by whole words, then by half of one.  Pieces may hold bytes of a neighbouring row or
// of what lies between, but none from outside the rows: at their first and last the values come one by one.
template <typename T> constexpr int kWords = 16 * (int)sizeof(T) / 4;
template <typename T, bool ROWS16>
__device__ __forceinline__ void load_sixteen(const CkptArgs& a, long long row, int c, unsigned* w) {
  constexpr int N = kWords<T>;
  const T* const p = static_cast<const T*>(a.x) + row * a.ld + c;
  const int live = min(16, a.cols - c);
  if (live <= 0) return;  // (w holds zeros)
  const char* const at = reinterpret_cast<const char*>(reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)15);
  const int by = ROWS16 ? 0 : (int)(reinterpret_cast<uintptr_t>(p) & 15), pieces = (by + live * (int)sizeof(T) + 15) / 16;
  if (at >= a.first && at + 16 * pieces <= a.end) {
    unsigned v[N + 4];
#pragma unroll
    for (int k = 0; k < N / 4 + !ROWS16; ++k) {
      uint4 x = make_uint4(0, 0, 0, 0);
      if (k < pieces) x = __ldcs(reinterpret_cast<const uint4*>(at) + k);
      v[4 * k] = x.x; v[4 * k + 1] = x.y; v[4 * k + 2] = x.z; v[4 * k + 3] = x.w;
    }
    if (!ROWS16) {
#pragma unroll
      for (int k = 0; k < N + 3; ++k) v[k] = by & 4 ? v[k + 1] : v[k];
#pragma unroll
      for (int k = 0; k < N + 1; ++k) v[k] = by & 8 ? v[k + 2] : v[k];
      if (sizeof(T) == 2) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = by & 2 ? __funnelshift_r(v[k], v[k + 1], 16) : v[k];
      }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) w[k] = v[k];
    if (live < 16) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        if (sizeof(T) == 4) w[k] = k < live ? w[k] : 0u;
        else w[k] = 2 * k + 1 < live ? w[k] : 2 * k < live ? w[k] & 0xffffu : 0u;
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      if (k >= live) break;
      if (sizeof(T) == 4) w[k % N] = as_bits(p[k]);
      else w[k / 2] |= as_bits(p[k]) << (16 * (k & 1));
    }
  }
}

// Codes and scales of a row, sixteen columns a thread.  The scale's byte is the exponent that brings the largest magnitude of the
// block into [128, 256); the product with its inverse is exact (but below 2^-126, far below the least code), and rounding to
// the nearest e4m3 is the only one.  131072 rows of 650 in bf16, a tenth padding: 49 us, 5.0 TB/s (it issues in 78 % of the
// cycles, 14 instructions a value; 53 us with the rows' last columns one by one, 72 with eight columns a thread, 115 with a 64-bit
// division for each).  Rows that start on 4 bytes: 60 us, and 167 with 4-byte loads.
template <typename T, bool ROWS16>
__global__ void __launch_bounds__(kCkptThreads) checkpoint_store_kernel(const CkptArgs a) {
  await_previous();
  let_next_start();
  constexpr int U = kStoreUnits<T>, N = kWords<T>;
  unsigned w[U][N];
  CkptPlace at[U];
  bool live[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    at[u] = CkptPlace::of<U>(a, u);
    live[u] = at[u].row < a.n;
  }
  if (a.tokens != nullptr) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (live[u])
        live[u] = (a.token64 ? static_cast<const long long*>(a.tokens)[at[u].row]
                             : static_cast<const int*>(a.tokens)[at[u].row]) >= 0;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
#pragma unroll
    for (int k = 0; k < N; ++k) w[u][k] = 0;
    if (live[u]) load_sixteen<T, ROWS16>(a, at[u].row, 16 * at[u].unit, w[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    // magnitudes compare as integers, NaN and infinity above all
    unsigned top = 0;
    if (sizeof(T) == 2) {
#pragma unroll
      for (int k = 0; k < N; ++k) top = max_abs2(top, w[u][k]);
      top = max(top << 16, top & 0xffff0000u);
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k) top = max(top, w[u][k] & 0x7fffffffu);
    }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    // floor(log2 of the largest) - 7 + 127; 1 where that is less (its factor 2^126 is the largest there is a use for)
    const bool odd = top >= 0x7f800000u;
    const int byte = odd ? 255 : top == 0 ? 0 : max((int)(top >> 23) - 7, 1);
    const float factor = __uint_as_float(odd ? 0x7fffffffu : (unsigned)(254 - byte) << 23);  // (NaN makes every code NaN)
    unsigned code[4];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float lo = sizeof(T) == 2 ? __uint_as_float(w[u][k % N] << 16) : __uint_as_float(w[u][(2 * k) % N]);
      const float hi = sizeof(T) == 2 ? __uint_as_float(w[u][k % N] & 0xffff0000u) : __uint_as_float(w[u][(2 * k + 1) % N]);
      unsigned short h;
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(h) : "f"(hi * factor), "f"(lo * factor));
      code[k / 2] = k & 1 ? code[k / 2] | (unsigned)h << 16 : h;
    }
    if (at[u].row >= a.n) continue;
    uint8_t* const to = a.code + at[u].row * (a.blocks * kBlock) + 16 * at[u].unit;
    *reinterpret_cast<uint4*>(to) = make_uint4(code[0], code[1], code[2], code[3]);
    if ((at[u].unit & 1) == 0) a.scale[at[u].row * a.blocks + (at[u].unit >> 1)] = (uint8_t)byte;
  }
}

// 2^(byte - 127), NaN for 255.
__device__ __forceinline__ float scale_value(unsigned byte) {
  return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7fffffffu : byte << 23);
}

// The values, 16 bytes of them a thread: V columns from column V * unit, or (rows that start anywhere) those that lie in one
// 16-byte piece of memory, whose codes start at any byte and may belong to two blocks.  131072 rows of 650 to bf16: 48 us, 5.4
// TB/s; rows that start on 4 bytes: 82 us, and 216 with 4-byte stores, which fill a 32-byte place of memory by eighths.
template <typename T, bool ROWS16>
__global__ void __launch_bounds__(kCkptThreads) checkpoint_load_kernel(const CkptArgs a) {
  await_previous();
  let_next_start();
  constexpr int U = kLoadUnits, V = 16 / (int)sizeof(T);
  CkptPlace at[U];
  int c[U];              // first column, negative where the piece begins before the row
  unsigned code[U][2], byte[U][2];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    at[u] = CkptPlace::of<U>(a, u);
    c[u] = V * at[u].unit;
    if (!ROWS16) c[u] -= (int)(reinterpret_cast<uintptr_t>(static_cast<const T*>(a.x) + at[u].row * a.ld) % 16 / sizeof(T));
    if (at[u].row >= a.n) c[u] = a.cols;
    if (c[u] >= a.cols) continue;
    const uint8_t* const codes = a.code + at[u].row * (a.blocks * kBlock);
    const uint8_t* const scales = a.scale + at[u].row * a.blocks;
    if (ROWS16) {
      if (V == 8) {
        const uint2 x = *reinterpret_cast<const uint2*>(codes + c[u]);
        code[u][0] = x.x;
        code[u][1] = x.y;
      } else {
        code[u][0] = *reinterpret_cast<const unsigned*>(codes + c[u]);
      }
      byte[u][0] = byte[u][1] = scales[c[u] / kBlock];
    } else {
      const int from = c[u] & ~3, by = 8 * (c[u] & 3);  // (columns below 0 or behind the codes: anything)
      unsigned w[V / 4 + 1];
#pragma unroll
      for (int k = 0; k < V / 4 + 1; ++k)
        w[k] = from + 4 * k >= 0 && from + 4 * k < a.blocks * kBlock
                   ? *reinterpret_cast<const unsigned*>(codes + from + 4 * k) : 0u;
#pragma unroll
      for (int k = 0; k < V / 4; ++k) code[u][k] = __funnelshift_r(w[k], w[k + 1], by);
      byte[u][0] = scales[max(c[u], 0) / kBlock];
      byte[u][1] = scales[min(c[u] + V - 1, a.cols - 1) / kBlock];
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (c[u] >= a.cols) continue;
    const float s0 = scale_value(byte[u][0]), s1 = scale_value(byte[u][1]);
    const int turn = ROWS16 ? V : kBlock - (c[u] & (kBlock - 1));  // values before the second block
    float v[V];
#pragma unroll
    for (int k = 0; k < V; k += 2) {
      const unsigned short h = (unsigned short)(code[u][k / 4] >> (8 * (k & 2)));
      unsigned f;
      asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(f) : "h"(h));
      const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&f));
      v[k] = p.x * (k < turn ? s0 : s1);
      v[k + 1] = p.y * (k + 1 < turn ? s0 : s1);
    }
    T* const p = static_cast<T*>(a.x) + at[u].row * a.ld + c[u];
    if (c[u] >= 0 && c[u] + V <= a.cols) {
      uint4 y;
      if constexpr (V == 8) {
        unsigned w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
          w[k] = *reinterpret_cast<const unsigned*>(&h);
        }
        y = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
        y = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
      }
      *reinterpret_cast<uint4*>(p) = y;
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k) {
        if (c[u] + k < 0 || c[u] + k >= a.cols) continue;
        if constexpr (V == 8) p[k] = __float2bfloat16_rn(v[k]);
        else p[k] = v[k];
      }
    }
  }
}

cudaError_t launch_checkpoint(acc_ctx* ctx, bool store, void* x, bool bf16, long long n, int cols, long long ld,
                              const void* tokens, bool tok64, uint8_t* code, uint8_t* scale, cudaStream_t s) {
  const int blocks = (cols + kBlock - 1) / kBlock, size = bf16 ? 2 : 4;
  const char* const first = static_cast<const char*>(x);
  CkptArgs a{x, n, ld, cols, tokens, tok64, code, scale, blocks, 0, 0.f, false, first, first + ((n - 1) * ld + cols) * size};
  const bool rows16 = (reinterpret_cast<uintptr_t>(x) | (n > 1 ? (uintptr_t)(ld * size) : 0)) % 16 == 0;
  // a row's pieces of 16 bytes of output are one more where it starts inside one
  a.units = store ? 2 * blocks : (cols + 16 / size - 1) / (16 / size) + !rows16;
  a.inv_units = 1.f / (float)a.units;
  a.narrow = n * a.units < (1ll << 32) - (1 << 16);
  PhaseTimer pt(ctx, store ? PH_CKPT_STORE : PH_CKPT_LOAD, s);
  auto go = [&](auto t) {
    using T = decltype(t);
    const long long per = kCkptThreads * (store ? kStoreUnits<T> : kLoadUnits), all = n * a.units;
    auto* kernel = store ? (rows16 ? checkpoint_store_kernel<T, true> : checkpoint_store_kernel<T, false>)
                         : (rows16 ? checkpoint_load_kernel<T, true> : checkpoint_load_kernel<T, false>);
    return launch_early(kernel, (unsigned)((all + per - 1) / per), kCkptThreads, s, a);
  };
  return bf16 ? go(__nv_bfloat16()) : go(0.f);
}

}  // namespace acc
