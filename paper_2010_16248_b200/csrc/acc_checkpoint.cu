// Activation checkpoints in 8 bits: e4m3 codes with a power of two for each 32 columns of a row, written and read back.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <type_traits>

#include "acc_internal.cuh"

namespace acc {

constexpr int kBlock = ACC_CHECKPOINT_BLOCK;  // columns that share a scale
static_assert(kBlock == 32, "lanes of a warp hold whole blocks");

// VEC neighbouring values as loaded and stored: 16 bytes where every row starts on 16, else two, else one.
template <typename T, int VEC> struct Some;
template <> struct Some<float, 4> { using type = float4; };
template <> struct Some<float, 2> { using type = float2; };
template <> struct Some<float, 1> { using type = float; };
template <> struct Some<__nv_bfloat16, 8> { using type = uint4; };
template <> struct Some<__nv_bfloat16, 2> { using type = unsigned; };
template <> struct Some<__nv_bfloat16, 1> { using type = unsigned short; };
template <int VEC> struct Codes;
template <> struct Codes<8> { using type = uint2; };
template <> struct Codes<4> { using type = unsigned; };
template <> struct Codes<2> { using type = unsigned short; };
template <> struct Codes<1> { using type = unsigned char; };

template <typename T, int VEC> union Values {
  typename Some<T, VEC>::type raw;
  T each[VEC];
  __device__ __forceinline__ Values() {}
};
__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_float(float& y, float x) { y = x; }
__device__ __forceinline__ void from_float(__nv_bfloat16& y, float x) { y = __float2bfloat16_rn(x); }

struct CkptArgs {
  void* x;              // [n] rows of ld elements
  long long n, ld;
  int cols;
  const void* tokens;   // nullptr, or one per row: rows of negative tokens are zeros and not read
  int token64;
  uint8_t* code;        // [n][32 blocks]
  uint8_t* scale;       // [n][blocks]
  int blocks;           // of a row
  int units;            // of VEC columns, of a row
  float inv_units;
};

// Where a thread's k-th unit lies: units count through the rows, a block of threads takes a stretch of them.  The first of the
// stretch in 64 bits, the way from there in fp32 (below 2^22, and half a unit away from the next whole number).
struct CkptPlace {
  long long row;
  int unit;
  template <int UNITS> __device__ __forceinline__ static CkptPlace of(const CkptArgs& a, int k) {
    const long long base = (long long)blockIdx.x * (blockDim.x * UNITS);
    const long long row0 = base / a.units;
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
// Units a thread has under way: 64 bytes and more of x.
template <int VEC> constexpr int kCkptUnits = VEC == 8 ? 4 : 8;

// Codes and scales of a row.  The scale's byte is the exponent that brings the largest magnitude of the block into [128, 256);
// values are then exact multiples of a power of two away from x, and rounding to the nearest e4m3 is the only one.
template <typename T, int VEC>
__global__ void __launch_bounds__(kCkptThreads) checkpoint_store_kernel(const CkptArgs a) {
  await_previous();
  let_next_start();
  constexpr int U = kCkptUnits<VEC>;
  Values<T, VEC> x[U];
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
      if (live[u]) live[u] = (a.token64 ? static_cast<const long long*>(a.tokens)[at[u].row] : static_cast<const int*>(a.tokens)[at[u].row]) >= 0;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
#pragma unroll
    for (int k = 0; k < VEC; ++k) from_float(x[u].each[k], 0.f);
    const int c = VEC * at[u].unit;
    const T* const p = static_cast<const T*>(a.x) + at[u].row * a.ld + c;
    if (live[u] && c + VEC <= a.cols) {
      x[u].raw = __ldcs(reinterpret_cast<const typename Some<T, VEC>::type*>(p));
    } else if (live[u]) {
#pragma unroll
      for (int k = 0; k < VEC; ++k)
        if (c + k < a.cols) x[u].each[k] = p[k];
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    // magnitudes compare as integers, NaN and infinity above all
    unsigned top = 0;
    if constexpr (sizeof(T) == 2 && VEC == 8) {
      const uint4 w = x[u].raw;
      const unsigned two = __vmaxu2(__vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu), __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu));
      top = max(two << 16, two & 0xffff0000u);
    } else {
#pragma unroll
      for (int k = 0; k < VEC; ++k) top = max(top, __float_as_uint(as_float(x[u].each[k])) & 0x7fffffffu);
    }
#pragma unroll
    for (int o = 1; o < kBlock / VEC; o *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    // floor(log2 of the largest) - 7 + 127; 1 where that is less (its factor 2^126 is the largest there is a use for)
    const int byte = top >= 0x7f800000u ? 255 : top == 0 ? 0 : max((int)(top >> 23) - 7, 1);
    const float factor = __int_as_float((254 - min(byte, 254)) << 23);
    union { unsigned char each[VEC]; typename Codes<VEC>::type raw; } code;
#pragma unroll
    for (int k = 0; k < VEC; k += 2) {
      unsigned short h;
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(h) : "f"(as_float(x[u].each[VEC > 1 ? k + 1 : k]) * factor), "f"(as_float(x[u].each[k]) * factor));
      if (byte == 255) h = 0x7f7f;
      code.each[k] = (unsigned char)h;
      if (VEC > 1) code.each[k + 1] = (unsigned char)(h >> 8);
    }
    if (at[u].row >= a.n) continue;
    *reinterpret_cast<typename Codes<VEC>::type*>(a.code + at[u].row * (a.blocks * kBlock) + VEC * at[u].unit) = code.raw;
    if (at[u].unit % (kBlock / VEC) == 0) a.scale[at[u].row * a.blocks + at[u].unit / (kBlock / VEC)] = (uint8_t)byte;
  }
}

// 2^(byte - 127), NaN for 255.
__device__ __forceinline__ float scale_value(unsigned byte) {
  return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7fffffffu : byte << 23);
}

template <typename T, int VEC>
__global__ void __launch_bounds__(kCkptThreads) checkpoint_load_kernel(const CkptArgs a) {
  await_previous();
  let_next_start();
  constexpr int U = kCkptUnits<VEC>;
  CkptPlace at[U];
  bool on[U];
  union { unsigned char each[VEC]; typename Codes<VEC>::type raw; } code[U];
  unsigned byte[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    at[u] = CkptPlace::of<U>(a, u);
    on[u] = at[u].row < a.n && VEC * at[u].unit < a.cols;
    if (!on[u]) continue;
    code[u].raw = *reinterpret_cast<const typename Codes<VEC>::type*>(a.code + at[u].row * (a.blocks * kBlock) + VEC * at[u].unit);
    byte[u] = a.scale[at[u].row * a.blocks + at[u].unit / (kBlock / VEC)];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (!on[u]) continue;
    const float s = scale_value(byte[u]);
    Values<T, VEC> y;
#pragma unroll
    for (int k = 0; k < VEC; k += 2) {
      unsigned short h = code[u].each[k];
      if (VEC > 1) h |= (unsigned short)(code[u].each[VEC > 1 ? k + 1 : k] << 8);
      unsigned f;
      asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(f) : "h"(h));
      const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&f));
      from_float(y.each[k], p.x * s);
      if (VEC > 1) from_float(y.each[VEC > 1 ? k + 1 : k], p.y * s);
    }
    const int c = VEC * at[u].unit;
    T* const p = static_cast<T*>(a.x) + at[u].row * a.ld + c;
    if (c + VEC <= a.cols) {
      *reinterpret_cast<typename Some<T, VEC>::type*>(p) = y.raw;
    } else {
#pragma unroll
      for (int k = 0; k < VEC; ++k)
        if (c + k < a.cols) p[k] = y.each[k];
    }
  }
}

cudaError_t launch_checkpoint(acc_ctx* ctx, bool store, void* x, bool bf16, long long n, int cols, long long ld,
                              const void* tokens, bool tok64, uint8_t* code, uint8_t* scale, cudaStream_t s) {
  const int blocks = (cols + kBlock - 1) / kBlock;
  CkptArgs a{x, n, ld, cols, tokens, tok64, code, scale, blocks, 0, 0.f};
  // 16 bytes where every row starts on 16 (and no row's last vector is read or written whole unless it is), two elements, or one
  const int size = bf16 ? 2 : 4;
  const uintptr_t each = reinterpret_cast<uintptr_t>(x) | (n > 1 ? (uintptr_t)(ld * size) : 0);
  const int vec = each % 16 == 0 ? 16 / size : each % (2 * size) == 0 ? 2 : 1;
  a.units = blocks * (kBlock / vec);
  a.inv_units = 1.f / (float)a.units;
  PhaseTimer pt(ctx, store ? PH_CKPT_STORE : PH_CKPT_LOAD, s);
  auto go = [&](auto t, auto v) {
    using T = decltype(t);
    constexpr int VEC = decltype(v)::value;
    const long long per = kCkptThreads * kCkptUnits<VEC>, all = n * a.units;
    return launch_early(store ? checkpoint_store_kernel<T, VEC> : checkpoint_load_kernel<T, VEC>,
                        (unsigned)((all + per - 1) / per), kCkptThreads, s, a);
  };
  auto typed = [&](auto t) {
    using T = decltype(t);
    if (vec > 2) return go(t, std::integral_constant<int, 16 / (int)sizeof(T)>());
    return vec == 2 ? go(t, std::integral_constant<int, 2>()) : go(t, std::integral_constant<int, 1>());
  };
  return bf16 ? typed(__nv_bfloat16()) : typed(0.f);
}

}  // namespace acc
