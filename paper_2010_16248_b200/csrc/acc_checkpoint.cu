// Activation checkpoints in 8 bits: e4m3 codes with a power of two for each 32 columns of a row, written and read back.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <type_traits>

#include "acc_internal.cuh"

namespace acc {

constexpr int kBlock = ACC_CHECKPOINT_BLOCK;  // columns that share a scale: four threads of eight
static_assert(kBlock == 32, "four neighbouring lanes hold a block");

// VEC neighbouring elements of a row whose start is aligned to VEC elements (or to 16 bytes), as fp32.
template <int VEC> __device__ __forceinline__ void load_eight(const float* p, float* v) {
  if constexpr (VEC == 8) {
    const float4 a = __ldcs(reinterpret_cast<const float4*>(p)), b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else if constexpr (VEC >= 2) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 a = *reinterpret_cast<const float2*>(p + 2 * k);
      v[2 * k] = a.x; v[2 * k + 1] = a.y;
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = p[k];
  }
}
template <int VEC> __device__ __forceinline__ void load_eight(const __nv_bfloat16* p, float* v) {
  unsigned w[4];
  if constexpr (VEC == 8) {
    const uint4 a = __ldcs(reinterpret_cast<const uint4*>(p));
    w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
  } else if constexpr (VEC >= 2) {
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = reinterpret_cast<const unsigned*>(p)[k];
  } else {
    const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = q[2 * k] | (unsigned)q[2 * k + 1] << 16;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[2 * k] = __uint_as_float(w[k] << 16);
    v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
  }
}
template <int VEC> __device__ __forceinline__ void store_eight(float* p, const float* v) {
  if constexpr (VEC == 8) {
    __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
    __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(v[4], v[5], v[6], v[7]));
  } else if constexpr (VEC >= 2) {
#pragma unroll
    for (int k = 0; k < 4; ++k) *reinterpret_cast<float2*>(p + 2 * k) = make_float2(v[2 * k], v[2 * k + 1]);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) p[k] = v[k];
  }
}
template <int VEC> __device__ __forceinline__ void store_eight(__nv_bfloat16* p, const float* v) {
  unsigned w[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
    w[k] = *reinterpret_cast<const unsigned*>(&h);
  }
  if constexpr (VEC == 8) {
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
  } else if constexpr (VEC >= 2) {
#pragma unroll
    for (int k = 0; k < 4; ++k) reinterpret_cast<unsigned*>(p)[k] = w[k];
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      reinterpret_cast<unsigned short*>(p)[2 * k] = (unsigned short)w[k];
      reinterpret_cast<unsigned short*>(p)[2 * k + 1] = (unsigned short)(w[k] >> 16);
    }
  }
}

struct CkptArgs {
  void* x;              // [n] rows of ld elements
  long long n, ld;
  int cols;
  const void* tokens;   // nullptr, or one per row: rows of negative tokens are zeros and not read
  int token64;
  uint2* code;          // [n][eights]
  uint8_t* scale;       // [n][blocks]
  int eights, blocks;   // of a row: eight columns each, thirty-two each
};

// Place of this thread's eight columns; false behind the last row.
struct CkptPlace { long long row; int eight; };
__device__ __forceinline__ bool ckpt_place(const CkptArgs& a, int per_block, int k, CkptPlace& p) {
  // (a block's first place in 64 bits, the rest of the way in 32)
  const long long base = (long long)blockIdx.x * per_block;
  const long long row0 = base / a.eights;
  const unsigned at = (unsigned)(base - row0 * a.eights) + k * blockDim.x + threadIdx.x;
  p.row = row0 + at / (unsigned)a.eights;
  p.eight = (int)(at % (unsigned)a.eights);
  return p.row < a.n;
}

constexpr int kCkptThreads = 256, kCkptUnits = 2;  // units of eight columns a thread

// Codes and scales of a row.  The scale's byte is the exponent that brings the largest magnitude of the block into [128, 256);
// values are then exact multiples of a power of two away from x, and rounding to the nearest e4m3 is the only one.
template <typename T, int VEC>
__global__ void __launch_bounds__(kCkptThreads) checkpoint_store_kernel(const CkptArgs a) {
  await_previous();
  let_next_start();
  float v[kCkptUnits][8];
  CkptPlace at[kCkptUnits];
  bool on[kCkptUnits];
#pragma unroll
  for (int u = 0; u < kCkptUnits; ++u) {
    on[u] = ckpt_place(a, kCkptThreads * kCkptUnits, u, at[u]);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[u][k] = 0.f;
    if (!on[u]) continue;
    if (a.tokens != nullptr) {
      const long long t = a.token64 ? static_cast<const long long*>(a.tokens)[at[u].row]
                                    : static_cast<const int*>(a.tokens)[at[u].row];
      if (t < 0) continue;
    }
    const int c = 8 * at[u].eight;
    const T* p = static_cast<const T*>(a.x) + at[u].row * a.ld + c;
    if (c + 8 <= a.cols) {
      load_eight<VEC>(p, v[u]);
    } else {
      for (int k = 0; k < a.cols - c; ++k) {
        if constexpr (sizeof(T) == 2) v[u][k] = __bfloat162float(p[k]);
        else v[u][k] = p[k];
      }
    }
  }
#pragma unroll
  for (int u = 0; u < kCkptUnits; ++u) {
    // magnitudes compare as integers, NaN and infinity above all
    unsigned top = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) top = max(top, __float_as_uint(v[u][k]) & 0x7fffffffu);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    // floor(log2 of the largest) - 7 + 127; 1 where that is less (its factor 2^126 is the largest there is a use for)
    int byte = top >= 0x7f800000u ? 255 : top == 0 ? 0 : max((int)(top >> 23) - 7, 1);
    const float factor = __int_as_float((254 - min(byte, 254)) << 23);
    unsigned w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      unsigned short h;
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(h) : "f"(v[u][2 * k + 1] * factor), "f"(v[u][2 * k] * factor));
      w[k] = h;
    }
    if (!on[u]) continue;
    uint2 code = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
    if (byte == 255) code = make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu);
    a.code[at[u].row * a.eights + at[u].eight] = code;
    if ((at[u].eight & 3) == 0) a.scale[at[u].row * a.blocks + (at[u].eight >> 2)] = (uint8_t)byte;
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
  CkptPlace at[kCkptUnits];
  bool on[kCkptUnits];
  uint2 code[kCkptUnits];
  unsigned byte[kCkptUnits];
#pragma unroll
  for (int u = 0; u < kCkptUnits; ++u) {
    on[u] = ckpt_place(a, kCkptThreads * kCkptUnits, u, at[u]) && 8 * at[u].eight < a.cols;
    if (!on[u]) continue;
    code[u] = __ldcs(a.code + at[u].row * a.eights + at[u].eight);
    byte[u] = a.scale[at[u].row * a.blocks + (at[u].eight >> 2)];
  }
#pragma unroll
  for (int u = 0; u < kCkptUnits; ++u) {
    if (!on[u]) continue;
    const float s = scale_value(byte[u]);
    float v[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const unsigned short h = (unsigned short)((k < 2 ? code[u].x : code[u].y) >> (16 * (k & 1)));
      unsigned f;
      asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(f) : "h"(h));
      const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&f));
      v[2 * k] = p.x * s;
      v[2 * k + 1] = p.y * s;
    }
    const int c = 8 * at[u].eight;
    T* p = static_cast<T*>(a.x) + at[u].row * a.ld + c;
    if (c + 8 <= a.cols) {
      store_eight<VEC>(p, v);
    } else {
      for (int k = 0; k < a.cols - c; ++k) {
        if constexpr (sizeof(T) == 2) p[k] = __float2bfloat16_rn(v[k]);
        else p[k] = v[k];
      }
    }
  }
}

// Widest access at which every eight columns of every row start aligned: 8 elements (16 bytes at least), 2, or 1.
static int ckpt_vec(const void* x, long long n, long long ld, int size) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(x) | (n > 1 ? (uintptr_t)(ld * size) : 0);
  return at % 16 == 0 ? 8 : at % (2 * size) == 0 ? 2 : 1;
}

cudaError_t launch_checkpoint(acc_ctx* ctx, bool store, void* x, bool bf16, long long n, int cols, long long ld,
                              const void* tokens, bool tok64, uint8_t* code, uint8_t* scale, cudaStream_t s) {
  const int blocks = (cols + kBlock - 1) / kBlock;
  const CkptArgs a{x, n, ld, cols, tokens, tok64, reinterpret_cast<uint2*>(code), scale, 4 * blocks, blocks};
  const long long units = n * a.eights, per = kCkptThreads * kCkptUnits;
  const int vec = ckpt_vec(x, n, ld, bf16 ? 2 : 4);
  PhaseTimer pt(ctx, store ? PH_CKPT_STORE : PH_CKPT_LOAD, s);
  auto go = [&](auto t, auto v) {
    using T = decltype(t);
    constexpr int VEC = decltype(v)::value;
    return launch_early(store ? checkpoint_store_kernel<T, VEC> : checkpoint_load_kernel<T, VEC>,
                        (unsigned)((units + per - 1) / per), kCkptThreads, s, a);
  };
  auto typed = [&](auto t) {
    if (vec == 8) return go(t, std::integral_constant<int, 8>());
    return vec == 2 ? go(t, std::integral_constant<int, 2>()) : go(t, std::integral_constant<int, 1>());
  };
  return bf16 ? typed(__nv_bfloat16()) : typed(0.f);
}

}  // namespace acc
