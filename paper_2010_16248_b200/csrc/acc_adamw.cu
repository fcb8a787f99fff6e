// AdamW update over the whole layer table, states in 32 bits or in 8 bits, and the clip factor it may be scaled by.
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "acc_internal.cuh"

namespace acc {

// The step's coefficients, worked out once per block in fp64 from the caller's doubles and the step count.
struct AdamCoef {  // 11 words
  float f;                 // factor on the gradient
  float b1, ob1, b2, ob2;  // beta1, 1 - beta1, beta2, 1 - beta2
  float lrwd;              // lr * weight_decay
  float size;              // lr / (1 - beta1^t)
  float rc2;               // 1 / sqrt(1 - beta2^t)
  float eps;
  unsigned key;            // of this step's random numbers (8-bit states)
  int skip;                // the factor is not finite: nothing changes (written by adamw_coef_kernel)
};

// b^t by squaring.  Every squaring doubles the relative error so far, so that of b^t grows like t 2^-53 (8000 of 2^-53 at
// 0.999^100000); what is needed is 1 - b^t, which sees t b^t 2^-53, and t b^t / (1 - b^t) <= 1 / (1 - b): its relative error
// stays under 2^-53 / (1 - b), far below the fp32 rounding that follows.
__device__ __forceinline__ double pow_int(double b, long long t) {
  double r = 1.0;
  for (; t > 0; t >>= 1) {
    if (t & 1) r *= b;
    b *= b;
  }
  return r;
}

// 32-bit integer mixing (two rounds of xor-shift and multiply, C. Wellons' constants): a bijection, so distinct elements
// of one step draw distinct words.
__device__ __forceinline__ unsigned mix32_open(unsigned x) {  // all but the last fold
  x ^= x >> 16;
  x *= 0x7feb352du;
  x ^= x >> 15;
  return x * 0x846ca68bu;
}
__device__ __forceinline__ unsigned mix32(unsigned x) {
  x = mix32_open(x);
  return x ^ (x >> 16);
}

// Two lanes take one power each.
__device__ __forceinline__ void adam_coef(AdamCoef* c, const double* hyper, long long t, float f,
                                          unsigned seed) {
  if (threadIdx.x >= 2) return;
  const double lr = hyper[0], b = hyper[1 + threadIdx.x];
  const double corr = 1.0 - pow_int(b, t);
  if (threadIdx.x == 0) {
    c->f = f;
    c->b1 = (float)b;
    c->ob1 = (float)(1.0 - b);
    c->lrwd = (float)(lr * hyper[4]);
    c->size = (float)(lr / corr);
    c->eps = (float)hyper[3];
    c->key = mix32(seed + 0x9e3779b9u * (unsigned)t);
  } else {
    c->b2 = (float)b;
    c->ob2 = (float)(1.0 - b);
    c->rc2 = (float)(1.0 / sqrt(corr));
  }
}

// A factor that is not finite means that the gradient's norm was not: the call then changes nothing.
__device__ __forceinline__ float adam_factor(const float* factor, bool& skip) {
  const float f = factor != nullptr ? *factor : 1.f;
  skip = !isfinite(f);
  return f;
}

// div.approx: 2 ulp for divisors in [2^-126, 2^126], one reciprocal and one product; the update's own roundings are of that
// size, and the correctly rounded quotient with its range checks costs the 8-bit kernel ten more instructions per element.
__device__ __forceinline__ float div_fast(float a, float b) {
  float r;
  asm("div.approx.ftz.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {  // NaN where either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// The update of one element: the old moments arrive as factors, beta1 m = ka a and beta2 v = kb b; m, v, r = sqrt(v) are
// the new ones in fp32; returns the new parameter.  The moments are sums of two rounded products and a rounded root, the
// formulas taken word by word: no fused step, so that a state's code does not hang on how a compiler contracts them.
__device__ __forceinline__ float adam_update(float d, float x, float a, float ka, float b, float kb, float& m, float& v,
                                             float& r, const AdamCoef& c, float lrwd) {
  const float g = c.f * d;
  m = __fadd_rn(__fmul_rn(ka, a), __fmul_rn(c.ob1, g));
  v = __fadd_rn(__fmul_rn(kb, b), __fmul_rn(c.ob2, __fmul_rn(g, g)));
  r = __fsqrt_rn(v);
  return fmaf(-c.size, div_fast(m, fmaf(r, c.rc2, c.eps)), fmaf(-lrwd, x, x));
}

__device__ __forceinline__ uint2 bf16x4(const float4 v) {
  const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x, v.y), hi = __floats2bfloat162_rn(v.z, v.w);
  return make_uint2(*reinterpret_cast<const unsigned*>(&lo), *reinterpret_cast<const unsigned*>(&hi));
}

// A warp takes one unit of 256 elements of a tile (a unit never spans layers, and with states in 8 bits it is a block of its
// own scale), eight elements per lane as two vectors of four at 4 lane and 128 + 4 lane: full lines, and a block's largest
// magnitude is one warp reduction away.  All of a warp's loads go out at once, before the coefficients are looked at.
//
// Coefficients.  Working them out takes fp64 powers, a quotient and a root, about 1 us.  Where all blocks are resident at
// once (ONE), each does so itself behind its loads, and the last block to finish advances the step count.  Larger tables,
// whose blocks follow one another on an SM and would pay that time again and again, take them from a kernel of one warp
// launched ahead; the update's blocks start beside it and wait for it behind their loads.  In every block / from a kernel
// ahead: 0.29 M parameters 3.4 / 3.7 us (and one launch less), 5.1 M in 8 bits 20.9 / 16.4 us, 50.1 M in 8 bits 171 / 138 us.
constexpr int kUnit = ACC_ADAMW_BLOCK, kUnitsPerTile = kTile / kUnit, kBlocksPerTile = kUnitsPerTile / 8;

__global__ void adamw_coef_kernel(AdamCoef* c, long long* step, const double* hyper,
                                  const float* factor, unsigned seed) {
  await_previous();
  let_next_start();  // (what the update loads ahead of its own wait was complete before this kernel's)
  bool skip;
  const float f = adam_factor(factor, skip);
  const long long t = *step + 1;
  adam_coef(c, hyper, t, f, seed);
  __syncwarp();
  if (threadIdx.x == 0) {
    c->skip = skip;
    if (!skip) *step = t;
  }
}

// ONE waits for the work ahead of the call itself; otherwise the coefficients' kernel has, before this one could begin.
template <bool ONE>
__device__ __forceinline__ void adam_enter() {
  if (ONE) await_previous();
  let_next_start();
}

// The block's coefficients, from `pre` or worked out here; false where nothing is to change.
template <bool ONE>
__device__ __forceinline__ bool adam_begin(AdamCoef& c, AdamCoef* sc, const AdamCoef* pre, const long long* step,
                                           const double* hyper, const float* factor,
                                           unsigned seed) {
  if (ONE) {
    bool skip;
    const float f = adam_factor(factor, skip);
    if (skip) return false;
    adam_coef(sc, hyper, *step + 1, f, seed);
    __syncthreads();
    c = *sc;
    return true;
  }
  await_previous();
  c = *pre;
  return c.skip == 0;
}

// ONE: every block has read the step count before it arrives here, so the last one may advance it; it also leaves the
// ticket at zero for the next call.
template <bool ONE>
__device__ __forceinline__ void adam_finish(long long* step, unsigned* ticket) {
  if (!ONE) return;
  __syncthreads();
  if (threadIdx.x == 0 && atomicAdd(ticket, 1u) == gridDim.x - 1) {
    *ticket = 0;
    *step += 1;
  }
}

// A warp's unit: where it starts, how many elements it has (<= 0: none), which scale it holds.
struct AdamUnit { long long base, block; int n; bool decay; };
__device__ __forceinline__ AdamUnit adam_unit(const FlatTile* __restrict__ tiles, int flags) {
  const FlatTile t = tiles[blockIdx.x / kBlocksPerTile];
  const int i = (int)(blockIdx.x % kBlocksPerTile) * 8 + (int)(threadIdx.x >> 5), e = i * kUnit;
  return AdamUnit{t.base + e, t.block0 + i, min(t.nelem - e, kUnit), t.matrix || !(flags & ACC_ADAMW_NO_VECTOR_DECAY)};
}

// States in 32 bits: 16 B read and 12 B written per parameter, some 15 operations: bound by HBM (50.1 M parameters: 213 us,
// 6.6 TB/s; 234 us with a block per tile of 8192 elements and a loop over it, 252 us as persistent blocks).
template <bool ONE>
__global__ void __launch_bounds__(256)
adamw_kernel(const FlatTile* __restrict__ tiles, const float* d, float* params, float* ms, float* vs,
             const AdamCoef* pre, long long* step, const double* hyper, const float* factor,
             unsigned short* low, int flags, unsigned* ticket) {
  __shared__ AdamCoef sc;
  adam_enter<ONE>();
  const int lane = threadIdx.x & 31;
  const AdamUnit u = adam_unit(tiles, flags);
  float4 gs[2], xs[2], mv[2], vv[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int e = 128 * h + 4 * lane;
    // (layers start at multiples of four elements and the buffers end at one, so whole vectors are in bounds)
    if (e < u.n) {
      gs[h] = ld_stream4(d + u.base + e);
      xs[h] = *reinterpret_cast<const float4*>(params + u.base + e);
      mv[h] = ld_stream4(ms + u.base + e);
      vv[h] = ld_stream4(vs + u.base + e);
    }
  }
  AdamCoef c;
  if (!adam_begin<ONE>(c, &sc, pre, step, hyper, factor, 0u)) return;
  const float lrwd = u.decay ? c.lrwd : 0.f;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int e = 128 * h + 4 * lane;
    if (e >= u.n) continue;
    float4 x = xs[h], m = mv[h], v = vv[h];
    const float4 g = gs[h];
    float r;
    x.x = adam_update(g.x, x.x, m.x, c.b1, v.x, c.b2, m.x, v.x, r, c, lrwd);
    x.y = adam_update(g.y, x.y, m.y, c.b1, v.y, c.b2, m.y, v.y, r, c, lrwd);
    x.z = adam_update(g.z, x.z, m.z, c.b1, v.z, c.b2, m.z, v.z, r, c, lrwd);
    x.w = adam_update(g.w, x.w, m.w, c.b1, v.w, c.b2, m.w, v.w, r, c, lrwd);
    const long long at = u.base + e;
    if (e + 4 <= u.n) {
      *reinterpret_cast<float4*>(params + at) = x;
      st_stream4(ms + at, m);
      st_stream4(vs + at, v);
      if (low != nullptr) *reinterpret_cast<uint2*>(low + at) = bf16x4(x);
    } else {
      const float x3[3] = {x.x, x.y, x.z}, m3[3] = {m.x, m.y, m.z}, v3[3] = {v.x, v.y, v.z};
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (e + k < u.n) {
          params[at + k] = x3[k];
          ms[at + k] = m3[k];
          vs[at + k] = v3[k];
          if (low != nullptr) low[at + k] = __bfloat16_as_ushort(__float2bfloat16_rn(x3[k]));
        }
    }
  }
  adam_finish<ONE>(step, ticket);
}

// ---- states in 8 bits --------------------------------------------------------------------------------------------
// m and r = sqrt(v) are e4m3 numbers (4 bits of exponent, 3 of mantissa, subnormals at 2^-9) times a power of two shared
// by 256 elements (an e8m0 byte).  The root halves v's range of exponents, so 17 octaves of r cover 34 of v.  Scales are
// powers of two, so scaling is exact and the only rounding of a state is that to three bits of mantissa.  That rounding is
// stochastic: with beta2 = 0.999 a step moves r by 0.05 % while half a step of the grid is 3 to 6 %, so rounding to
// nearest would keep r where it is for good; with 16 random bits the expected value moves as the formula says.  A positive
// r is never rounded to 0, which would leave m divided by eps alone.
__device__ __forceinline__ float scale_of(unsigned byte) {  // 2^(byte - 127); 255 marks a block that is not finite
  return __uint_as_float(byte == 255u ? 0x7fc00000u : byte == 0u ? 0x00400000u : byte << 23);
}

// Scale byte for a block whose largest magnitude has the bits `top`: that element lands in [128, 256), one octave under
// the largest e4m3, so that rounding up needs no clamp.  `lowest` keeps what the codes stand for, and r's square, normal.
__device__ __forceinline__ unsigned scale_byte(unsigned top, int lowest) {
  if (top == 0u) return 0u;
  if (top >= 0x7f800000u) return 255u;
  return (unsigned)max((int)(top >> 23) - 7, lowest);
}
constexpr int kLowestM = 10, kLowestR = 73;

// e4m3's exponent bias is 120 below fp32's, so y 2^-120 in fp32 has y's e4m3 code in its bits 20 to 26, subnormals
// included (fp32's own subnormals begin where e4m3's do), and what rounding cuts below: adding 20 random bits there and
// cutting rounds up with the probability that the cut bits stand for.  This is the factor 2^(127 - byte - 120), as one
// float where that is normal; a block of larger values takes 2^-120 first (`big`).  Below the normal codes the product is
// an fp32 subnormal that keeps 20 bits under a step of the grid: it is cut, not rounded (__fmul_rz), as rounding up would
// carry some values before their random bits do.  What is cut lies below the 16 random bits and decides nothing.
__device__ __forceinline__ float code_factor(unsigned byte, bool& big) {
  big = byte > 133u;
  return byte == 0u || byte == 255u ? 0.f : __uint_as_float((big ? 254u - byte : 134u - byte) << 23);
}

__device__ __forceinline__ void decode4(unsigned codes, float* out) {
  const __half2 lo(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(codes & 0xffffu), __NV_E4M3));
  const __half2 hi(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(codes >> 16), __NV_E4M3));
  const float2 a = __half22float2(lo), b = __half22float2(hi);
  out[0] = a.x; out[1] = a.y; out[2] = b.x; out[3] = b.y;
}

// The top bytes of four words.
__device__ __forceinline__ unsigned top_bytes(unsigned a, unsigned b, unsigned c, unsigned d) {
  return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}

// 16.03 B per parameter and some 65 instructions, issued in 60 % of the cycles: 50.1 M parameters take 138 us, 5.8 TB/s (48
// registers and 40 warps per SM; 8 us more at 64 registers and 32 warps; the 48 spill 12 bytes in the kernel of small tables).
struct Adam8Regs { float4 d[2], x[2]; unsigned m[2], r[2], ms, rs; };
struct Adam8Args {
  const float* d; float* params; unsigned char* mc; unsigned char* rc; unsigned char* ms; unsigned char* rs;
  unsigned short* low;
};
__device__ __forceinline__ void adam8_load(Adam8Regs& q, const AdamUnit& u, int lane, const Adam8Args& p) {
  if (u.n <= 0) return;
  q.ms = p.ms[u.block];
  q.rs = p.rs[u.block];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int e = 128 * h + 4 * lane;
    q.d[h] = q.x[h] = make_float4(0.f, 0.f, 0.f, 0.f);
    q.m[h] = q.r[h] = 0u;
    if (e < u.n) {
      q.d[h] = ld_stream4(p.d + u.base + e);
      q.x[h] = *reinterpret_cast<const float4*>(p.params + u.base + e);
      q.m[h] = __ldcs(reinterpret_cast<const unsigned*>(p.mc + u.base + e));
      q.r[h] = __ldcs(reinterpret_cast<const unsigned*>(p.rc + u.base + e));
    }
  }
}

// FULL: the unit has all of its 256 elements.
template <bool FULL>
__device__ __forceinline__ void adam8_unit(const Adam8Regs& q, const AdamUnit& u, int lane, const Adam8Args& p,
                                           const AdamCoef& c) {
  const float lrwd = u.decay ? c.lrwd : 0.f;
  const float sr = scale_of(q.rs);
  const float km = scale_of(q.ms) * c.b1, kr = sr * sr * c.b2;  // powers of two: exact
  float m[8], r[8];
  float topm = 0.f, topr = 0.f;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float a[4], b[4];
    decode4(q.m[h], a);
    decode4(q.r[h], b);
    const float dv[4] = {q.d[h].x, q.d[h].y, q.d[h].z, q.d[h].w};
    float x[4] = {q.x[h].x, q.x[h].y, q.x[h].z, q.x[h].w};
    const int e = 128 * h + 4 * lane;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = 4 * h + k;
      float v;
      x[k] = adam_update(dv[k], x[k], a[k], km, b[k] * b[k], kr, m[i], v, r[i], c, lrwd);
      if (FULL || e + k < u.n) {
        topm = max_nan(topm, fabsf(m[i]));
        topr = max_nan(topr, r[i]);
      }
    }
    const long long at = u.base + e;
    const float4 xo = make_float4(x[0], x[1], x[2], x[3]);
    if (FULL || e + 4 <= u.n) {
      *reinterpret_cast<float4*>(p.params + at) = xo;
      if (p.low != nullptr) *reinterpret_cast<uint2*>(p.low + at) = bf16x4(xo);
    } else {
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (e + k < u.n) {
          p.params[at + k] = x[k];
          if (p.low != nullptr) p.low[at + k] = __bfloat16_as_ushort(__float2bfloat16_rn(x[k]));
        }
    }
  }
  const unsigned bm = scale_byte(__reduce_max_sync(0xffffffffu, __float_as_uint(topm)), kLowestM);
  const unsigned br = scale_byte(__reduce_max_sync(0xffffffffu, __float_as_uint(topr)), kLowestR);
  bool bigm, bigr;
  const float fm = code_factor(bm, bigm), fr = code_factor(br, bigr);
  if (bigm || bigr) {  // (the whole warp; 255 comes here too, and leaves codes that its scale of NaN makes NaN)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (bigm) m[i] = bm == 255u ? 0.f : __fmul_rz(m[i], 0x1p-120f);
      // (a positive r stays positive, however far below its block's largest)
      if (bigr) r[i] = br == 255u || r[i] == 0.f ? 0.f : fmaxf(__fmul_rz(r[i], 0x1p-120f), 0x1p-149f);
    }
  }
  if (lane == 0) { p.ms[u.block] = (unsigned char)bm; p.rs[u.block] = (unsigned char)br; }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int e = 128 * h + 4 * lane;
    // (units start at multiples of four elements, so the element's number is its vector's with k in the low bits)
    const unsigned seed = c.key ^ (unsigned)(u.base + e);
    unsigned cm[4], cr[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const unsigned w = mix32_open(seed ^ (unsigned)k), hi = w >> 16;  // random word: its halves are w ^ hi and hi
      const unsigned tm = __float_as_uint(__fmul_rz(m[4 * h + k], fm)) + (((w ^ hi) & 0xffffu) << 4);
      cm[k] = (tm & 0x80000000u) | ((tm << 4) & 0x7fffffffu);
      const float rk = r[4 * h + k];
      const float y = rk > 0.f ? fmaxf(__fmul_rz(rk, fr), 0x1p-129f) : 0.f;  // 2^-129: code 1
      cr[k] = (__float_as_uint(y) + (hi << 4)) << 4;
    }
    const unsigned wm = top_bytes(cm[0], cm[1], cm[2], cm[3]), wr = top_bytes(cr[0], cr[1], cr[2], cr[3]);
    const long long at = u.base + e;
    if (FULL || e + 4 <= u.n) {
      __stcs(reinterpret_cast<unsigned*>(p.mc + at), wm);
      __stcs(reinterpret_cast<unsigned*>(p.rc + at), wr);
    } else {
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (e + k < u.n) {
          p.mc[at + k] = (unsigned char)(wm >> (8 * k));
          p.rc[at + k] = (unsigned char)(wr >> (8 * k));
        }
    }
  }
}

template <bool ONE>
__global__ void __launch_bounds__(256, 5)
adamw_8bit_kernel(const FlatTile* __restrict__ tiles, const Adam8Args p, const AdamCoef* pre, long long* step,
                  const double* hyper, const float* factor, unsigned seed, int flags,
                  unsigned* ticket) {
  __shared__ AdamCoef sc;
  adam_enter<ONE>();
  const int lane = threadIdx.x & 31;
  const AdamUnit u = adam_unit(tiles, flags);
  Adam8Regs q;
  adam8_load(q, u, lane, p);
  AdamCoef c;
  if (!adam_begin<ONE>(c, &sc, pre, step, hyper, factor, seed)) return;
  if (u.n == kUnit) adam8_unit<true>(q, u, lane, p, c);
  else if (u.n > 0) adam8_unit<false>(q, u, lane, p, c);
  adam_finish<ONE>(step, ticket);
}

// One block: norm = sqrt(sum of the layers' squared norms, fp64, fixed order); factor = min(1, max_norm / norm), NaN where
// the norm is not finite.
__global__ void __launch_bounds__(256)
clip_factor_kernel(const double* n2_layers, int n_layers, double max_norm, float* factor, double* norm) {
  __shared__ double sm[8];
  await_previous();
  let_next_start();
  double acc = 0.0;
  for (int l = threadIdx.x; l < n_layers; l += 256) acc += n2_layers[l];
  acc = warp_sum(acc);
  if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = acc;
  __syncthreads();
  if (threadIdx.x == 0) {
    double s = 0.0;
    for (int i = 0; i < 8; ++i) s += sm[i];
    const double n = sqrt(s);
    *factor = !isfinite(n) ? __int_as_float(0x7fc00000) : n > max_norm ? (float)(max_norm / n) : 1.f;
    if (norm != nullptr) *norm = n;
  }
}

// Launches an update's kernel over every tile: kernel_one where its blocks all fit at once, else the coefficients' kernel
// and kernel_many, which starts beside it.
template <typename... Args>
static cudaError_t adam_launch(acc_ctx* ctx, int phase, int occupancy, void (*kernel_one)(Args...),
                               void (*kernel_many)(Args...), int64_t* step, const double* hyper, const float* factor,
                               unsigned seed, cudaStream_t s, Args... args) {
  const unsigned grid = (unsigned)ctx->plan.tiles.size() * kBlocksPerTile;
  const bool one = grid <= (unsigned)(occupancy * ctx->sm_count);
  if (one) {
    PhaseTimer pt(ctx, phase, s);
    return launch_early(kernel_one, grid, 256, s, args...);
  }
  cudaError_t e;
  {
    PhaseTimer pt(ctx, PH_ADAMW_COEF, s);
    e = launch_early(adamw_coef_kernel, 1, 32, s, reinterpret_cast<AdamCoef*>(ctx->d_status + kAdamCoefWord),
                     reinterpret_cast<long long*>(step), hyper, factor, seed);
  }
  PhaseTimer pt(ctx, phase, s);
  return e == cudaSuccess ? launch_early(kernel_many, grid, 256, s, args...) : e;
}

cudaError_t launch_adamw(acc_ctx* ctx, const float* d, float* params, float* m, float* v, int64_t* step,
                         const double* hyper, const float* factor, uint16_t* low, int flags, cudaStream_t s) {
  return adam_launch(ctx, PH_ADAMW, ctx->occ_adamw, adamw_kernel<true>, adamw_kernel<false>, step, hyper, factor, 0u, s,
                     (const FlatTile*)ctx->d_flat_tiles, d, params, m, v,
                     (const AdamCoef*)(ctx->d_status + kAdamCoefWord), reinterpret_cast<long long*>(step), hyper, factor,
                     (unsigned short*)low, flags, reinterpret_cast<unsigned*>(ctx->d_status + kAdamTicketWord));
}

cudaError_t launch_adamw_8bit(acc_ctx* ctx, const float* d, float* params, uint8_t* m_code, uint8_t* r_code,
                              uint8_t* m_scale, uint8_t* r_scale, int64_t* step, const double* hyper,
                              const float* factor, uint16_t* low, uint32_t seed, int flags, cudaStream_t s) {
  const Adam8Args p{d, params, m_code, r_code, m_scale, r_scale, low};
  return adam_launch(ctx, PH_ADAMW_8BIT, ctx->occ_adamw_8bit, adamw_8bit_kernel<true>, adamw_8bit_kernel<false>, step,
                     hyper, factor, (unsigned)seed, s, (const FlatTile*)ctx->d_flat_tiles, p,
                     (const AdamCoef*)(ctx->d_status + kAdamCoefWord), reinterpret_cast<long long*>(step), hyper, factor,
                     (unsigned)seed, flags, reinterpret_cast<unsigned*>(ctx->d_status + kAdamTicketWord));
}

// Once per context, at creation: how many blocks of the update's kernels an SM holds.
cudaError_t prepare_adamw(acc_ctx* ctx) {
  cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&ctx->occ_adamw, adamw_kernel<true>, 256, 0);
  if (e == cudaSuccess)
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&ctx->occ_adamw_8bit, adamw_8bit_kernel<true>, 256, 0);
  return e;
}

cudaError_t launch_clip_factor(acc_ctx* ctx, const double* n2_layers, double max_norm, float* factor, double* norm,
                               cudaStream_t s) {
  {
    PhaseTimer pt(ctx, PH_CLIP_FACTOR, s);
    return launch_early(clip_factor_kernel, 1, 256, s, n2_layers, ctx->cfg.n_layers, max_norm, factor, norm);
  }
}

}  // namespace acc
