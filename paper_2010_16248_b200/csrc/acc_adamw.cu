// AdamW update over the whole layer table, states in 32 bits or in 8 bits, and the clip factor it may be scaled by.
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "acc_internal.cuh"

namespace acc {

// The step's coefficients, worked out once per block in fp64 from the caller's doubles and the step count.
struct AdamCoef {
  float f;                 // factor on the gradient
  float b1, ob1, b2, ob2;  // beta1, 1 - beta1, beta2, 1 - beta2
  float lrwd;              // lr * weight_decay
  float size;              // lr / (1 - beta1^t)
  float rc2;               // 1 / sqrt(1 - beta2^t)
  float eps;
  unsigned key;            // of this step's random numbers (8-bit states)
};

// b^t by squaring: t has at most 63 bits, so the relative error stays under 126 * 2^-53.
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
__host__ __device__ __forceinline__ unsigned mix32(unsigned x) {
  x ^= x >> 16;
  x *= 0x7feb352du;
  x ^= x >> 15;
  x *= 0x846ca68bu;
  return x ^ (x >> 16);
}

// Two lanes take one power each; the result is valid for every thread after the next __syncthreads.
__device__ __forceinline__ void adam_coef(AdamCoef* c, const double* __restrict__ hyper, const long long* step, float f,
                                          unsigned seed) {
  if (threadIdx.x >= 2) return;
  const long long t = *step + 1;
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

// Every block has read the step count before it arrives here, so the last one may advance it; it also leaves the ticket
// at zero for the next call.
__device__ __forceinline__ void adam_finish(long long* step, unsigned* ticket) {
  __syncthreads();
  if (threadIdx.x == 0 && atomicAdd(ticket, 1u) == gridDim.x - 1) {
    *ticket = 0;
    *step += 1;
  }
}

// A factor that is not finite means that the gradient's norm was not: the call then changes nothing.
__device__ __forceinline__ float adam_factor(const float* factor, bool& skip) {
  const float f = factor != nullptr ? __ldg(factor) : 1.f;
  skip = !isfinite(f);
  return f;
}

// m, v (or r with v = r^2) in, new m, v out, in fp32; returns the new x.
__device__ __forceinline__ float adam_update(float d, float x, float& m, float& v, float& r, const AdamCoef& c,
                                             float lrwd) {
  const float g = c.f * d;
  m = fmaf(c.b1, m, c.ob1 * g);
  v = fmaf(c.b2, v, c.ob2 * (g * g));
  r = sqrtf(v);
  return fmaf(-c.size, m / fmaf(r, c.rc2, c.eps), fmaf(-lrwd, x, x));
}

__device__ __forceinline__ uint2 bf16x4(const float4 v) {
  const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x, v.y), hi = __floats2bfloat162_rn(v.z, v.w);
  return make_uint2(*reinterpret_cast<const unsigned*>(&lo), *reinterpret_cast<const unsigned*>(&hi));
}

// States in 32 bits: 16 B read and 12 B written per parameter, 15 operations: bound by HBM.  A block takes `share` elements
// of a tile, four at a time per thread.
__global__ void __launch_bounds__(256)
adamw_kernel(const DevLayer* __restrict__ layers, const Tile* __restrict__ tiles, int split, const float* __restrict__ d,
             float* __restrict__ params, float* __restrict__ ms, float* __restrict__ vs, long long* step,
             const double* __restrict__ hyper, const float* __restrict__ factor, unsigned short* __restrict__ low,
             int flags, unsigned* ticket) {
  __shared__ AdamCoef sc;
  bool skip;
  const float f = adam_factor(factor, skip);
  if (skip) return;
  const Tile t = tiles[blockIdx.x / split];
  const int share = kTile / split, first = (int)(blockIdx.x % split) * share;
  if (first < t.nelem) adam_coef(&sc, hyper, step, f, 0u);
  const DevLayer& L = layers[t.layer];
  const long long base = L.offset + t.elem0;
  const int end = min(first + share, t.nelem);
  const bool decay = L.kind == ACC_MATRIX || !(flags & ACC_ADAMW_NO_VECTOR_DECAY);
  __syncthreads();
  const AdamCoef c = sc;
  const float lrwd = decay ? c.lrwd : 0.f;
  for (int e = first + 4 * (int)threadIdx.x; e < end; e += 4 * 256) {
    // (layers start at multiples of four elements and the buffers end at one, so whole vectors are in bounds)
    const float4 dv = ld_stream4(d + base + e);
    float4 x = *reinterpret_cast<const float4*>(params + base + e);
    float4 m = ld_stream4(ms + base + e), v = ld_stream4(vs + base + e);
    float r;
    x.x = adam_update(dv.x, x.x, m.x, v.x, r, c, lrwd);
    x.y = adam_update(dv.y, x.y, m.y, v.y, r, c, lrwd);
    x.z = adam_update(dv.z, x.z, m.z, v.z, r, c, lrwd);
    x.w = adam_update(dv.w, x.w, m.w, v.w, r, c, lrwd);
    if (e + 4 <= end) {
      *reinterpret_cast<float4*>(params + base + e) = x;
      st_stream4(ms + base + e, m);
      st_stream4(vs + base + e, v);
      if (low != nullptr) *reinterpret_cast<uint2*>(low + base + e) = bf16x4(x);
    } else {
      const float xs[3] = {x.x, x.y, x.z}, mv[3] = {m.x, m.y, m.z}, vv[3] = {v.x, v.y, v.z};
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (e + k < end) {
          params[base + e + k] = xs[k];
          ms[base + e + k] = mv[k];
          vs[base + e + k] = vv[k];
          if (low != nullptr) low[base + e + k] = __bfloat16_as_ushort(__float2bfloat16_rn(xs[k]));
        }
    }
  }
  adam_finish(step, ticket);
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

// What a magnitude is multiplied by before its code is taken; 0 where every code of the block is 0.
__device__ __forceinline__ float inverse_scale(unsigned byte) {
  return byte == 0u || byte == 255u ? 0.f : __uint_as_float((254u - byte) << 23);
}

// e4m3 magnitude of y in [0, 256), rounded up with the probability that the cut bits stand for (16 random bits).
__device__ __forceinline__ unsigned encode(float y, unsigned rnd) {
  if (y >= 0.015625f) return ((__float_as_uint(y) + (rnd << 4)) >> 20) - (120u << 3);
  return (unsigned)floorf(fmaf(y, 512.f, (float)rnd * 0x1p-16f));
}

__device__ __forceinline__ float4 decode4(unsigned codes, float scale) {
  const __half2 lo(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(codes & 0xffffu), __NV_E4M3));
  const __half2 hi(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(codes >> 16), __NV_E4M3));
  const float2 a = __half22float2(lo), b = __half22float2(hi);
  return make_float4(a.x * scale, a.y * scale, b.x * scale, b.y * scale);
}

// A warp takes a block of 256 elements, eight per lane as two vectors of four (lane's first element 4 lane and 128 + 4
// lane), so that the block's largest magnitudes are one warp reduction away and every access is a full line.
// 16.03 B per parameter, bound by HBM.
__global__ void __launch_bounds__(256)
adamw_8bit_kernel(const DevLayer* __restrict__ layers, const Tile* __restrict__ tiles, int split,
                  const float* __restrict__ d, float* __restrict__ params, unsigned char* __restrict__ mc,
                  unsigned char* __restrict__ rc, unsigned char* __restrict__ msc, unsigned char* __restrict__ rsc,
                  long long* step, const double* __restrict__ hyper, const float* __restrict__ factor,
                  unsigned short* __restrict__ low, unsigned seed, int flags, unsigned* ticket) {
  __shared__ AdamCoef sc;
  bool skip;
  const float f = adam_factor(factor, skip);
  if (skip) return;
  const Tile t = tiles[blockIdx.x / split];
  const int share = kTile / split, first = (int)(blockIdx.x % split) * share;
  if (first < t.nelem) adam_coef(&sc, hyper, step, f, seed);
  const DevLayer& L = layers[t.layer];
  const long long base = L.offset + t.elem0;
  const long long block0 = L.adam_block0 + t.elem0 / ACC_ADAMW_BLOCK;
  const int end = min(first + share, t.nelem);
  const bool decay = L.kind == ACC_MATRIX || !(flags & ACC_ADAMW_NO_VECTOR_DECAY);
  __syncthreads();
  const AdamCoef c = sc;
  const float lrwd = decay ? c.lrwd : 0.f;
  const int lane = threadIdx.x & 31;
  for (int b0 = first + ACC_ADAMW_BLOCK * (int)(threadIdx.x >> 5); b0 < end; b0 += ACC_ADAMW_BLOCK * 8) {
    const long long blk = block0 + b0 / ACC_ADAMW_BLOCK;
    float dv[8], x[8], m[8], r[8];
    const float sm = scale_of(msc[blk]), sr = scale_of(rsc[blk]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int e = b0 + 128 * h + 4 * lane;
      float4 dd = make_float4(0.f, 0.f, 0.f, 0.f), xx = dd, mm = dd, rr = dd;
      if (e < end) {
        dd = ld_stream4(d + base + e);
        xx = *reinterpret_cast<const float4*>(params + base + e);
        mm = decode4(__ldcs(reinterpret_cast<const unsigned*>(mc + base + e)), sm);
        rr = decode4(__ldcs(reinterpret_cast<const unsigned*>(rc + base + e)), sr);
      }
      dv[4 * h] = dd.x; dv[4 * h + 1] = dd.y; dv[4 * h + 2] = dd.z; dv[4 * h + 3] = dd.w;
      x[4 * h] = xx.x; x[4 * h + 1] = xx.y; x[4 * h + 2] = xx.z; x[4 * h + 3] = xx.w;
      m[4 * h] = mm.x; m[4 * h + 1] = mm.y; m[4 * h + 2] = mm.z; m[4 * h + 3] = mm.w;
      r[4 * h] = rr.x; r[4 * h + 1] = rr.y; r[4 * h + 2] = rr.z; r[4 * h + 3] = rr.w;
    }
    unsigned topm = 0u, topr = 0u;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      float v = r[k] * r[k];
      x[k] = adam_update(dv[k], x[k], m[k], v, r[k], c, lrwd);
      if (b0 + 128 * (k >> 2) + 4 * lane + (k & 3) < end) {
        topm = max(topm, __float_as_uint(m[k]) & 0x7fffffffu);
        topr = max(topr, __float_as_uint(r[k]) & 0x7fffffffu);
      }
    }
    topm = __reduce_max_sync(0xffffffffu, topm);
    topr = __reduce_max_sync(0xffffffffu, topr);
    const unsigned bm = scale_byte(topm, kLowestM), br = scale_byte(topr, kLowestR);
    const float im = inverse_scale(bm), ir = inverse_scale(br);
    if (lane == 0) { msc[blk] = (unsigned char)bm; rsc[blk] = (unsigned char)br; }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int e = b0 + 128 * h + 4 * lane;
      unsigned cm = 0u, cr = 0u;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float mk = m[4 * h + k], rk = r[4 * h + k];
        const unsigned rnd = mix32(c.key ^ (unsigned)(base + e + k));
        unsigned qm = 0u, qr = 0u;
        if (bm != 255u) qm = encode(fabsf(mk) * im, rnd & 0xffffu) | (__float_as_uint(mk) >> 31 << 7);
        if (br != 255u) qr = encode(rk * ir, rnd >> 16);
        if (qr == 0u && rk > 0.f) qr = 1u;
        cm |= qm << (8 * k);
        cr |= qr << (8 * k);
      }
      const float4 xo = make_float4(x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]);
      if (e + 4 <= end) {
        *reinterpret_cast<float4*>(params + base + e) = xo;
        __stcs(reinterpret_cast<unsigned*>(mc + base + e), cm);
        __stcs(reinterpret_cast<unsigned*>(rc + base + e), cr);
        if (low != nullptr) *reinterpret_cast<uint2*>(low + base + e) = bf16x4(xo);
      } else {
#pragma unroll
        for (int k = 0; k < 3; ++k)
          if (e + k < end) {
            params[base + e + k] = x[4 * h + k];
            mc[base + e + k] = (unsigned char)(cm >> (8 * k));
            rc[base + e + k] = (unsigned char)(cr >> (8 * k));
            if (low != nullptr) low[base + e + k] = __bfloat16_as_ushort(__float2bfloat16_rn(x[4 * h + k]));
          }
      }
    }
  }
  adam_finish(step, ticket);
}

// One block: norm = sqrt(sum of the layers' squared norms, fp64, fixed order); factor = min(1, max_norm / norm), NaN where
// the norm is not finite.
__global__ void __launch_bounds__(256)
clip_factor_kernel(const double* __restrict__ n2_layers, int n_layers, double max_norm, float* __restrict__ factor,
                   double* __restrict__ norm) {
  __shared__ double sm[8];
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

// Blocks per tile: small tables are cut finer, so that every SM has work.
static int tile_split(int n_tiles, int sm_count, int most) {
  int split = 1;
  while (split < most && n_tiles * split < 4 * sm_count) split *= 2;
  return split;
}

cudaError_t launch_adamw(acc_ctx* ctx, const float* d, float* params, float* m, float* v, int64_t* step,
                         const double* hyper, const float* factor, uint16_t* low, int flags, cudaStream_t s) {
  const int nt = (int)ctx->plan.tiles.size(), split = tile_split(nt, ctx->sm_count, 8);
  {
    PhaseTimer pt(ctx, PH_ADAMW, s);
    adamw_kernel<<<nt * split, 256, 0, s>>>(ctx->d_layers, ctx->d_tiles, split, d, params, m, v,
                                            reinterpret_cast<long long*>(step), hyper, factor, low, flags,
                                            reinterpret_cast<unsigned*>(ctx->d_status + kAdamTicketWord));
  }
  return cudaGetLastError();
}

cudaError_t launch_adamw_8bit(acc_ctx* ctx, const float* d, float* params, uint8_t* m_code, uint8_t* r_code,
                              uint8_t* m_scale, uint8_t* r_scale, int64_t* step, const double* hyper,
                              const float* factor, uint16_t* low, uint32_t seed, int flags, cudaStream_t s) {
  const int nt = (int)ctx->plan.tiles.size(), split = tile_split(nt, ctx->sm_count, 4);
  {
    PhaseTimer pt(ctx, PH_ADAMW_8BIT, s);
    adamw_8bit_kernel<<<nt * split, 256, 0, s>>>(ctx->d_layers, ctx->d_tiles, split, d, params, m_code, r_code, m_scale,
                                                 r_scale, reinterpret_cast<long long*>(step), hyper, factor, low, seed,
                                                 flags, reinterpret_cast<unsigned*>(ctx->d_status + kAdamTicketWord));
  }
  return cudaGetLastError();
}

cudaError_t launch_clip_factor(acc_ctx* ctx, const double* n2_layers, double max_norm, float* factor, double* norm,
                               cudaStream_t s) {
  {
    PhaseTimer pt(ctx, PH_CLIP_FACTOR, s);
    clip_factor_kernel<<<1, 256, 0, s>>>(n2_layers, ctx->cfg.n_layers, max_norm, factor, norm);
  }
  return cudaGetLastError();
}

}  // namespace acc
