// Log probabilities of given tokens from a row of logits each, with the entropy and the likeliest tokens of the row; and the
// gradient of both into the logits.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <algorithm>

#include "acc_internal.cuh"

namespace acc {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// 2^x, 2 ulp; 0 below 2^-126.
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The larger of two; NaN when one of them is.
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
// The same of two pairs of bf16, of the lanes of a warp.
__device__ __forceinline__ unsigned max2(unsigned a, unsigned b) {
  unsigned y;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
  return y;
}
__device__ __forceinline__ float max_warp(float a) {
  float y;
  asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(a));
  return y;
}
// Two fp32 operations at once.
union Pair { float2 f; unsigned long long u; };
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  Pair x, y, z, r;
  x.f = a; y.f = b; z.f = c;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.u) : "l"(x.u), "l"(y.u), "l"(z.u));
  return r.f;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  Pair x, y, r;
  x.f = a; y.f = b;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.u) : "l"(x.u), "l"(y.u));
  return r.f;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  Pair x, y, r;
  x.f = a; y.f = b;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.u) : "l"(x.u), "l"(y.u));
  return r.f;
}
constexpr float kMinusInf = -__builtin_huge_valf();
__device__ __forceinline__ float not_a_number() { return __int_as_float(0x7fffffff); }

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

// Eight neighbouring values as loaded: 16 bytes of bf16, 32 of fp32.
template <typename T> struct Eight;
template <> struct Eight<__nv_bfloat16> {
  uint4 a;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void fill_minus_inf() { a = make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
  // The largest of the eight, NaN when one of them is; and the eight as pairs, none below `least`.
  __device__ __forceinline__ float largest() const {
    const unsigned m = max2(max2(a.x, a.y), max2(a.z, a.w));
    return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
  }
  __device__ __forceinline__ void pairs(float2* v, float least) const {
    const unsigned l = __float_as_uint(least) >> 16, l2 = l | l << 16;
    const unsigned w[4] = {max2(a.x, l2), max2(a.y, l2), max2(a.z, l2), max2(a.w, l2)};
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = make_float2(__uint_as_float(w[k] << 16), __uint_as_float(w[k] & 0xffff0000u));
  }
  __device__ __forceinline__ void get(float* v) const {
    const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = __uint_as_float(w[k] << 16);
      v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void put(const float* v) {
    unsigned w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
      w[k] = *reinterpret_cast<const unsigned*>(&h);
    }
    a = make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = a; }
};
template <> struct Eight<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const float4*>(p);
    b = *reinterpret_cast<const float4*>(p + 4);
  }
  __device__ __forceinline__ void fill_minus_inf() { a = b = make_float4(kMinusInf, kMinusInf, kMinusInf, kMinusInf); }
  __device__ __forceinline__ float largest() const {
    return max_nan(max_nan(max_nan(a.x, a.y), max_nan(a.z, a.w)), max_nan(max_nan(b.x, b.y), max_nan(b.z, b.w)));
  }
  __device__ __forceinline__ void pairs(float2* v, float least) const {
    v[0] = make_float2(max_nan(a.x, least), max_nan(a.y, least)); v[1] = make_float2(max_nan(a.z, least), max_nan(a.w, least));
    v[2] = make_float2(max_nan(b.x, least), max_nan(b.y, least)); v[3] = make_float2(max_nan(b.z, least), max_nan(b.w, least));
  }
  __device__ __forceinline__ void get(float* v) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
  __device__ __forceinline__ void put(const float* v) {
    a = make_float4(v[0], v[1], v[2], v[3]);
    b = make_float4(v[4], v[5], v[6], v[7]);
  }
  __device__ __forceinline__ void store(float* p) const {
    *reinterpret_cast<float4*>(p) = a;
    *reinterpret_cast<float4*>(p + 4) = b;
  }
};

// A row's elements as groups of eight that start on a boundary of eight elements, and up to seven single ones on either side:
// rows may begin at any element, so every row length and stride takes wide loads.
struct RowSpan {
  int head, groups, size;  // elements before the first group; groups; all elements
  template <typename T> __device__ __forceinline__ static RowSpan of(const T* row, int size) {
    const int ahead = (int)((8 - (reinterpret_cast<uintptr_t>(row) / sizeof(T)) % 8) % 8);
    const int head = ahead < size ? ahead : size;
    return {head, (size - head) / 8, size};
  }
  // Index of single element s of 0..13, or -1: seven places before the groups, seven behind.
  __device__ __forceinline__ int single(int s) const {
    if (s < 7) return s < head ? s : -1;
    const int i = head + 8 * groups + s - 7;
    return s < 14 && i < size ? i : -1;
  }
};

// The running statistics of a set of logits z with largest m: s = sum 2^d, t = sum 2^d d.  d = z c2 - ref(m), one rounding, with
// c2 = scale log2(e) and ref(m) = m c2 rounded: the largest logit's own d is then what ref(m) left out, left(m), not 0, and the
// row's end puts that right.  It is half a step of m c2, 2^-5 at most below the limit of 2^20; from there on, where it would grow
// until 2^d is no number of use, d = (z - m) c2.  Sums that count from unlike references are brought together by their lefts.
// A distance below -200 counts as -200, where 2^d is 0: -inf and masks of any size then add nothing, not 0 * inf.
struct Scale {
  float c2, limit, least;  // |m| below limit has a ref; a logit below `least` counts as `least`: its 2^d is 0, and d finite
  // (`least` is finite too.  At a scale so small that the type's lowest value may have a share of the row nothing is near: each d
  // is bounded itself, and -inf alone has none.)
  static Scale of(float scale) {
    const float c2 = scale * kLog2e;
    return {c2, c2 < 0x1p-100f ? 0.f : 0x1p20f / c2, std::max(-0x1p120f / c2, -0x1.fffffep127f)};
  }
  __device__ __forceinline__ bool near(float m) const { return fabsf(m) < limit; }
  __device__ __forceinline__ float ref(float m) const { return __fmul_rn(m, c2); }  // (never part of an fma)
  __device__ __forceinline__ float left(float m) const { return near(m) ? fmaf(m, c2, -ref(m)) : 0.f; }
  __device__ __forceinline__ float distance(float z, float m) const {
    return fmaxf(near(z) && near(m) ? ref(z) - ref(m) : fmaf(z - m, c2, left(m) - left(z)), -200.f);
  }
};
struct Stats { float m, s, t; };

// The sum of s and t over a warp, from the lanes' own m to the largest.
__device__ __forceinline__ Stats merge_warp(const Stats& a, const Scale& k) {
  const float m = max_warp(a.m), d = k.distance(a.m, m), f = exp2_fast(d);
  return {m, warp_sum(f * a.s), warp_sum(f * fmaf(a.s, d, a.t))};
}
__device__ __forceinline__ Stats merge(const Stats& a, const Stats& b, const Scale& k) {
  const float m = max_nan(a.m, b.m), da = k.distance(a.m, m), db = k.distance(b.m, m);
  const float fa = exp2_fast(da), fb = exp2_fast(db);
  return {m, fa * a.s + fb * b.s, fa * fmaf(a.s, da, a.t) + fb * fmaf(b.s, db, b.t)};
}

// The same while a thread adds to it: two sums of each, for two fp32 operations at once.
template <bool ENT> struct Running {
  float m = kMinusInf;
  float2 s = {0.f, 0.f}, t = {0.f, 0.f};
  // To a largest of at least `top` (NaN when something in the row is).
  __device__ __forceinline__ void raise(float top, const Scale& k) {
    if (top <= m) return;
    const float next = max_nan(m, top), d = k.distance(m, next), f = exp2_fast(d);
    if (ENT) t = {f * fmaf(s.x, d, t.x), f * fmaf(s.y, d, t.y)};
    s = {f * s.x, f * s.y};
    m = next;
  }
  __device__ __forceinline__ void add_far(float z, const Scale& k) {
    const float d = fmaxf((z - m) * k.c2, -200.f), e = exp2_fast(d);
    s.x += e;
    if (ENT) t.x = fmaf(e, d, t.x);
  }
  __device__ __forceinline__ void add_one(float z, const Scale& k) {
    raise(z, k);
    if (!k.near(m)) return add_far(z, k);
    const float d = fmaf(fmaxf(z, k.least), k.c2, -k.ref(m)), e = exp2_fast(d);
    s.x += e;
    if (ENT) t.x = fmaf(e, d, t.x);
  }
  // N groups of eight values, of which the first `count` are there and the others -inf.
  template <int N, typename T> __device__ __forceinline__ void add(const Eight<T> (&x)[N], int count, const Scale& k) {
    float top = x[0].largest();
#pragma unroll
    for (int i = 1; i < N; ++i) top = max_nan(top, x[i].largest());
    raise(top, k);
    if (k.near(m)) {
      const float2 c = {k.c2, k.c2}, r = {-k.ref(m), -k.ref(m)};
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (i >= count) break;
        float2 z[4];
        x[i].pairs(z, k.least);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 d = fma2(z[j], c, r), e = {exp2_fast(d.x), exp2_fast(d.y)};
          s = add2(s, e);
          if (ENT) t = fma2(e, d, t);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float z[8];
        x[i].get(z);
#pragma unroll
        for (int j = 0; j < 8; ++j) add_far(z[j], k);
      }
    }
  }
};

// Statistics of this thread's share of a row: groups first + own, first + own + stride, ... below last, and single elements.
template <typename T, bool ENT>
__device__ __forceinline__ Stats row_share(const T* row, const RowSpan& r, int first, int last, int own, int stride,
                                           int single, const Scale& c) {
  constexpr int kBatch = 4;
  Running<ENT> a;
  const T* p = row + r.head + 8ll * (first + own);
  int left = (last - first - own + stride - 1) / stride;  // groups of this thread that are not loaded
  auto load = [&](Eight<T> (&x)[kBatch]) {
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      if (k < left) x[k].load(p + 8 * k * stride);
      else x[k].fill_minus_inf();
    }
    p += 8ll * kBatch * stride;
    left -= kBatch;
  };
  while (left > 0) {
    Eight<T> x[kBatch];
    load(x);
    a.add(x, left >= 0 ? kBatch : left + kBatch, c);
  }
  const int i = r.single(single);
  if (i >= 0) a.add_one(to_float(row[i]), c);
  return {a.m, a.s.x + a.s.y, a.t.x + a.t.y};
}

// ---- the likeliest tokens ---------------------------------------------------------------------------------------
// Tokens in order of falling logit, then of rising index, as one integer: larger means earlier.  -0 equals +0.
using Key = unsigned long long;
__device__ __forceinline__ Key make_key(float z, int index) {
  const unsigned b = __float_as_uint(z + 0.f);
  return (Key)((b >> 31) ? ~b : b | 0x80000000u) << 32 | (unsigned)~index;
}
__device__ __forceinline__ float key_logit(Key k) {
  const unsigned u = (unsigned)(k >> 32);
  return __uint_as_float((u >> 31) ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ int key_index(Key k) { return (int)~(unsigned)k; }

struct LogArgs {
  const void* logits;
  const void* tokens;   // nullptr: every row counts and none has a given token
  int token64;
  long long n, ld;
  int vocab;
  float scale;          // of the logits
  Scale c;
  float* logp;          // each output may be nullptr
  float2* norm;
  float* entropy;
  int top;
  int* top_index;
  float* top_logp;
  int* status;
  int parts_log2;       // blocks per row
};

// The given token of a row: its index; -1 where none was asked for; -2 for a row that is not to be read (a negative token
// pads the batch, one beyond the vocabulary is reported).
__device__ __forceinline__ int given_token(const void* tokens, int token64, long long row, int vocab, int* status) {
  if (tokens == nullptr) return -1;
  const long long t = token64 ? static_cast<const long long*>(tokens)[row] : static_cast<const int*>(tokens)[row];
  if (t < 0) return -2;
  if (t >= vocab) {
    if (status != nullptr) atomicCAS(status, 0, ACC_EINDEX);
    return -2;
  }
  return (int)t;
}

// What a row's owner writes once it has the row's statistics; returns log S, NaN for a row with a NaN or +inf.
__device__ __forceinline__ float finish_row(const LogArgs& a, long long row, const Stats& s, int token, float given) {
  const Scale& k = a.c;
  // (s and t count from ref(m): the distance of m from it enters log S, and cancels in the entropy)
  float log_s = logf(s.s), entropy = log_s - s.t / s.s * kLn2;
  log_s -= k.left(s.m) * kLn2;
  if (s.m == kMinusInf) log_s = entropy = 0.f;  // nothing to choose from
  if (!(s.m < -kMinusInf)) log_s = entropy = not_a_number();
  if (a.norm != nullptr) a.norm[row] = make_float2(s.m, log_s);
  if (a.entropy != nullptr) a.entropy[row] = entropy;
  if (a.logp != nullptr) a.logp[row] = given == kMinusInf ? (log_s == log_s ? kMinusInf : log_s) : (given - s.m) * a.scale - log_s;
  return log_s;
}
__device__ __forceinline__ void skip_row(const LogArgs& a, long long row, int lane, int lanes) {
  if (lane == 0) {
    if (a.norm != nullptr) a.norm[row] = make_float2(0.f, 0.f);
    if (a.entropy != nullptr) a.entropy[row] = 0.f;
    if (a.logp != nullptr) a.logp[row] = 0.f;
  }
  for (int k = lane; k < a.top; k += lanes) {
    if (a.top_index != nullptr) a.top_index[row * a.top + k] = -1;
    if (a.top_logp != nullptr) a.top_logp[row * a.top + k] = kMinusInf;
  }
}
__device__ __forceinline__ void write_top(const LogArgs& a, long long row, int k, Key key, float m, float log_s) {
  const bool fine = log_s == log_s, some = fine && key != 0;
  if (a.top_index != nullptr) a.top_index[row * a.top + k] = some ? key_index(key) : -1;
  if (a.top_logp != nullptr)
    a.top_logp[row * a.top + k] = some ? (key_logit(key) - m) * a.scale - log_s : fine ? kMinusInf : not_a_number();
}

constexpr int kGroupMaxima = 64, kCandidates = 1024;
static_assert(kGroupMaxima >= ACC_LOGPROBS_MAX_TOP, "as many maxima as alternatives");

template <int THREADS> struct RowShared {
  Stats stats[THREADS / 32];
  Stats all;
  float maxima[kGroupMaxima];
  float bar;                     // a bound that at least `top` logits of the share reach
  int count;
  unsigned char owner[THREADS / 32][32];  // of each warp: the lanes whose shares are read again
  Key best[ACC_LOGPROBS_MAX_TOP];
  Key list[kCandidates];
};

// list[0 .. count) -> best[0 .. top), in order; keys are distinct, so the order in which the list was filled does not matter.
template <int THREADS> __device__ __forceinline__ void rank_list(RowShared<THREADS>& sh, int count, int top) {
  if ((int)threadIdx.x < top) sh.best[threadIdx.x] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < count; i += THREADS) {
    const Key own = sh.list[i];
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < count; ++j) rank += sh.list[j] > own;
    if (rank < top) sh.best[rank] = own;
  }
  __syncthreads();
}

// Calls f(z, index) for every element of this thread's share of [first, last) groups and the singles.
template <typename T, typename F>
__device__ __forceinline__ void each_value(const T* row, const RowSpan& r, int first, int last, int own, int stride, int single,
                                           F f) {
  for (int g = first + own; g < last; g += stride) {
    Eight<T> x;
    x.load(row + r.head + 8ll * g);
    float z[8];
    x.get(z);
#pragma unroll
    for (int k = 0; k < 8; ++k) f(z[k], r.head + 8 * g + k);
  }
  const int i = r.single(single);
  if (i >= 0) f(to_float(row[i]), i);
}

// The `top` largest keys of a block's share of a row into sh.best.  Every thread knows the largest logit of its own share; the
// `top`-th largest of 64 such maxima, of neighbouring threads, is a bar that at least `top` logits reach, and only the shares of
// threads whose maximum reaches it are read again, by whole warps: for top = 20 about 25.  Ties at the bar may be many
// (a mask of the type's lowest value leaves them): then those above it are taken and those at it searched in order of index.
template <typename T, int THREADS>
__device__ __forceinline__ void select_top(RowShared<THREADS>& sh, const T* row, const RowSpan& r, int first, int last, int single,
                                           float own_max, int top) {
  constexpr int kMaximumOf = THREADS / kGroupMaxima;
  const int tid = threadIdx.x, lane = tid & 31;
  float m = own_max;
#pragma unroll
  for (int o = 1; o < kMaximumOf; o *= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (tid % kMaximumOf == 0) sh.maxima[tid / kMaximumOf] = m;
  if (tid == 0) { sh.bar = kMinusInf; sh.count = 0; }
  __syncthreads();
  if (tid < kGroupMaxima) {
    const float own = sh.maxima[tid];
    int rank = 0;
#pragma unroll 16
    for (int j = 0; j < kGroupMaxima; ++j) rank += sh.maxima[j] > own || (sh.maxima[j] == own && j < tid);
    if (rank == top - 1) sh.bar = own;
  }
  __syncthreads();
  const float bar = sh.bar;
  auto push = [&](float z, int index) {
    const int at = atomicAdd(&sh.count, 1);
    if (at < kCandidates) sh.list[at] = make_key(z, index);
  };
  // (-inf is no alternative, whatever the bar)
  auto gather = [&](bool above) {
    auto take = [&](float z) { return above ? z > bar : z >= bar && z > kMinusInf; };
    const unsigned owners = __ballot_sync(0xffffffffu, take(own_max));
    if (take(own_max)) sh.owner[tid >> 5][__popc(owners & ((1u << lane) - 1))] = (unsigned char)lane;
    __syncwarp();
    // the owners' groups as one list, a lane each, four at a time
    const int each = (last - first + THREADS - 1) / THREADS, items = __popc(owners) * each;
    constexpr int kTogether = 4;
    for (int i = lane; i < items; i += 32 * kTogether) {
      Eight<T> x[kTogether];
      int group[kTogether];
#pragma unroll
      for (int k = 0; k < kTogether; ++k) {
        const int item = i + 32 * k, owner = item < items ? item / each : 0;
        group[k] = item < items ? first + (tid & ~31) + sh.owner[tid >> 5][owner] + (item - owner * each) * THREADS : last;
        if (group[k] < last) x[k].load(row + r.head + 8ll * group[k]);
      }
#pragma unroll
      for (int k = 0; k < kTogether; ++k) {
        if (group[k] >= last || !take(x[k].largest())) continue;
        float z[8];
        x[k].get(z);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (take(z[j])) push(z[j], r.head + 8 * group[k] + j);
      }
    }
    const int i = r.single(single);
    if (i >= 0) {
      const float z = to_float(row[i]);
      if (take(z)) push(z, i);
    }
    __syncthreads();
    return sh.count;
  };
  int count = gather(false);
  if (count > kCandidates) {
    __syncthreads();
    if (tid == 0) sh.count = 0;
    __syncthreads();
    count = gather(true);
    constexpr int kSearch = 32;  // groups of a step of the search: as many elements as the list keeps free
    if (count + 8 * kSearch + 14 <= kCandidates) {
      // at the bar, in order of index: the singles before the groups, the groups, the singles behind them
      for (int g = first; count < top && g < last; g += kSearch) {
        __syncthreads();
        each_value(row, r, g, min(last, g + kSearch), tid, THREADS, g == first && tid < 7 ? single : -1,
                   [&](float z, int i) { if (z == bar) push(z, i); });
        __syncthreads();
        count = sh.count;
      }
      __syncthreads();
      if (count < top && tid >= 7) {
        const int i = r.single(single);
        if (i >= 0 && to_float(row[i]) == bar) push(bar, i);
      }
      __syncthreads();
      count = sh.count;
    } else {
      // a share with more than that above its bar: one pass for each of the `top`
      Key below = ~0ull;
      for (int k = 0; k < top; ++k) {
        Key best = 0;
        each_value(row, r, first, last, tid, THREADS, single, [&](float z, int i) {
          const Key key = make_key(z, i);
          if (z > kMinusInf && key < below && key > best) best = key;
        });
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
        __syncthreads();
        if (lane == 0) sh.list[tid >> 5] = best;
        __syncthreads();
        best = 0;
        for (int j = 0; j < THREADS / 32; ++j) best = max(best, sh.list[j]);
        if (tid == 0) sh.best[k] = best;
        below = best;
      }
      __syncthreads();
      return;
    }
  }
  rank_list(sh, count, top);
}

// A row per cluster of `parts` blocks: each takes a stretch of its groups, and the first joins them over the cluster's shared
// memory.  One pass over the logits.  5600 rows of 33278, a tenth padding, fp32 85 % and bf16 82 % of the memory's rate (62 us,
// 336 MB): the exponentials alone keep their unit busy half of that time, and a row's end (two joins, a logarithm) is not hidden
// by other rows altogether.  The alternatives cost a second look at a tenth of the logits, in pieces of 16 bytes: 2048 rows of
// 131071 with 20 take 117 us where 87 do without, and read 640 MB where 483 are there.  (Tried: a bar from a row's first quarter
// and a list of what passes it afterwards, 134 us; the largest of every 2 KB kept and only those read again, 114 us but 5 us
// more on rows of a few thousand.)
template <typename T, bool ENT, bool TOP, int THREADS>
__global__ void __launch_bounds__(THREADS, (TOP ? 1280 : sizeof(T) == 2 ? 1536 : 1024) / THREADS) logprobs_kernel(const LogArgs a) {
  namespace cg = cooperative_groups;
  __shared__ __align__(16) RowShared<THREADS> sh;
  await_previous();
  let_next_start();
  const int parts = 1 << a.parts_log2, tid = threadIdx.x;
  const long long row = blockIdx.x >> a.parts_log2;
  const int part = blockIdx.x & (parts - 1);
  const int token = given_token(a.tokens, a.token64, row, a.vocab, tid == 0 && part == 0 ? a.status : nullptr);
  if (token == -2) {
    if (part == 0) skip_row(a, row, tid, THREADS);
    return;
  }
  const T* z = static_cast<const T*>(a.logits) + row * a.ld;
  const RowSpan r = RowSpan::of(z, a.vocab);
  const int first = (int)((long long)r.groups * part >> a.parts_log2);
  const int last = (int)((long long)r.groups * (part + 1) >> a.parts_log2);
  // the singles before the groups belong to the first part, those behind them to the last
  const int single = tid < 7 ? (part == 0 ? tid : -1) : tid < 14 && part == parts - 1 ? tid : -1;
  const Scale& c = a.c;
  const Stats own = row_share<T, ENT>(z, r, first, last, tid, THREADS, single < 0 ? 14 : single, c);
  {
    const Stats w = merge_warp(own, c);
    if ((tid & 31) == 0) sh.stats[tid >> 5] = w;
  }
  __syncthreads();
  if (tid < 32) {
    Stats w = tid < THREADS / 32 ? sh.stats[tid] : Stats{kMinusInf, 0.f, 0.f};
    w = merge_warp(w, c);
    if (tid == 0) sh.all = w;
  }
  if (TOP) select_top(sh, z, r, first, last, single < 0 ? 14 : single, own.m, a.top);
  __syncthreads();
  Stats all = sh.all;
  if (parts > 1) {
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    if (part == 0) {
      for (int p = 1; p < parts; ++p) all = merge(all, *cluster.map_shared_rank(&sh.all, p), c);
      if (TOP) {
        for (int i = tid; i < parts * a.top; i += THREADS) sh.list[i] = cluster.map_shared_rank(sh.best, i / a.top)[i % a.top];
        __syncthreads();
        // (empty places are zeros: behind every key, and equal, so none of them is ranked below `top` in place of a key)
        rank_list(sh, parts * a.top, a.top);
      }
    }
    cluster.sync();
    if (part != 0) return;
  }
  float log_s = 0.f;
  if (tid < 32) {
    if (tid == 0) log_s = finish_row(a, row, all, token, token >= 0 ? to_float(z[token]) : 0.f);
    log_s = __shfl_sync(0xffffffffu, log_s, 0);
    if (TOP && tid < a.top) write_top(a, row, tid, sh.best[tid], all.m, log_s);
  }
}

// A row per warp.  The alternatives as above, with a bar from the 32 lanes' maxima, below which two logits in three stay.
constexpr int kWarpList = 192;
template <typename T, bool ENT, bool TOP>
__global__ void __launch_bounds__(256) logprobs_warp_kernel(const LogArgs a) {
  __shared__ __align__(16) Key lists[TOP ? 8 : 1][kWarpList];
  __shared__ Key bests[TOP ? 8 : 1][ACC_LOGPROBS_MAX_TOP];
  __shared__ int counts[8];
  await_previous();
  let_next_start();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long row = (long long)blockIdx.x * 8 + warp;
  if (row >= a.n) return;
  const int token = given_token(a.tokens, a.token64, row, a.vocab, lane == 0 ? a.status : nullptr);
  if (token == -2) {
    skip_row(a, row, lane, 32);
    return;
  }
  const T* z = static_cast<const T*>(a.logits) + row * a.ld;
  const RowSpan r = RowSpan::of(z, a.vocab);
  const Scale& c = a.c;
  const Stats own = row_share<T, ENT>(z, r, 0, r.groups, lane, 32, lane, c), all = merge_warp(own, c);
  float log_s = 0.f;
  if (lane == 0) log_s = finish_row(a, row, all, token, token >= 0 ? to_float(z[token]) : 0.f);
  if (!TOP) return;
  log_s = __shfl_sync(0xffffffffu, log_s, 0);
  int above = 0;
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    const float m = __shfl_sync(0xffffffffu, own.m, j);
    above += m > own.m || (m == own.m && j < lane);
  }
  const unsigned at_bar = __ballot_sync(0xffffffffu, above == a.top - 1);
  const float bar = __shfl_sync(0xffffffffu, own.m, at_bar != 0 ? __ffs(at_bar) - 1 : 0);  // (a row with NaN may have none)
  if (lane == 0) counts[warp] = 0;
  bests[warp][lane] = 0;
  __syncwarp();
  auto take = [&](float v) { return v >= bar && v > kMinusInf; };
  auto push = [&](float v, int i) {
    const int at = atomicAdd(&counts[warp], 1);
    if (at < kWarpList) lists[warp][at] = make_key(v, i);
  };
  for (int g = lane; g < r.groups; g += 32) {
    Eight<T> x;
    x.load(z + r.head + 8ll * g);
    if (!take(x.largest())) continue;
    float v[8];
    x.get(v);
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (take(v[k])) push(v[k], r.head + 8 * g + k);
  }
  const int single = r.single(lane);
  if (single >= 0 && take(to_float(z[single]))) push(to_float(z[single]), single);
  __syncwarp();
  const int count = counts[warp];
  if (count <= kWarpList) {
    for (int i = lane; i < count; i += 32) {
      const Key key = lists[warp][i];
      int rank = 0;
#pragma unroll 8
      for (int j = 0; j < count; ++j) rank += lists[warp][j] > key;
      if (rank < a.top) bests[warp][rank] = key;
    }
  } else {
    // one after another: a lane's best key below its last; only the lane whose key was taken looks again
    auto next = [&](Key below) {
      Key best = 0;
      each_value(z, r, 0, r.groups, lane, 32, lane, [&](float v, int i) {
        const Key key = make_key(v, i);
        if (v > kMinusInf && key < below && key > best) best = key;
      });
      return best;
    };
    Key mine = next(~0ull);
    for (int k = 0; k < a.top; ++k) {
      Key best = mine;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
      if (lane == 0) bests[warp][k] = best;
      if (best != 0 && mine == best) mine = next(best);
    }
  }
  __syncwarp();
  if (lane < a.top) write_top(a, row, lane, bests[warp][lane], all.m, log_s);
}

// Rows up to the first length take a warp each, and up to the second where that leaves every SM its warps: 65536 rows of 2000 in
// bf16 53 us, with a block of 128 threads each 105; 16384 of 8000 51 and 53.
constexpr int kWarpVocab = 1024, kWarpVocabMany = 8192;
static bool warp_rows(const acc_ctx* ctx, long long n, int vocab) {
  return vocab <= kWarpVocab || (vocab <= kWarpVocabMany && n >= 32ll * ctx->sm_count);
}

// Blocks per row: as many as keep the GPU busy when there are few rows, each with a stretch worth a block's start.  One row of
// 33278 in fp32 with five alternatives on the GPU: 7.0 us in eight parts, 11.2 in one; 64 rows 8.7 and 11.7; 150 rows 10.4 in two
// and 12.0 in one; 600 rows of 131071 with 20: 48 us in one, 58 in eight.
static int row_parts_log2(const acc_ctx* ctx, long long n, int vocab) {
  int p = 0;
  while (p < 3 && (n << (p + 1)) <= 4ll * ctx->sm_count && vocab >> (p + 1) >= 2048) ++p;
  return p;
}

cudaError_t launch_token_logprobs(acc_ctx* ctx, const void* logits, bool bf16, long long n, int vocab, long long ld,
                                  const void* tokens, bool tok64, float scale, float* logp, float* norm, float* entropy,
                                  int top, int* top_index, float* top_logp, cudaStream_t s) {
  LogArgs a{logits, tokens, tok64, n, ld, vocab, scale, Scale::of(scale), logp, reinterpret_cast<float2*>(norm), entropy, top,
            top_index, top_logp, ctx->d_status, 0};
  PhaseTimer pt(ctx, PH_LOGPROBS, s);
  auto go = [&](auto t) {
    using T = decltype(t);
    const bool ent = entropy != nullptr;
    if (warp_rows(ctx, n, vocab)) {
      auto* kernel = top > 0 ? (ent ? logprobs_warp_kernel<T, true, true> : logprobs_warp_kernel<T, false, true>)
                             : (ent ? logprobs_warp_kernel<T, true, false> : logprobs_warp_kernel<T, false, false>);
      return launch_early(kernel, (unsigned)((n + 7) / 8), 256, s, a);
    }
    a.parts_log2 = row_parts_log2(ctx, n, vocab);
    auto block = [&](auto threads) {
      constexpr int N = decltype(threads)::value;
      auto* kernel = top > 0 ? (ent ? logprobs_kernel<T, true, true, N> : logprobs_kernel<T, false, true, N>)
                             : (ent ? logprobs_kernel<T, true, false, N> : logprobs_kernel<T, false, false, N>);
      return launch_early_as(kernel, (unsigned)(n << a.parts_log2), N, 0, 1 << a.parts_log2, s, a);
    };
    // 5600 rows of 33278 in bf16: 70 us with 128 threads a row and 73 with 256 (more rows' ends overlap); 2048 rows of 131071:
    // 101 us and 89 (fewer rows are left for the last wave).
    return vocab < 65536 ? block(std::integral_constant<int, 128>()) : block(std::integral_constant<int, 256>());
  };
  return bf16 ? go(__nv_bfloat16()) : go(0.f);
}

// ---- gradient ----------------------------------------------------------------------------------------------------
// dz_j = scale [ g (1[j = token] - p_j) - h p_j (log p_j + H) ]  with  log p_j = (z_j - max) scale - log S.  5600 rows of 33278 in
// bf16, a tenth padding: 112 us, 6.3 TB/s of reading and writing.

struct LogGradArgs {
  const void* logits;
  const void* tokens;
  int token64;
  long long n, ld, ld_out;
  int vocab;
  float scale;
  const float2* norm;
  const float* g_logp;     // nullptr: 0
  const float* g_entropy;  // nullptr: 0
  const float* entropy;
  int g_step;              // elements between the rows' values of g_logp: 0 when one serves all
  int h_step;
  void* out;
  int* status;
  int segments, stretch;   // blocks per row, groups of eight (elements, on the narrow way) of a block
};

// What one row's elements need: dz = p (w0 + w1 log2 p), with log2 p = (z - m) c2 - log2_s.
struct RowGrad {
  float m, c2, log2_s, w0, w1, g;
  template <bool ENT> __device__ __forceinline__ float at(float z) const {
    float l = fmaf(z - m, c2, -log2_s);
    if (ENT) l = fmaxf(l, -200.f);  // 2^-200 is 0, and so is its product
    return exp2_fast(l) * (ENT ? fmaf(w1, l, w0) : w0);
  }
  template <bool ENT> __device__ __forceinline__ float2 at(float2 z) const {
    float2 l = fma2(add2(z, {-m, -m}), {c2, c2}, {-log2_s, -log2_s});
    if (ENT) l = {fmaxf(l.x, -200.f), fmaxf(l.y, -200.f)};
    const float2 p = {exp2_fast(l.x), exp2_fast(l.y)};
    return mul2(p, ENT ? fma2({w1, w1}, l, {w0, w0}) : float2{w0, w0});
  }
};

// ROW_THREADS threads share a row: a block with `segments` blocks per row, or a warp.  SAME: input and output rows start at
// the same place within eight elements, so that both take wide accesses; otherwise elements one at a time (5600 rows of 33278 in
// bf16, 33278 apart into rows 33280 apart: 374 us; 117 where both are 33280 apart, 121 where both are 33278).
template <typename In, typename Out, bool ENT, int ROW_THREADS, bool SAME>
__global__ void __launch_bounds__(256) logprobs_grad_kernel(const LogGradArgs a) {
  await_previous();
  let_next_start();
  const int lane = threadIdx.x % ROW_THREADS;
  const unsigned unit = ROW_THREADS == 256 ? blockIdx.x : blockIdx.x * (256 / ROW_THREADS) + threadIdx.x / ROW_THREADS;
  const long long row = ROW_THREADS == 256 && a.segments > 1 ? unit / (unsigned)a.segments : unit;
  const int segment = ROW_THREADS == 256 ? (int)(unit - (unsigned)row * a.segments) : 0;
  if (row >= a.n) return;
  const int token = given_token(a.tokens, a.token64, row, a.vocab, lane == 0 && segment == 0 ? a.status : nullptr);
  const In* z = static_cast<const In*>(a.logits) + row * a.ld;
  Out* out = static_cast<Out*>(a.out) + row * a.ld_out;
  const RowSpan r = SAME ? RowSpan::of(z, a.vocab) : RowSpan{0, 0, a.vocab};
  RowGrad f{};
  bool zero = token == -2;
  if (!zero) {
    const float2 norm = a.norm[row];
    f.m = norm.x;
    f.c2 = a.scale * kLog2e;
    f.log2_s = norm.y * kLog2e;
    f.g = a.g_logp != nullptr && token >= 0 ? a.g_logp[row * a.g_step] * a.scale : 0.f;
    f.w0 = -f.g;
    if (ENT) {
      const float h = a.g_entropy[row * a.h_step] * a.scale;
      f.w0 = -fmaf(h, a.entropy[row], f.g);
      f.w1 = -h * kLn2;
    }
    zero = f.m == kMinusInf;
    if (norm.y != norm.y || f.m != f.m) f.w0 = not_a_number();
  }
  auto single = [&](int i) {
    float v = 0.f;
    if (!zero) v = f.template at<ENT>(to_float(z[i])) + (i == token ? f.g : 0.f);
    if constexpr (sizeof(Out) == 2) out[i] = __float2bfloat16_rn(v);
    else out[i] = v;
  };
  if (!SAME) {
    // (unsigned: a step past the last element of the longest rows is beyond 2^31)
    const unsigned from = (unsigned)segment * a.stretch, vocab = a.vocab;
    const unsigned to = ROW_THREADS == 256 ? min(vocab, from + a.stretch) : vocab;
    for (unsigned i = from + lane; i < to; i += ROW_THREADS) single((int)i);
    return;
  }
  const int first = segment * a.stretch, last = ROW_THREADS == 256 ? min(r.groups, first + a.stretch) : r.groups;
  constexpr int kTogether = 4;
  for (int g = first + lane; g < last; g += ROW_THREADS * kTogether) {
    Eight<In> x[kTogether];
#pragma unroll
    for (int k = 0; k < kTogether; ++k)
      if (!zero && g + k * ROW_THREADS < last) x[k].load(z + r.head + 8ll * (g + k * ROW_THREADS));
#pragma unroll
    for (int k = 0; k < kTogether; ++k) {
      if (g + k * ROW_THREADS >= last) break;
      const int i = r.head + 8 * (g + k * ROW_THREADS);
      float v[8] = {};
      if (!zero) {
        x[k].get(v);
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          const float2 y = f.template at<ENT>(float2{v[j], v[j + 1]});
          v[j] = y.x;
          v[j + 1] = y.y;
        }
        if ((unsigned)(token - i) < 8u) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] += i + j == token ? f.g : 0.f;
        }
      }
      Eight<Out> y;
      y.put(v);
      y.store(out + i);
    }
  }
  if (segment == 0 && lane < 14) {
    const int i = r.single(lane);
    if (i >= 0) single(i);
  }
}

// Blocks of a row: one where there are rows enough (its start, a chain of loads, is then paid once: 5600 rows of 33278 took 149 us
// in five blocks each and take 119 in one), more where there are few (64 rows of 131071 in fp32: 11.5 us in 37, 19.3 in one).
static int grad_segments(const acc_ctx* ctx, long long n, int vocab) {
  const long long some = (16ll * ctx->sm_count + n - 1) / n, most = (vocab + 2047ll) / 2048;
  return (int)std::max<long long>(1, std::min(some, most));
}
static bool grad_warp_rows(const acc_ctx* ctx, long long n, int vocab) { return warp_rows(ctx, n, vocab); }
long long logprobs_grad_blocks(const acc_ctx* ctx, long long n, int vocab) {
  return grad_warp_rows(ctx, n, vocab) ? (n + 7) / 8 : n * grad_segments(ctx, n, vocab);
}

cudaError_t launch_token_logprobs_grad(acc_ctx* ctx, const void* logits, bool bf16, long long n, int vocab, long long ld,
                                       const void* tokens, bool tok64, float scale, const float* norm, const float* g_logp,
                                       long long g_count, const float* g_entropy, long long h_count, const float* entropy,
                                       void* out, bool out_bf16, long long ld_out, cudaStream_t s) {
  LogGradArgs a{logits, tokens, tok64, n, ld, ld_out, vocab, scale, reinterpret_cast<const float2*>(norm), g_logp, g_entropy,
                entropy, g_count > 1, h_count > 1, out, ctx->d_status, 1, 0};
  const size_t in_size = bf16 ? 2 : 4, out_size = out_bf16 ? 2 : 4;
  const bool same = (reinterpret_cast<uintptr_t>(logits) / in_size) % 8 == (reinterpret_cast<uintptr_t>(out) / out_size) % 8 &&
                    (n == 1 || (ld - ld_out) % 8 == 0);
  const bool warp = grad_warp_rows(ctx, n, vocab);
  if (!warp) {
    a.segments = grad_segments(ctx, n, vocab);
    a.stretch = (int)(((same ? vocab / 8 : vocab) + a.segments - 1ll) / a.segments);
  }
  PhaseTimer pt(ctx, PH_LOGPROBS_GRAD, s);
  auto go = [&](auto in, auto o, auto ent) {
    using In = decltype(in);
    using Out = decltype(o);
    constexpr bool ENT = decltype(ent)::value;
    auto* kernel = warp ? (same ? logprobs_grad_kernel<In, Out, ENT, 32, true> : logprobs_grad_kernel<In, Out, ENT, 32, false>)
                        : (same ? logprobs_grad_kernel<In, Out, ENT, 256, true> : logprobs_grad_kernel<In, Out, ENT, 256, false>);
    return launch_early(kernel, (unsigned)logprobs_grad_blocks(ctx, n, vocab), 256, s, a);
  };
  auto typed = [&](auto ent) {
    if (bf16) return out_bf16 ? go(__nv_bfloat16(), __nv_bfloat16(), ent) : go(__nv_bfloat16(), 0.f, ent);
    return out_bf16 ? go(0.f, __nv_bfloat16(), ent) : go(0.f, 0.f, ent);
  };
  return g_entropy != nullptr ? typed(std::true_type()) : typed(std::false_type());
}

}  // namespace acc
