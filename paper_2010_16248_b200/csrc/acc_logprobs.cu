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

// The running statistics of a set of logits z: m = max z, s = sum 2^d, t = sum 2^d d with d = (z - m) * scale * log2(e).  A
// distance below -200 counts as -200, where 2^d is 0: -inf and the type's lowest value then add nothing, not 0 * inf.
struct Stats { float m, s, t; };

__device__ __forceinline__ float distance(float z, float m, float c2) { return fmaxf((z - m) * c2, -200.f); }

__device__ __forceinline__ Stats merge(const Stats& a, const Stats& b, float c2) {
  const float m = max_nan(a.m, b.m);
  const float da = distance(a.m, m, c2), db = distance(b.m, m, c2);
  const float fa = exp2_fast(da), fb = exp2_fast(db);
  return {m, fa * a.s + fb * b.s, fa * fmaf(a.s, da, a.t) + fb * fmaf(b.s, db, b.t)};
}
__device__ __forceinline__ Stats merge_warp(Stats a, float c2) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const Stats b{__shfl_xor_sync(0xffffffffu, a.m, o), __shfl_xor_sync(0xffffffffu, a.s, o),
                  __shfl_xor_sync(0xffffffffu, a.t, o)};
    a = merge(a, b, c2);
  }
  return a;
}

// Adds N values whose largest is `top` (NaN when one of them is).
template <bool ENT, int N> __device__ __forceinline__ void add_values(Stats& a, const float* z, float top, float c2) {
  if (!(top <= a.m)) {
    const float m = max_nan(a.m, top), d = distance(a.m, m, c2), f = exp2_fast(d);
    if (ENT) a.t = f * fmaf(a.s, d, a.t);
    a.s *= f;
    a.m = m;
  }
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const float d = distance(z[k], a.m, c2), e = exp2_fast(d);
    a.s += e;
    if (ENT) a.t = fmaf(e, d, a.t);
  }
}

// Statistics of this thread's share of a row: groups first + own, first + own + stride, ... below last, and single elements.
template <typename T, bool ENT>
__device__ __forceinline__ Stats row_share(const T* row, const RowSpan& r, int first, int last, int own, int stride,
                                           int single, float c2) {
  constexpr int kBatch = 4;
  Stats a{kMinusInf, 0.f, 0.f};
  const T* p = row + r.head;
  for (int g = first + own; g < last; g += kBatch * stride) {
    Eight<T> x[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (g + k * stride < last) x[k].load(p + 8ll * (g + k * stride));
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      if (g + k * stride >= last) break;
      float z[8];
      x[k].get(z);
      float top = z[0];
#pragma unroll
      for (int j = 1; j < 8; ++j) top = max_nan(top, z[j]);
      add_values<ENT, 8>(a, z, top, c2);
    }
  }
  const int i = r.single(single);
  if (i >= 0) {
    const float z = to_float(row[i]);
    add_values<ENT, 1>(a, &z, z, c2);
  }
  return a;
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
  float* logp;          // each output may be nullptr
  float2* norm;
  float* entropy;
  int top;
  int* top_index;
  float* top_logp;
  int* status;
  int parts;            // blocks per row
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
  float log_s = logf(s.s), entropy = log_s - s.t / s.s * kLn2;
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

constexpr int kRowThreads = 256, kGroupMaxima = kRowThreads / 4, kCandidates = 1024;

struct RowShared {
  Stats stats[kRowThreads / 32];
  Stats all;
  float maxima[kGroupMaxima];
  float bar;                     // a bound that at least `top` logits of the share reach
  int count;
  Key best[ACC_LOGPROBS_MAX_TOP];
  Key list[kCandidates];
};

// list[0 .. count) -> best[0 .. top), in order; keys are distinct, so the order in which the list was filled does not matter.
__device__ __forceinline__ void rank_list(RowShared& sh, int count, int top) {
  if ((int)threadIdx.x < top) sh.best[threadIdx.x] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < count; i += kRowThreads) {
    const Key own = sh.list[i];
    int rank = 0;
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
// `top`-th largest of 64 such maxima, four threads each, is a bar that at least `top` logits reach, and only the shares of
// threads whose maximum reaches it are read again, by whole warps: for top = 20 about 25 of 256.  Ties at the bar may be many
// (a mask of the type's lowest value leaves them): then those above it are taken and those at it searched in order of index.
template <typename T>
__device__ __forceinline__ void select_top(RowShared& sh, const T* row, const RowSpan& r, int first, int last, int single,
                                           float own_max, int top) {
  const int tid = threadIdx.x, lane = tid & 31;
  float m = own_max;
  m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
  m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
  if ((tid & 3) == 0) sh.maxima[tid >> 2] = m;
  if (tid == 0) { sh.bar = kMinusInf; sh.count = 0; }
  __syncthreads();
  if (tid < kGroupMaxima) {
    const float own = sh.maxima[tid];
    int rank = 0;
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
    unsigned todo = __ballot_sync(0xffffffffu, take(own_max));
    while (todo != 0) {
      const int owner = (tid & ~31) + __ffs(todo) - 1;
      todo &= todo - 1;
      each_value(row, r, first + owner, last, lane * kRowThreads, 32 * kRowThreads, -1,
                 [&](float z, int i) { if (take(z)) push(z, i); });
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
        each_value(row, r, g, min(last, g + kSearch), tid, kRowThreads, g == first && tid < 7 ? single : -1,
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
        each_value(row, r, first, last, tid, kRowThreads, single, [&](float z, int i) {
          const Key key = make_key(z, i);
          if (z > kMinusInf && key < below && key > best) best = key;
        });
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
        __syncthreads();
        if (lane == 0) sh.list[tid >> 5] = best;
        __syncthreads();
        best = 0;
        for (int j = 0; j < kRowThreads / 32; ++j) best = max(best, sh.list[j]);
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
// memory.  One pass over the logits; the alternatives cost a second look at a tenth of them, which the L2 cache still holds.
template <typename T, bool ENT, bool TOP>
__global__ void __launch_bounds__(kRowThreads) logprobs_kernel(const LogArgs a) {
  namespace cg = cooperative_groups;
  __shared__ RowShared sh;
  await_previous();
  let_next_start();
  const int parts = a.parts, tid = threadIdx.x;
  const long long row = blockIdx.x / parts;
  const int part = blockIdx.x % parts;
  const int token = given_token(a.tokens, a.token64, row, a.vocab, tid == 0 && part == 0 ? a.status : nullptr);
  if (token == -2) {
    if (part == 0) skip_row(a, row, tid, kRowThreads);
    return;
  }
  const T* z = static_cast<const T*>(a.logits) + row * a.ld;
  const RowSpan r = RowSpan::of(z, a.vocab);
  const int first = (int)((long long)r.groups * part / parts), last = (int)((long long)r.groups * (part + 1) / parts);
  // the singles before the groups belong to the first part, those behind them to the last
  const int single = tid < 7 ? (part == 0 ? tid : -1) : tid < 14 && part == parts - 1 ? tid : -1;
  const float c2 = a.scale * kLog2e;
  const Stats own = row_share<T, ENT>(z, r, first, last, tid, kRowThreads, single < 0 ? 14 : single, c2);
  {
    const Stats w = merge_warp(own, c2);
    if ((tid & 31) == 0) sh.stats[tid >> 5] = w;
  }
  __syncthreads();
  if (tid < 32) {
    Stats w = tid < kRowThreads / 32 ? sh.stats[tid] : Stats{kMinusInf, 0.f, 0.f};
    w = merge_warp(w, c2);
    if (tid == 0) sh.all = w;
  }
  if (TOP) select_top(sh, z, r, first, last, single < 0 ? 14 : single, own.m, a.top);
  __syncthreads();
  Stats all = sh.all;
  if (parts > 1) {
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    if (part == 0) {
      for (int p = 1; p < parts; ++p) all = merge(all, *cluster.map_shared_rank(&sh.all, p), c2);
      if (TOP) {
        for (int i = tid; i < parts * a.top; i += kRowThreads) sh.list[i] = cluster.map_shared_rank(sh.best, i / a.top)[i % a.top];
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

// A row per warp, for vocabularies of which a lane's share is a few vectors; the alternatives one after another.
template <typename T, bool ENT, bool TOP>
__global__ void __launch_bounds__(256) logprobs_warp_kernel(const LogArgs a) {
  await_previous();
  let_next_start();
  const long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (row >= a.n) return;
  const int token = given_token(a.tokens, a.token64, row, a.vocab, lane == 0 ? a.status : nullptr);
  if (token == -2) {
    skip_row(a, row, lane, 32);
    return;
  }
  const T* z = static_cast<const T*>(a.logits) + row * a.ld;
  const RowSpan r = RowSpan::of(z, a.vocab);
  const float c2 = a.scale * kLog2e;
  const Stats all = merge_warp(row_share<T, ENT>(z, r, 0, r.groups, lane, 32, lane, c2), c2);
  float log_s = 0.f;
  if (lane == 0) log_s = finish_row(a, row, all, token, token >= 0 ? to_float(z[token]) : 0.f);
  if (!TOP) return;
  log_s = __shfl_sync(0xffffffffu, log_s, 0);
  // a lane's best key below its last; only the lane whose key was taken looks again
  auto next = [&](Key below) {
    Key best = 0;
    each_value(z, r, 0, r.groups, lane, 32, lane, [&](float v, int i) {
      const Key key = make_key(v, i);
      if (v > kMinusInf && key < below && key > best) best = key;
    });
    return best;
  };
  Key mine = next(~0ull), kept = 0;
  for (int k = 0; k < a.top; ++k) {
    Key best = mine;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
    if (lane == k) kept = best;
    if (best == 0) break;
    if (mine == best) mine = next(best);
  }
  if (lane < a.top) write_top(a, row, lane, kept, all.m, log_s);
}

// Vocabularies up to this length take a warp per row.
constexpr int kWarpVocab = 1024;

// Blocks per row: as many as keep the GPU busy when there are few rows, each with a stretch worth a block's start.
static int row_parts(const acc_ctx* ctx, long long n, int vocab) {
  int parts = 1;
  while (parts < 8 && n * parts * 2 <= 4ll * ctx->sm_count && vocab / (parts * 2) >= 2048) parts *= 2;
  return parts;
}

cudaError_t launch_token_logprobs(acc_ctx* ctx, const void* logits, bool bf16, long long n, int vocab, long long ld,
                                  const void* tokens, bool tok64, float scale, float* logp, float* norm, float* entropy,
                                  int top, int* top_index, float* top_logp, cudaStream_t s) {
  LogArgs a{logits, tokens, tok64, n, ld, vocab, scale, logp, reinterpret_cast<float2*>(norm), entropy, top, top_index,
            top_logp, ctx->d_status, 1};
  PhaseTimer pt(ctx, PH_LOGPROBS, s);
  auto go = [&](auto t) {
    using T = decltype(t);
    const bool ent = entropy != nullptr;
    if (vocab <= kWarpVocab) {
      auto* kernel = top > 0 ? (ent ? logprobs_warp_kernel<T, true, true> : logprobs_warp_kernel<T, false, true>)
                             : (ent ? logprobs_warp_kernel<T, true, false> : logprobs_warp_kernel<T, false, false>);
      return launch_early(kernel, (unsigned)((n + 7) / 8), 256, s, a);
    }
    a.parts = row_parts(ctx, n, vocab);
    auto* kernel = top > 0 ? (ent ? logprobs_kernel<T, true, true> : logprobs_kernel<T, false, true>)
                           : (ent ? logprobs_kernel<T, true, false> : logprobs_kernel<T, false, false>);
    return launch_early_as(kernel, (unsigned)(n * a.parts), kRowThreads, 0, a.parts, s, a);
  };
  return bf16 ? go(__nv_bfloat16()) : go(0.f);
}

// ---- gradient ----------------------------------------------------------------------------------------------------
// dz_j = scale [ g (1[j = token] - p_j) - h p_j (log p_j + H) ]  with  log p_j = (z_j - max) scale - log S.

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
  int segments;            // blocks per row
};

// What one row's elements need.
struct RowGrad {
  float m, c2, log2_s;     // log2 p = (z - m) c2 - log2_s
  float g, h, h_entropy;   // times scale; h_entropy = h H
  int token;
  template <bool ENT> __device__ __forceinline__ float at(float z, int index) const {
    float l = fmaf(z - m, c2, -log2_s);
    if (ENT) l = fmaxf(l, -200.f);  // 2^-200 is 0, and so is its product
    const float p = exp2_fast(l);
    const float w = ENT ? fmaf(h * kLn2, l, g + h_entropy) : g;
    return index == token ? g - p * w : -p * w;
  }
};

constexpr int kGradBatch = 4;  // groups of eight elements that a thread loads together

// ROW_THREADS threads share a row: a block with `segments` blocks per row, or a warp.  SAME: input and output rows start at
// the same place within eight elements, so that both take wide accesses; otherwise elements one at a time.
template <typename In, typename Out, bool ENT, int ROW_THREADS, bool SAME>
__global__ void __launch_bounds__(256) logprobs_grad_kernel(const LogGradArgs a) {
  await_previous();
  let_next_start();
  const int lane = threadIdx.x % ROW_THREADS;
  const long long unit = ROW_THREADS == 256 ? blockIdx.x : (long long)blockIdx.x * (256 / ROW_THREADS) + threadIdx.x / ROW_THREADS;
  const long long row = ROW_THREADS == 256 ? unit / a.segments : unit;
  const int segment = ROW_THREADS == 256 ? (int)(unit - row * a.segments) : 0;
  if (row >= a.n) return;
  const int token = given_token(a.tokens, a.token64, row, a.vocab, lane == 0 && segment == 0 ? a.status : nullptr);
  const In* z = static_cast<const In*>(a.logits) + row * a.ld;
  Out* out = static_cast<Out*>(a.out) + row * a.ld_out;
  const RowSpan r = SAME ? RowSpan::of(z, a.vocab) : RowSpan{0, 0, a.vocab};
  RowGrad f{};
  f.token = token;
  bool zero = token == -2;
  if (!zero) {
    const float2 norm = a.norm[row];
    f.m = norm.x;
    f.c2 = a.scale * kLog2e;
    f.log2_s = norm.y * kLog2e;
    f.g = a.g_logp != nullptr ? a.g_logp[row * a.g_step] * a.scale : 0.f;
    if (ENT) {
      f.h = a.g_entropy[row * a.h_step] * a.scale;
      f.h_entropy = f.h * a.entropy[row];
    }
    if (token < 0) f.g = 0.f;  // no token was given
    zero = f.m == kMinusInf;
    if (norm.y != norm.y || f.m != f.m) f.g = f.h_entropy = not_a_number();
  }
  auto single = [&](int i) {
    float v = 0.f;
    if (!zero) v = f.template at<ENT>(to_float(z[i]), i);
    if constexpr (sizeof(Out) == 2) out[i] = __float2bfloat16_rn(v);
    else out[i] = v;
  };
  if (!SAME) {
    const int from = segment * 256 * kGradBatch * 8;
    const int to = ROW_THREADS == 256 ? min(a.vocab, from + 256 * kGradBatch * 8) : a.vocab;
    for (int i = from + lane; i < to; i += ROW_THREADS) single(i);
    return;
  }
  const int g0 = segment * ROW_THREADS * kGradBatch + lane;
  const int last = ROW_THREADS == 256 ? min(r.groups, (segment + 1) * ROW_THREADS * kGradBatch) : r.groups;
  for (int g = g0; g < last; g += ROW_THREADS * kGradBatch) {
    Eight<In> x[kGradBatch];
#pragma unroll
    for (int k = 0; k < kGradBatch; ++k)
      if (!zero && g + k * ROW_THREADS < last) x[k].load(z + r.head + 8ll * (g + k * ROW_THREADS));
#pragma unroll
    for (int k = 0; k < kGradBatch; ++k) {
      if (g + k * ROW_THREADS >= last) break;
      const int i = r.head + 8 * (g + k * ROW_THREADS);
      float v[8] = {};
      if (!zero) {
        x[k].get(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = f.template at<ENT>(v[j], i + j);
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

// Blocks of a row, for rows of more than a warp's share.
static int grad_segments(int vocab) { return (vocab + 256 * kGradBatch * 8 - 1) / (256 * kGradBatch * 8); }
long long logprobs_grad_blocks(long long n, int vocab) {
  return vocab <= kWarpVocab ? (n + 7) / 8 : n * grad_segments(vocab);
}

cudaError_t launch_token_logprobs_grad(acc_ctx* ctx, const void* logits, bool bf16, long long n, int vocab, long long ld,
                                       const void* tokens, bool tok64, float scale, const float* norm, const float* g_logp,
                                       long long g_count, const float* g_entropy, long long h_count, const float* entropy,
                                       void* out, bool out_bf16, long long ld_out, cudaStream_t s) {
  LogGradArgs a{logits, tokens, tok64, n, ld, ld_out, vocab, scale, reinterpret_cast<const float2*>(norm), g_logp, g_entropy,
                entropy, g_count > 1, h_count > 1, out, ctx->d_status, 1};
  const size_t in_size = bf16 ? 2 : 4, out_size = out_bf16 ? 2 : 4;
  const bool same = (reinterpret_cast<uintptr_t>(logits) / in_size) % 8 == (reinterpret_cast<uintptr_t>(out) / out_size) % 8 &&
                    (n == 1 || (ld - ld_out) % 8 == 0);
  const bool warp = vocab <= kWarpVocab;
  if (!warp) a.segments = grad_segments(vocab);
  PhaseTimer pt(ctx, PH_LOGPROBS_GRAD, s);
  auto go = [&](auto in, auto o, auto ent) {
    using In = decltype(in);
    using Out = decltype(o);
    constexpr bool ENT = decltype(ent)::value;
    auto* kernel = warp ? (same ? logprobs_grad_kernel<In, Out, ENT, 32, true> : logprobs_grad_kernel<In, Out, ENT, 32, false>)
                        : (same ? logprobs_grad_kernel<In, Out, ENT, 256, true> : logprobs_grad_kernel<In, Out, ENT, 256, false>);
    return launch_early(kernel, (unsigned)logprobs_grad_blocks(n, vocab), 256, s, a);
  };
  auto typed = [&](auto ent) {
    if (bf16) return out_bf16 ? go(__nv_bfloat16(), __nv_bfloat16(), ent) : go(__nv_bfloat16(), 0.f, ent);
    return out_bf16 ? go(0.f, __nv_bfloat16(), ent) : go(0.f, 0.f, ent);
  };
  return g_entropy != nullptr ? typed(std::true_type()) : typed(std::false_type());
}

}  // namespace acc
