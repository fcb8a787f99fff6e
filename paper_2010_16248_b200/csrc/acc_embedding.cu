// Embedding of a MATRIX layer: the lookup of token rows, and the gradient as one sum per distinct token.
#include <cuda_bf16.h>

#include "acc_internal.cuh"

namespace acc {

// VEC adjacent values of fp32 or bf16, as fp32.  VEC is the widest width at which every row of the layer starts aligned.
template <int VEC> struct Vals { float v[VEC]; };

template <int VEC> __device__ __forceinline__ Vals<VEC> load_vals(const float* p) {
  Vals<VEC> r;
  if constexpr (VEC == 4) {
    const float4 a = *reinterpret_cast<const float4*>(p);
    r.v[0] = a.x; r.v[1] = a.y; r.v[2] = a.z; r.v[3] = a.w;
  } else if constexpr (VEC == 2) {
    const float2 a = *reinterpret_cast<const float2*>(p);
    r.v[0] = a.x; r.v[1] = a.y;
  } else {
    r.v[0] = *p;
  }
  return r;
}
template <int VEC> __device__ __forceinline__ Vals<VEC> load_vals(const __nv_bfloat16* p) {
  Vals<VEC> r;
  if constexpr (VEC == 4) {
    const uint2 a = *reinterpret_cast<const uint2*>(p);
    r.v[0] = __uint_as_float(a.x << 16); r.v[1] = __uint_as_float(a.x & 0xffff0000u);
    r.v[2] = __uint_as_float(a.y << 16); r.v[3] = __uint_as_float(a.y & 0xffff0000u);
  } else if constexpr (VEC == 2) {
    const unsigned a = *reinterpret_cast<const unsigned*>(p);
    r.v[0] = __uint_as_float(a << 16); r.v[1] = __uint_as_float(a & 0xffff0000u);
  } else {
    r.v[0] = __bfloat162float(*p);
  }
  return r;
}
template <int VEC> __device__ __forceinline__ void store_vals(float* p, const Vals<VEC>& r) {
  if constexpr (VEC == 4) *reinterpret_cast<float4*>(p) = make_float4(r.v[0], r.v[1], r.v[2], r.v[3]);
  else if constexpr (VEC == 2) *reinterpret_cast<float2*>(p) = make_float2(r.v[0], r.v[1]);
  else *p = r.v[0];
}
template <int VEC> __device__ __forceinline__ void store_vals(__nv_bfloat16* p, const Vals<VEC>& r) {
  if constexpr (VEC == 1) {
    *p = __float2bfloat16_rn(r.v[0]);
  } else {
    unsigned w[VEC / 2];
#pragma unroll
    for (int k = 0; k < VEC / 2; ++k) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(r.v[2 * k], r.v[2 * k + 1]);
      w[k] = *reinterpret_cast<const unsigned*>(&h);
    }
    if constexpr (VEC == 4) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<unsigned*>(p) = w[0];
  }
}

// A token's row, or `rows` where there is none: ids below zero pad the batch; ids beyond the table are reported in the
// status word and read nothing.
__device__ __forceinline__ unsigned token_row(long long tok, int rows, int* status) {
  if (tok < 0) return (unsigned)rows;
  if (tok >= rows) {
    atomicCAS(status, 0, ACC_EINDEX);
    return (unsigned)rows;
  }
  return (unsigned)tok;
}

// One warp per token:  out_i = scale * row(tok_i), rounded once; zeros where there is no row.
template <typename Tok, typename Out, int VEC>
__global__ void __launch_bounds__(256)
embedding_lookup_kernel(const float* __restrict__ table, int rows, int cols, const Tok* __restrict__ tokens, long long n,
                        float scale, Out* __restrict__ out, int* status) {
  const long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (i >= n) return;
  const int lane = threadIdx.x & 31;
  const unsigned row = token_row((long long)tokens[i], rows, status);
  const float* src = table + (long long)row * cols;
  Out* dst = out + i * cols;
  const int nv = cols / VEC;
  if (row == (unsigned)rows) {
    for (int j = lane; j < nv; j += 32) store_vals<VEC>(dst + (long long)j * VEC, Vals<VEC>{});
    return;
  }
#pragma unroll 4
  for (int j = lane; j < nv; j += 32) {
    Vals<VEC> a = load_vals<VEC>(src + (long long)j * VEC);
#pragma unroll
    for (int k = 0; k < VEC; ++k) a.v[k] *= scale;
    store_vals<VEC>(dst + (long long)j * VEC, a);
  }
}

// ---- gradient ----------------------------------------------------------------------------------------------------
// G_w[r] (+)= scale * sum over the tokens i of worker w with tok_i = r of dy_i.  The tokens of a worker are sorted by
// (row, position); the sorted order is cut into chunks of 32 entries, whatever the rows, so that a frequent token costs no
// more than 32 rare ones.  A row whose entries lie inside one chunk is final there; one that crosses a chunk's edge leaves
// a partial sum in that chunk's head or tail slot, and the next level adds the slots of 32 chunks in the same way, until
// one chunk is left.  Every sum has one writer and a fixed order, so results do not change from run to run.

struct EmbArgs {
  long long offset;      // of the layer inside a worker's slice
  long long stride;      // elements between workers
  long long size;        // rows * cols
  int rows, cols, n;     // n: tokens per worker
};

// Zeros of every worker's slice of the layer, cut into pieces of kZeroPiece elements.
constexpr int kZeroPiece = 32768;
__device__ __forceinline__ void zero_piece(float* __restrict__ grads, const EmbArgs& a, long long piece, long long pieces_per_worker) {
  const long long w = piece / pieces_per_worker;
  const long long e0 = (piece - w * pieces_per_worker) * kZeroPiece;
  float* g = grads + w * a.stride + a.offset + e0;
  const int n = (int)min((long long)kZeroPiece, a.size - e0);
  for (int i = 4 * (int)threadIdx.x; i + 4 <= n; i += 4 * (int)blockDim.x) st_stream4(g + i, make_float4(0.f, 0.f, 0.f, 0.f));
  for (int i = (n & ~3) + (int)threadIdx.x; i < n; i += blockDim.x) g[i] = 0.f;
}

// Up to kRankMost tokens per worker: a token's place is the number of tokens before it in (row, position) order, counted
// against all of them in shared memory.  Quadratic, but 256 tokens per block and no pass waits for another: 700 tokens
// take 1/3 of one radix pass's launches.  Blocks behind the counting ones write zeros meanwhile.
constexpr int kRankMost = 2048, kRankBlock = 256;
template <typename Tok>
__global__ void __launch_bounds__(kRankBlock)
embedding_rank_kernel(const Tok* __restrict__ tokens, EmbArgs a, unsigned* __restrict__ keys, unsigned* __restrict__ pos,
                      int rank_blocks, int blocks_per_worker, float* __restrict__ grads, long long pieces_per_worker,
                      int* status) {
  if ((int)blockIdx.x >= rank_blocks) {
    zero_piece(grads, a, (long long)blockIdx.x - rank_blocks, pieces_per_worker);
    return;
  }
  __shared__ __align__(16) unsigned sk[kRankMost];
  const int w = blockIdx.x / blocks_per_worker, first = (int)(blockIdx.x % blocks_per_worker) * kRankBlock;
  const Tok* tok = tokens + (long long)w * a.n;
  const int n4 = (a.n + 3) & ~3;
  for (int j = threadIdx.x; j < n4; j += kRankBlock)
    sk[j] = j < a.n ? token_row((long long)tok[j], a.rows, status) : 0xffffffffu;
  __syncthreads();
  const int i = first + (int)threadIdx.x;
  const unsigned key = i < a.n ? sk[i] : 0u;
  int rank = 0;
  // tokens before this block's come first among equals, those behind it last
  const int last = min(first + kRankBlock, n4);
  for (int j = 0; j < first; j += 4) {
    const uint4 o = *reinterpret_cast<const uint4*>(sk + j);
    rank += (o.x <= key) + (o.y <= key) + (o.z <= key) + (o.w <= key);
  }
  for (int j = first; j < last; ++j) rank += sk[j] < key || (sk[j] == key && j < i);
  for (int j = last; j < n4; j += 4) {
    const uint4 o = *reinterpret_cast<const uint4*>(sk + j);
    rank += (o.x < key) + (o.y < key) + (o.z < key) + (o.w < key);
  }
  if (i < a.n) {
    keys[(long long)w * a.n + rank] = key;
    pos[(long long)w * a.n + rank] = (unsigned)i;
  }
}

// More tokens: a stable radix sort, eight bits of the row at a time, in tiles of kSortTile tokens.
constexpr int kSortTile = 2048, kSortThreads = 256, kSortWarps = kSortThreads / 32;

__device__ __forceinline__ long long sort_hist_at(int w, int digit, int tile, int n_tiles) {
  return ((long long)w * 256 + digit) * n_tiles + tile;
}

// First pass: rows from tokens, positions in order, and the first digit's histogram of every tile.
template <typename Tok>
__global__ void __launch_bounds__(kSortThreads)
embedding_keys_kernel(const Tok* __restrict__ tokens, EmbArgs a, unsigned* __restrict__ keys, unsigned* __restrict__ pos,
                      unsigned* __restrict__ hist, int n_tiles, int sort_blocks, float* __restrict__ grads,
                      long long pieces_per_worker, int* status) {
  if ((int)blockIdx.x >= sort_blocks) {
    zero_piece(grads, a, (long long)blockIdx.x - sort_blocks, pieces_per_worker);
    return;
  }
  __shared__ unsigned h[256];
  h[threadIdx.x] = 0u;
  __syncthreads();
  const int w = blockIdx.x / n_tiles, tile = blockIdx.x % n_tiles;
  const long long w0 = (long long)w * a.n;
  const int end = min((tile + 1) * kSortTile, a.n);
  for (int i = tile * kSortTile + (int)threadIdx.x; i < end; i += kSortThreads) {
    const unsigned key = token_row((long long)tokens[w0 + i], a.rows, status);
    keys[w0 + i] = key;
    pos[w0 + i] = (unsigned)i;
    atomicAdd(&h[key & 255u], 1u);
  }
  __syncthreads();
  hist[sort_hist_at(w, threadIdx.x, tile, n_tiles)] = h[threadIdx.x];
}

__global__ void __launch_bounds__(kSortThreads)
embedding_hist_kernel(const unsigned* __restrict__ keys, int n, int shift, unsigned* __restrict__ hist, int n_tiles) {
  __shared__ unsigned h[256];
  h[threadIdx.x] = 0u;
  __syncthreads();
  const int w = blockIdx.x / n_tiles, tile = blockIdx.x % n_tiles;
  const long long w0 = (long long)w * n;
  const int end = min((tile + 1) * kSortTile, n);
  for (int i = tile * kSortTile + (int)threadIdx.x; i < end; i += kSortThreads)
    atomicAdd(&h[(keys[w0 + i] >> shift) & 255u], 1u);
  __syncthreads();
  hist[sort_hist_at(w, threadIdx.x, tile, n_tiles)] = h[threadIdx.x];
}

// One block per worker: exclusive sum over (digit, tile), in place.
__global__ void __launch_bounds__(1024)
embedding_scan_kernel(unsigned* __restrict__ hist, int n_tiles) {
  __shared__ unsigned part[32];
  unsigned* h = hist + (long long)blockIdx.x * 256 * n_tiles;
  const int total = 256 * n_tiles, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned before = 0u;
  for (int i0 = 0; i0 < total; i0 += 1024) {
    const int i = i0 + (int)threadIdx.x;
    const unsigned own = i < total ? h[i] : 0u;
    unsigned inc = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned up = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += up;
    }
    if (lane == 31) part[warp] = inc;
    __syncthreads();
    unsigned p = part[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned up = __shfl_up_sync(0xffffffffu, p, o);
      if (lane >= o) p += up;
    }
    const unsigned below = warp > 0 ? __shfl_sync(0xffffffffu, p, warp - 1) : 0u;
    const unsigned all = __shfl_sync(0xffffffffu, p, 31);
    if (i < total) h[i] = before + below + inc - own;
    before += all;
    __syncthreads();
  }
}

// Moves a tile's entries to their places.  A warp takes 256 adjacent entries, 32 at a time in order; lanes with the same
// digit rank themselves by lane, the warp's running counts give the rank among its earlier ones.
__global__ void __launch_bounds__(kSortThreads)
embedding_scatter_kernel(const unsigned* __restrict__ keys, const unsigned* __restrict__ pos, int n, int shift,
                         const unsigned* __restrict__ hist, int n_tiles, unsigned* __restrict__ keys_out,
                         unsigned* __restrict__ pos_out) {
  __shared__ unsigned cnt[kSortWarps][256];
  const int w = blockIdx.x / n_tiles, tile = blockIdx.x % n_tiles;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long w0 = (long long)w * n;
#pragma unroll
  for (int k = 0; k < kSortWarps; ++k) cnt[k][threadIdx.x] = 0u;
  __syncthreads();
  constexpr int kRounds = kSortTile / kSortThreads;
  const int i0 = tile * kSortTile + warp * (kSortTile / kSortWarps) + lane;
  unsigned key[kRounds], rank[kRounds];
#pragma unroll
  for (int k = 0; k < kRounds; ++k) key[k] = i0 + 32 * k < n ? keys[w0 + i0 + 32 * k] : 0u;
#pragma unroll
  for (int k = 0; k < kRounds; ++k) {
    const bool on = i0 + 32 * k < n;
    const unsigned digit = on ? (key[k] >> shift) & 255u : 256u;
    const unsigned same = __match_any_sync(0xffffffffu, digit);
    const unsigned ahead = on ? cnt[warp][digit] : 0u;
    rank[k] = ahead + __popc(same & ((1u << lane) - 1u));
    __syncwarp();
    if (on && (same >> lane) == 1u) cnt[warp][digit] = rank[k] + 1u;  // the last of the equal lanes
    __syncwarp();
  }
  __syncthreads();
  {
    unsigned run = hist[sort_hist_at(w, threadIdx.x, tile, n_tiles)];
#pragma unroll
    for (int k = 0; k < kSortWarps; ++k) {
      const unsigned c = cnt[k][threadIdx.x];
      cnt[k][threadIdx.x] = run;
      run += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kRounds; ++k) {
    if (i0 + 32 * k >= n) continue;
    const long long to = w0 + cnt[warp][(key[k] >> shift) & 255u] + rank[k];
    keys_out[to] = key[k];
    pos_out[to] = pos[w0 + i0 + 32 * k];
  }
}

// One level of sums.  FIRST: the entries are 32 sorted tokens, read from dy; otherwise they are the head and tail slots of
// 32 chunks of the level below, each of which covers `span` sorted tokens.  A thread owns VEC columns and adds eight
// entries' loads at a time.
constexpr int kChunk = 32;
template <typename In, int VEC, bool FIRST>
__global__ void __launch_bounds__(256)
embedding_sum_kernel(const In* __restrict__ dy, const float* __restrict__ below, const unsigned* __restrict__ keys,
                     const unsigned* __restrict__ pos, EmbArgs a, int span, int chunks_below, int chunks, int shares,
                     float scale,
                     int accumulate, float* __restrict__ grads, float* __restrict__ slots) {
  __shared__ unsigned skey[2 * kChunk + 1], ssrc[2 * kChunk];
  __shared__ int warp_n[2];
  // block order: column share fastest, then chunk, then worker
  const int share = blockIdx.x % shares, item = blockIdx.x / shares;
  const int w = item / chunks, chunk = item % chunks;
  const unsigned* kw = keys + (long long)w * a.n;
  const unsigned* pw = pos + (long long)w * a.n;
  const unsigned none = (unsigned)a.rows;
  // whether one row's entries lie on both sides of sorted place `at`
  auto crosses = [&](long long at) { return at > 0 && at < a.n && kw[at] != none && kw[at - 1] == kw[at]; };
  const long long chunk_span = FIRST ? kChunk : (long long)span * kChunk;
  const long long begin = chunk * chunk_span, end = min((long long)a.n, begin + chunk_span);
  const int lane = threadIdx.x & 31;
  if (threadIdx.x < 2 * kChunk) {
    bool valid = false;
    unsigned key = none, src = 0u;
    if (FIRST) {
      const long long e = begin + threadIdx.x;
      if (threadIdx.x < kChunk && e < end) {
        key = kw[e];
        valid = key != none;
        src = pw[e];
      }
    } else {
      const long long s = (long long)chunk * kChunk + (threadIdx.x >> 1);
      if (s < chunks_below) {
        const long long b = s * span, e = min((long long)a.n, b + span);
        const bool head = crosses(b);
        if ((threadIdx.x & 1) == 0) {
          valid = head;
          key = kw[b];
        } else {
          key = kw[e - 1];
          valid = crosses(e) && !(head && kw[b] == key);
        }
        src = (unsigned)(2 * s + (threadIdx.x & 1));
      }
    }
    const unsigned on = __ballot_sync(0xffffffffu, valid);
    if (lane == 0) warp_n[threadIdx.x >> 5] = __popc(on);
    __syncwarp();
    // entries in order, without gaps (the second warp's go behind the first's, filled in below)
    const int at = __popc(on & ((1u << lane) - 1u));
    if (threadIdx.x < 32) {
      if (valid) { skey[at] = key; ssrc[at] = src; }
    }
    asm volatile("bar.sync 1, 64;" ::: "memory");
    if (threadIdx.x >= 32 && valid) { skey[warp_n[0] + at] = key; ssrc[warp_n[0] + at] = src; }
  }
  __syncthreads();
  const int count = warp_n[0] + warp_n[1];
  if (count == 0) return;
  const bool open_left = crosses(begin), open_right = crosses(end);
  const int col = (share * (int)blockDim.x + (int)threadIdx.x) * VEC;
  if (col >= a.cols) return;
  const In* dw = FIRST ? dy + (long long)w * a.n * a.cols + col : nullptr;
  const float* bw = FIRST ? nullptr : below + (long long)w * 2 * chunks_below * a.cols + col;
  float* gw = grads + (long long)w * a.stride + a.offset + col;
  float* sw = slots + ((long long)w * chunks + chunk) * 2 * a.cols + col;
  Vals<VEC> sum{};
  bool first_run = true;
  for (int e0 = 0; e0 < count; e0 += 8) {
    Vals<VEC> v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      v[k] = Vals<VEC>{};
      if (e0 + k < count) {
        const long long src = (long long)ssrc[e0 + k] * a.cols;
        if constexpr (FIRST) v[k] = load_vals<VEC>(dw + src);
        else v[k] = load_vals<VEC>(bw + src);
      }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int e = e0 + k;
      if (e >= count) break;
#pragma unroll
      for (int j = 0; j < VEC; ++j) sum.v[j] += v[k].v[j];
      const bool last = e + 1 == count;
      if (!last && skey[e + 1] == skey[e]) continue;
      if (first_run && open_left) {
        store_vals<VEC>(sw, sum);
      } else if (last && open_right) {
        store_vals<VEC>(sw + a.cols, sum);
      } else {
        float* g = gw + (long long)skey[e] * a.cols;
        Vals<VEC> o{};
        if (accumulate) o = load_vals<VEC>(g);
#pragma unroll
        for (int j = 0; j < VEC; ++j) o.v[j] = fmaf(scale, sum.v[j], o.v[j]);
        store_vals<VEC>(g, o);
      }
      sum = Vals<VEC>{};
      first_run = false;
    }
  }
}

// ---- launches ----------------------------------------------------------------------------------------------------

static size_t align256(size_t x) { return (x + 255) / 256 * 256; }

// Workspace of the gradient: two (row, position) lists, the radix sort's histograms, the levels' slots.
struct EmbPlan {
  size_t keys[2], pos[2], hist, slots[2], total;
  int n_tiles;
};
static EmbPlan emb_plan(int W, int cols, long long n) {
  EmbPlan p{};
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t at = o; o = align256(o + bytes); return at; };
  const bool radix = n > kRankMost;
  for (int k = 0; k < 2; ++k) {
    p.keys[k] = take(k == 0 || radix ? sizeof(unsigned) * (size_t)W * n : 0);
    p.pos[k] = take(k == 0 || radix ? sizeof(unsigned) * (size_t)W * n : 0);
  }
  p.n_tiles = (int)((n + kSortTile - 1) / kSortTile);
  p.hist = take(radix ? sizeof(unsigned) * (size_t)W * 256 * p.n_tiles : 0);
  // slots of the first level, and of the second (the third uses the first's again, and so on)
  const long long c1 = (n + kChunk - 1) / kChunk, c2 = (c1 + kChunk - 1) / kChunk;
  p.slots[0] = take(c1 > 1 ? sizeof(float) * (size_t)W * c1 * 2 * cols : 0);
  p.slots[1] = take(c2 > 1 ? sizeof(float) * (size_t)W * c2 * 2 * cols : 0);
  p.total = o < 256 ? 256 : o;
  return p;
}

size_t embedding_workspace(const acc_ctx* ctx, int layer, long long n) {
  return emb_plan(ctx->cfg.n_workers, ctx->plan.layers[layer].cols, n).total;
}

template <typename Tok, typename Out, int VEC>
static void lookup(const DevLayer& L, const float* params, const void* tokens, long long n, float scale, void* out,
                   int* status, cudaStream_t s) {
  embedding_lookup_kernel<Tok, Out, VEC><<<(unsigned)((n + 7) / 8), 256, 0, s>>>(
      params + L.offset, L.rows, L.cols, static_cast<const Tok*>(tokens), n, scale, static_cast<Out*>(out), status);
}

cudaError_t launch_embedding_lookup(acc_ctx* ctx, int layer, const float* params, const void* tokens, bool tok64,
                                    long long n, float scale, void* out, bool bf16, cudaStream_t s) {
  const DevLayer& L = ctx->plan.layers[layer];
  {
    PhaseTimer pt(ctx, PH_EMB_LOOKUP, s);
    auto go = [&](auto tok, auto o) {
      using Tok = decltype(tok);
      using Out = decltype(o);
      if (L.vec == 4) lookup<Tok, Out, 4>(L, params, tokens, n, scale, out, ctx->d_status, s);
      else if (L.vec == 2) lookup<Tok, Out, 2>(L, params, tokens, n, scale, out, ctx->d_status, s);
      else lookup<Tok, Out, 1>(L, params, tokens, n, scale, out, ctx->d_status, s);
    };
    if (tok64) bf16 ? go((long long)0, __nv_bfloat16()) : go((long long)0, 0.f);
    else bf16 ? go(0, __nv_bfloat16()) : go(0, 0.f);
  }
  return cudaGetLastError();
}

template <typename In, int VEC>
static void sum_levels(acc_ctx* ctx, const EmbArgs& a, const EmbPlan& p, char* ws, const unsigned* keys,
                       const unsigned* pos, const void* dy, float scale, int accumulate, float* grads, cudaStream_t s) {
  const int W = ctx->cfg.n_workers;
  // columns in equal shares of at most 256 threads
  const int nv = a.cols / VEC, shares = (nv + 255) / 256, threads = ((nv + shares - 1) / shares + 31) / 32 * 32;
  const int block = threads < 64 ? 64 : threads;
  const int per = (nv + block - 1) / block;
  float* slots[2] = {reinterpret_cast<float*>(ws + p.slots[0]), reinterpret_cast<float*>(ws + p.slots[1])};
  long long span = kChunk;
  int chunks = (a.n + kChunk - 1) / kChunk;
  {
    PhaseTimer pt(ctx, PH_EMB_SUM, s);
    embedding_sum_kernel<In, VEC, true><<<(unsigned)((long long)W * chunks * per), block, 0, s>>>(
        static_cast<const In*>(dy), nullptr, keys, pos, a, 1, 0, chunks, per, scale, accumulate, grads, slots[0]);
  }
  for (int level = 1; chunks > 1; ++level) {
    const int below = chunks;
    chunks = (below + kChunk - 1) / kChunk;
    PhaseTimer pt(ctx, PH_EMB_JOIN, s);
    embedding_sum_kernel<float, VEC, false><<<(unsigned)((long long)W * chunks * per), block, 0, s>>>(
        nullptr, slots[(level - 1) & 1], keys, pos, a, (int)span, below, chunks, per, scale, accumulate, grads,
        slots[level & 1]);
    span *= kChunk;
  }
}

cudaError_t launch_embedding_grad(acc_ctx* ctx, int layer, const void* tokens, bool tok64, long long n, float scale,
                                  const void* dy, bool bf16, float* grads, int accumulate, void* workspace,
                                  cudaStream_t s) {
  const DevLayer& L = ctx->plan.layers[layer];
  const int W = ctx->cfg.n_workers;
  EmbArgs a{L.offset, ctx->cfg.worker_stride, (long long)L.rows * L.cols, L.rows, L.cols, (int)n};
  char* ws = static_cast<char*>(workspace);
  const long long pieces = (a.size + kZeroPiece - 1) / kZeroPiece;
  const long long zero_blocks = accumulate ? 0 : pieces * W;
  if (n == 0 && accumulate) return cudaSuccess;
  const EmbPlan p = emb_plan(W, L.cols, n);
  unsigned* keys[2] = {reinterpret_cast<unsigned*>(ws + p.keys[0]), reinterpret_cast<unsigned*>(ws + p.keys[1])};
  unsigned* pos[2] = {reinterpret_cast<unsigned*>(ws + p.pos[0]), reinterpret_cast<unsigned*>(ws + p.pos[1])};
  int at = 0;
  if (n <= kRankMost) {
    const int per_worker = (int)((n + kRankBlock - 1) / kRankBlock), rank_blocks = per_worker * W;
    PhaseTimer pt(ctx, PH_EMB_RANK, s);
    const unsigned grid = (unsigned)(rank_blocks + zero_blocks);
    if (tok64)
      embedding_rank_kernel<long long><<<grid, kRankBlock, 0, s>>>(static_cast<const long long*>(tokens), a, keys[0], pos[0],
                                                                   rank_blocks, per_worker, grads, pieces, ctx->d_status);
    else
      embedding_rank_kernel<int><<<grid, kRankBlock, 0, s>>>(static_cast<const int*>(tokens), a, keys[0], pos[0], rank_blocks,
                                                             per_worker, grads, pieces, ctx->d_status);
  } else {
    unsigned* hist = reinterpret_cast<unsigned*>(ws + p.hist);
    const int blocks = p.n_tiles * W;
    {
      PhaseTimer pt(ctx, PH_EMB_KEYS, s);
      const unsigned grid = (unsigned)(blocks + zero_blocks);
      if (tok64)
        embedding_keys_kernel<long long><<<grid, kSortThreads, 0, s>>>(static_cast<const long long*>(tokens), a, keys[0],
                                                                       pos[0], hist, p.n_tiles, blocks, grads, pieces,
                                                                       ctx->d_status);
      else
        embedding_keys_kernel<int><<<grid, kSortThreads, 0, s>>>(static_cast<const int*>(tokens), a, keys[0], pos[0], hist,
                                                                 p.n_tiles, blocks, grads, pieces, ctx->d_status);
    }
    for (int shift = 0; shift < 32 && (shift == 0 || (a.rows >> shift) != 0); shift += 8) {
      if (shift > 0) {
        PhaseTimer pt(ctx, PH_EMB_HIST, s);
        embedding_hist_kernel<<<blocks, kSortThreads, 0, s>>>(keys[at], a.n, shift, hist, p.n_tiles);
      }
      {
        PhaseTimer pt(ctx, PH_EMB_SCAN, s);
        embedding_scan_kernel<<<W, 1024, 0, s>>>(hist, p.n_tiles);
      }
      {
        PhaseTimer pt(ctx, PH_EMB_SCATTER, s);
        embedding_scatter_kernel<<<blocks, kSortThreads, 0, s>>>(keys[at], pos[at], a.n, shift, hist, p.n_tiles,
                                                                 keys[at ^ 1], pos[at ^ 1]);
      }
      at ^= 1;
    }
  }
  if (n > 0) {
    auto go = [&](auto in) {
      using In = decltype(in);
      if (L.vec == 4) sum_levels<In, 4>(ctx, a, p, ws, keys[at], pos[at], dy, scale, accumulate, grads, s);
      else if (L.vec == 2) sum_levels<In, 2>(ctx, a, p, ws, keys[at], pos[at], dy, scale, accumulate, grads, s);
      else sum_levels<In, 1>(ctx, a, p, ws, keys[at], pos[at], dy, scale, accumulate, grads, s);
    };
    if (bf16) go(__nv_bfloat16());
    else go(0.f);
  }
  return cudaGetLastError();
}

}  // namespace acc
