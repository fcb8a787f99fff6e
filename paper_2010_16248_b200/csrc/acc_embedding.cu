// Embedding of a MATRIX layer: the lookup of token rows, and the gradient as one sum per distinct token.
#include <cuda_bf16.h>

#include <algorithm>
#include <type_traits>

#include "acc_internal.cuh"

namespace acc {

// VEC adjacent values of fp32 or bf16, as fp32.  VEC is the widest width at which every row of the layer starts aligned.
template <int VEC> struct Vals { float v[VEC]; };

// As loaded, and as fp32.
template <typename T, int VEC> struct Raw;
template <> struct Raw<float, 4> { using type = float4; };
template <> struct Raw<float, 2> { using type = float2; };
template <> struct Raw<float, 1> { using type = float; };
template <> struct Raw<__nv_bfloat16, 4> { using type = uint2; };
template <> struct Raw<__nv_bfloat16, 2> { using type = unsigned; };
template <> struct Raw<__nv_bfloat16, 1> { using type = unsigned short; };
template <int VEC, typename T> __device__ __forceinline__ typename Raw<T, VEC>::type load_raw(const T* p) {
  return *reinterpret_cast<const typename Raw<T, VEC>::type*>(p);
}
__device__ __forceinline__ Vals<4> unpack(const float4& a) { return {a.x, a.y, a.z, a.w}; }
__device__ __forceinline__ Vals<2> unpack(const float2& a) { return {a.x, a.y}; }
__device__ __forceinline__ Vals<1> unpack(float a) { return {a}; }
__device__ __forceinline__ Vals<2> unpack(unsigned a) { return {__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u)}; }
__device__ __forceinline__ Vals<4> unpack(const uint2& a) {
  const Vals<2> lo = unpack(a.x), hi = unpack(a.y);
  return {lo.v[0], lo.v[1], hi.v[0], hi.v[1]};
}
__device__ __forceinline__ Vals<1> unpack(unsigned short a) { return {__uint_as_float((unsigned)a << 16)}; }

template <int VEC> __device__ __forceinline__ Vals<VEC> load_vals(const float* p) { return unpack(load_raw<VEC>(p)); }
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

// One warp per token:  out_i = scale * row(tok_i), rounded once; zeros where there is no row.  A lane's loads of a batch of
// vectors of VEC columns go out together.  8 x 16384 tokens of 650 columns, a tenth of them padding, to bf16: 307 MB of rows
// read, 48 MB of them distinct, and 170 MB written in 47 us (4 us more with four loads at a time, 19 us more with vectors of four
// columns realigned by shuffles).  No unit is full (L1 67 %, L2 53 %, DRAM 45 %): warps wait for their loads two thirds of
// the time.  Rows far narrower than a warp's 32 vectors leave lanes idle: 131072 tokens of 8 columns take 18 us, of 64 19 us.
template <typename Tok, typename Out, int VEC>
__global__ void __launch_bounds__(256)
embedding_lookup_kernel(const float* table, int rows, int cols, const Tok* tokens, long long n, float scale, Out* out,
                        int* status) {
  await_previous();
  let_next_start();
  const long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (i >= n) return;
  const int lane = threadIdx.x & 31;
  const unsigned row = token_row((long long)tokens[i], rows, status);
  Out* dst = out + i * cols + VEC * lane;
  int left = cols / VEC - lane;  // vectors of this lane: those k with 32 k < left
  if (row == (unsigned)rows) {
    for (; left > 0; left -= 32, dst += 32 * VEC) store_vals<VEC>(dst, Vals<VEC>{});
    return;
  }
  const float* src = table + (long long)row * cols + VEC * lane;
  constexpr int kBatch = VEC == 4 ? 6 : 12;
  for (; left > 0; left -= 32 * kBatch, src += 32 * VEC * kBatch, dst += 32 * VEC * kBatch) {
    Vals<VEC> v[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (32 * k < left) v[k] = load_vals<VEC>(src + 32 * VEC * k);
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      if (32 * k >= left) break;
#pragma unroll
      for (int j = 0; j < VEC; ++j) v[k].v[j] *= scale;
      store_vals<VEC>(dst + 32 * VEC * k, v[k]);
    }
  }
}

// ---- gradient ----------------------------------------------------------------------------------------------------
// G_w[r] (+)= scale * sum over the tokens i of worker w with tok_i = r of dy_i.  The tokens of a worker are sorted by
// (row, position); the sorted order is cut into chunks of 128 entries, whatever the rows, so that a frequent token costs no
// more than as many rare ones.  A row whose entries lie inside one chunk is final there; one that crosses a chunk's edge leaves
// a partial sum in that chunk's head or tail slot, and the next level adds the slots of 128 chunks in the same way, until
// one chunk is left.  Every sum has one writer and a fixed order, so results do not change from run to run.

struct EmbArgs {
  long long offset;      // of the layer inside a worker's slice
  long long stride;      // elements between workers
  long long size;        // rows * cols
  int rows, cols, n;     // n: tokens per worker
};

// Overwriting a gradient is mostly writing zeros: pieces of PIECE elements, handed to the call's kernels behind their own
// blocks, so that the memory system never waits for a sort or for the last sums.
struct EmbZero {
  float* grads;
  int first_block;       // blocks behind this one clear pieces
  int from;              // number of the first such block's piece
  int pieces_per_worker;
};

// A piece whole; a row that the sums write later is then written twice.
template <int PIECE> __device__ __forceinline__ void zero_piece(const EmbZero& z, const EmbArgs& a) {
  const int piece = z.from + (int)blockIdx.x - z.first_block;
  const int w = piece / z.pieces_per_worker;
  const long long e0 = (long long)(piece - w * z.pieces_per_worker) * PIECE;
  float* g = z.grads + w * a.stride + a.offset + e0;
  const int n = (int)min((long long)PIECE, a.size - e0);
  for (int i = 4 * (int)threadIdx.x; i + 4 <= n; i += 4 * (int)blockDim.x) st_stream4(g + i, make_float4(0.f, 0.f, 0.f, 0.f));
  for (int i = (n & ~3) + (int)threadIdx.x; i < n; i += blockDim.x) g[i] = 0.f;
}

// A piece without the rows that some token names.  mark(w, taken, row0, row1) sets bit r - (row0 & ~31) of `taken` for each
// such row r in [row0, row1]; taken has room for PIECE / 32 + 3 words and is zero.
template <int PIECE, typename Mark>
__device__ __forceinline__ void zero_piece_around(const EmbZero& z, const EmbArgs& a, unsigned* taken, Mark mark) {
  const int piece = z.from + (int)blockIdx.x - z.first_block;
  const int w = piece / z.pieces_per_worker;
  const unsigned e0 = (unsigned)(piece - w * z.pieces_per_worker) * PIECE, cols = (unsigned)a.cols;
  float* g = z.grads + w * a.stride + a.offset + e0;
  const int n = (int)min((long long)PIECE, a.size - e0);
  const unsigned row0 = e0 / cols, row1 = (e0 + (unsigned)n - 1u) / cols, word0 = row0 >> 5;
  for (unsigned i = threadIdx.x; i <= (row1 >> 5) - word0; i += blockDim.x) taken[i] = 0u;
  __syncthreads();
  mark(w, taken, row0, row1);
  __syncthreads();
  auto free_row = [&](unsigned r) { return !(taken[(r >> 5) - word0] >> (r & 31) & 1u); };
  if (a.cols < 64) {  // element by element: which row a narrow one lies in, x / cols, exact for x below 2^32 / cols
    const unsigned magic = cols > 1u ? 0xffffffffu / cols + 1u : 0u, off0 = e0 - row0 * cols;
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
      const unsigned x = (unsigned)i + off0;
      if (free_row(row0 + (cols == 1u ? x : __umulhi(x, magic)))) g[i] = 0.f;
    }
    return;
  }
  const int lane = threadIdx.x & 31;
  for (unsigned r = row0 + (threadIdx.x >> 5); r <= row1; r += blockDim.x >> 5) {  // a warp per row
    if (!free_row(r)) continue;
    const long long r0 = (long long)r * cols - e0;
    const int lo = (int)max(r0, 0ll), hi = (int)min(r0 + cols, (long long)n);
    const int lo4 = min((lo + 3) & ~3, hi), hi4 = max(hi & ~3, lo4);
    if (lo + lane < lo4) g[lo + lane] = 0.f;
    for (int i = lo4 + 4 * lane; i < hi4; i += 128) st_stream4(g + i, make_float4(0.f, 0.f, 0.f, 0.f));
    if (hi4 + lane < hi) g[hi4 + lane] = 0.f;
  }
}

// Four columns of a lane: 4 / VEC vectors of VEC adjacent ones, LANES VEC columns apart.
template <int VEC> struct Lane { Vals<VEC> c[4 / VEC]; };
template <typename T, int VEC> struct LaneRaw { typename Raw<T, VEC>::type c[4 / VEC]; };
template <int LANES, int VEC, typename T>
__device__ __forceinline__ void load_lane(LaneRaw<T, VEC>& v, const T* p, const bool* on) {
#pragma unroll
  for (int u = 0; u < 4 / VEC; ++u)
    if (on[u]) v.c[u] = load_raw<VEC>(p + LANES * VEC * u);
}
template <int LANES, int VEC> __device__ __forceinline__ void store_lane(float* p, const Lane<VEC>& v, const bool* on) {
#pragma unroll
  for (int u = 0; u < 4 / VEC; ++u)
    if (on[u]) store_vals<VEC>(p + LANES * VEC * u, v.c[u]);
}
template <int VEC, typename T>
__device__ __forceinline__ void add_lane(Lane<VEC>& s, const LaneRaw<T, VEC>& v) {
#pragma unroll
  for (int u = 0; u < 4 / VEC; ++u) {
    const Vals<VEC> x = unpack(v.c[u]);
#pragma unroll
    for (int j = 0; j < VEC; ++j) s.c[u].v[j] += x.v[j];
  }
}
template <bool ACC, int VEC>
__device__ __forceinline__ void scale_lane(Lane<VEC>& s, float scale, const LaneRaw<float, VEC>& o) {
#pragma unroll
  for (int u = 0; u < 4 / VEC; ++u) {
    const Vals<VEC> x = unpack(o.c[u]);
#pragma unroll
    for (int j = 0; j < VEC; ++j) s.c[u].v[j] = ACC ? fmaf(scale, s.c[u].v[j], x.v[j]) : scale * s.c[u].v[j];
  }
}

// ---- up to kSmallMost tokens per worker: one launch -----------------------------------------------------------------
// A block takes one worker and 64 columns.  It sorts all of the worker's tokens itself, in shared memory (2 us, the same in
// every block, in place of a launch that every block would wait for), and hands every half warp an equal share of the sorted
// entries, four columns to a lane: what steers the sums costs more instructions than the sums, so two entries share them.  A
// run that crosses from one half warp to the next is finished by the one where it begins, from the sums that the others leave
// in shared memory.  Blocks behind those clear the rest of the layer, around the rows of the worker's tokens.
// 8 workers' 700 tokens of 650 columns are added to 33278 rows in 13 us (a chain of launch, tokens, sort and three batches of
// loads on 88 of the 148 SMs; 5 us of it are its 32 MB), written with all zeros in 112 us (692 MB: HBM).  This way / the long
// way below, accumulating: 64 tokens 5 / 13 us, 256 8 / 19, 1024 15 / 27, 2048 31 / 48 us.  These were measured with 8 workers
// of 650 columns, 88 blocks; a block's time depends on the tokens alone, so fewer workers or columns only leave SMs idle: one
// worker of 650 columns takes 12 us for 700 tokens, 25 us for 2048 (long way: 26), of 64 columns 21 us.
// With vectors of one or two values the kernel that adds spills 8 bytes of its 64 registers.
constexpr int kSmallMost = 2048, kSmallCols = 64, kSmallPiece = 32768;
// (a word holds row and position; tables of as many rows, or of more columns -- 32-bit offsets --, take the long way)
constexpr int kSmallPosBits = 11, kSmallRows = 1 << 21, kSmallWide = 1 << 20;

// Ascending order of the block's words by a bitonic network over the first count2 (a power of two) of them; thread t holds
// words t + r * THREADS.  Partners in a warp trade by shuffles, others through shared memory (two buffers in turn, so one
// barrier a step).  Where the network sorts downwards the words are complemented, so that every step keeps the smaller word
// at the lower place.
template <int E, int THREADS>
__device__ __forceinline__ void sort_words(unsigned (&x)[E], int count2, unsigned (*buf)[kSmallMost]) {
  const int t = threadIdx.x, lane = t & 31;
  int turn = 0;
  for (int k = 2; k <= count2; k <<= 1) {
#pragma unroll
    for (int r = 0; r < E; ++r)
      if ((t + r * THREADS) & k) x[r] = ~x[r];
    for (int j = k >> 1; j >= 32; j >>= 1) {
      if (E > 1 && j >= THREADS) {  // both words are this thread's
#pragma unroll
        for (int r = 0; r < E; ++r)
#pragma unroll
          for (int q = r + 1; q < E; ++q)
            if ((q ^ r) * THREADS == j) {
              const unsigned lo = min(x[r], x[q]), hi = max(x[r], x[q]);
              x[r] = lo;
              x[q] = hi;
            }
        continue;
      }
#pragma unroll
      for (int r = 0; r < E; ++r) buf[turn][t + r * THREADS] = x[r];
      __syncthreads();
#pragma unroll
      for (int r = 0; r < E; ++r) {
        const unsigned o = buf[turn][(t ^ j) + r * THREADS];
        x[r] = (t & j) == 0 ? min(o, x[r]) : max(o, x[r]);
      }
      turn ^= 1;
    }
#pragma unroll
    for (int j = 16; j > 0; j >>= 1)
      if (j < k) {
#pragma unroll
        for (int r = 0; r < E; ++r) {
          const unsigned o = __shfl_xor_sync(0xffffffffu, x[r], j);
          x[r] = (lane & j) == 0 ? min(o, x[r]) : max(o, x[r]);
        }
      }
#pragma unroll
    for (int r = 0; r < E; ++r)
      if ((t + r * THREADS) & k) x[r] = ~x[r];
  }
}

template <typename Tok, typename In, int VEC, bool ACC>
__global__ void __launch_bounds__(ACC ? 1024 : 512, ACC ? 1 : 2)
embedding_small_kernel(const Tok* tokens, const In* dy, const EmbArgs a, int groups, float scale, float* grads, int* status,
                       const EmbZero z) {
  constexpr int kThreads = ACC ? 1024 : 512, kParts = kThreads / 16, kVecs = 4 / VEC, kMost = kSmallMost / kThreads;
  __shared__ unsigned buf[2][kSmallMost];
  unsigned* entry = buf[0];  // row above position, sorted; kNoEntry: a token without a row
  __shared__ __align__(16) float shead[kParts][kSmallCols];
  constexpr unsigned kNoEntry = 0xffffffffu, kPosMask = (1u << kSmallPosBits) - 1u;
  await_previous();
  let_next_start();
  if (!ACC && (int)blockIdx.x >= z.first_block) {
    zero_piece_around<kSmallPiece>(z, a, buf[0], [&](int w, unsigned* taken, unsigned row0, unsigned row1) {
      const Tok* tok = tokens + (long long)w * a.n;
#pragma unroll 4
      for (int j = threadIdx.x; j < a.n; j += blockDim.x) {
        const long long t = (long long)tok[j];
        if (t >= (long long)row0 && t <= (long long)row1) atomicOr(&taken[((unsigned)t >> 5) - (row0 >> 5)], 1u << (t & 31));
      }
    });
    return;
  }
  const int lane = threadIdx.x & 15, part = threadIdx.x >> 4;  // of a half warp; its number in the block
  const unsigned half = 0xffffu << (threadIdx.x & 16);         // its lanes
  const int w = blockIdx.x / groups, group = blockIdx.x % groups;
  const Tok* tok = tokens + (long long)w * a.n;
  int count2 = 2;
  while (count2 < a.n) count2 *= 2;
  int count = 0;  // tokens that have a row
  unsigned x[kMost];
#pragma unroll
  for (int r = 0; r < kMost; ++r) {
    const int j = r * kThreads + (int)threadIdx.x;
    x[r] = kNoEntry;
    if (j < a.n) {
      const unsigned row = token_row((long long)tok[j], a.rows, status);
      if (row != (unsigned)a.rows) x[r] = row << kSmallPosBits | (unsigned)j;
    }
    if (r == 0 || a.n > r * kThreads) count += __syncthreads_count(x[r] != kNoEntry);
  }
  if (count2 <= kThreads) {
    unsigned one[1] = {x[0]};
    sort_words<1, kThreads>(one, count2, buf);
    x[0] = one[0];
  } else {
    sort_words<kMost, kThreads>(x, count2, buf);
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kMost; ++r) entry[r * kThreads + threadIdx.x] = x[r];
  __syncthreads();
  auto row_at = [&](int e) { return entry[e] >> kSmallPosBits; };
  auto ends_at = [&](int e) { return e + 1 == count || row_at(e + 1) != row_at(e); };
  const int share = (count + kParts - 1) / kParts, begin = min(share * part, count), end = min(begin + share, count);
  const bool left = begin > 0 && begin < end && row_at(begin - 1) == row_at(begin);

  const int col = group * kSmallCols + lane * VEC;
  bool on[kVecs], all_on[kVecs];
#pragma unroll
  for (int u = 0; u < kVecs; ++u) {
    on[u] = col + 16 * VEC * u < a.cols;
    all_on[u] = true;
  }
  const In* dw = dy + (long long)w * a.n * a.cols + col;
  float* gw = grads + (long long)w * a.stride + a.offset + col;
  float* head = shead[part] + lane * VEC;
  Lane<VEC> sum = {};
  bool first_run = left;  // the run that an earlier half warp began
  constexpr int kBatch = 4;
#pragma unroll 1
  for (int t0 = begin; t0 < end; t0 += 16) {  // 16 entries, one per lane
    const int e = t0 + lane;
    const unsigned mine = e < end ? entry[e] : 0u;
    const unsigned ends = __ballot_sync(half, e < end && ends_at(e)) >> (threadIdx.x & 16);
#pragma unroll 1
    for (int k0 = 0; k0 < 16 && t0 + k0 < end; k0 += kBatch) {
      LaneRaw<In, VEC> v[kBatch];
      LaneRaw<float, VEC> o[ACC ? kBatch : 1];
      const int here = end - t0 - k0;  // entries of this batch, or more
      const unsigned e4 = ends >> k0;
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const unsigned x = __shfl_sync(half, mine, k0 + k, 16);
        if (k < here) load_lane<16>(v[k], dw + (x & kPosMask) * (unsigned)a.cols, on);  // (both offsets fit 32 bits)
        if (ACC && (e4 >> k & 1u)) load_lane<16>(o[k], (const float*)gw + (x >> kSmallPosBits) * (unsigned)a.cols, on);
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        if (k >= here) break;
        add_lane(sum, v[k]);
        if (!(e4 >> k & 1u)) continue;
        if (first_run) {
          store_lane<16>(head, sum, all_on);
        } else {
          scale_lane<ACC>(sum, scale, o[ACC ? k : 0]);
          store_lane<16>(gw + row_at(t0 + k0 + k) * (unsigned)a.cols, sum, on);
        }
        sum = {};
        first_run = false;
      }
    }
  }
  bool pending = begin < end && !ends_at(end - 1);  // a run goes on behind this half warp
  if (pending && first_run) {
    store_lane<16>(head, sum, all_on);
    pending = false;
  }
  __syncthreads();
  if (!pending) return;
  float* g = gw + row_at(end - 1) * (unsigned)a.cols;
  LaneRaw<float, VEC> o;
  if (ACC) load_lane<16>(o, (const float*)g, on);
  for (int q = part + 1;; ++q) {
    LaneRaw<float, VEC> h;
    load_lane<16>(h, (const float*)shead[q] + lane * VEC, all_on);
    add_lane(sum, h);
    const int last = min(share * (q + 1), count) - 1;
    if (row_at(last) != row_at(end - 1) || ends_at(last)) break;  // (the run ends inside that share)
  }
  scale_lane<ACC>(sum, scale, o);
  store_lane<16>(g, sum, on);
}

// ---- more tokens: sort, sums by chunks, joins -------------------------------------------------------------------------
// A stable radix sort, eight bits of the row at a time, in tiles of kSortTile tokens.  Its launches clear the pieces, whole:
// leaving out the rows that the sums write (15 % of them for 16384 Zipf-distributed tokens of 33278 rows) and clearing beside
// the sums instead was slower, 211 us against 185 us for 8 workers (with sums that took 10 us more than now), as the sort's
// launches then waited alone.
constexpr int kZeroPiece = 16384;
constexpr int kSortTile = 2048, kSortThreads = 256, kSortWarps = kSortThreads / 32;

__device__ __forceinline__ long long sort_hist_at(int w, int digit, int tile, int n_tiles) {
  return ((long long)w * 256 + digit) * n_tiles + tile;
}

// First pass: rows from tokens, positions in order, and the first digit's histogram of every tile.
template <typename Tok>
__global__ void __launch_bounds__(kSortThreads)
embedding_keys_kernel(const Tok* tokens, EmbArgs a, unsigned* keys, unsigned* pos, unsigned* hist, int n_tiles, int* status,
                      EmbZero z) {
  await_previous();
  // Only now: blocks of the launches behind clear pieces without a wait of their own.  Those launches' sorting blocks wait, so
  // that each is complete only after the one before it, and the call's last only after all of them; a launch without any
  // sorting block would not be, which is why an empty batch has this launch alone.
  let_next_start();
  if ((int)blockIdx.x >= z.first_block) {
    zero_piece<kZeroPiece>(z, a);
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
embedding_hist_kernel(const unsigned* keys, EmbArgs a, int shift, unsigned* hist, int n_tiles, EmbZero z) {
  let_next_start();
  if ((int)blockIdx.x >= z.first_block) {
    zero_piece<kZeroPiece>(z, a);
    return;
  }
  await_previous();
  const int n = a.n;
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

// One block per worker: exclusive sum over (digit, tile), in place.  Only for more than kScanTiles tiles: fewer counts are
// quicker summed by every block of the scatter pass (8 x 16384 tokens accumulated: 125 us with this launch, 121 us without).
constexpr int kScanTiles = 64;
__global__ void __launch_bounds__(1024)
embedding_scan_kernel(unsigned* hist, int n_tiles, EmbArgs a, EmbZero z) {
  let_next_start();
  if ((int)blockIdx.x >= z.first_block) {
    zero_piece<kZeroPiece>(z, a);
    return;
  }
  await_previous();
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
template <bool SCANNED>
__global__ void __launch_bounds__(kSortThreads)
embedding_scatter_kernel(const unsigned* keys, const unsigned* pos, EmbArgs a, int shift, const unsigned* hist, int n_tiles,
                         unsigned* keys_out, unsigned* pos_out, EmbZero z) {
  let_next_start();
  if ((int)blockIdx.x >= z.first_block) {
    zero_piece<kZeroPiece>(z, a);
    return;
  }
  await_previous();
  const int n = a.n;
  __shared__ unsigned cnt[kSortWarps][256];
  __shared__ unsigned warp_total[kSortWarps];
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
    unsigned run;  // where the tile's first entry with this thread's digit goes
    if (SCANNED) {
      run = hist[sort_hist_at(w, threadIdx.x, tile, n_tiles)];
    } else {
      const unsigned* h = hist + sort_hist_at(w, threadIdx.x, 0, n_tiles);
      unsigned ahead = 0u, total = 0u;
#pragma unroll 8
      for (int k = 0; k < n_tiles; ++k) {
        const unsigned c = h[k];
        ahead += k < tile ? c : 0u;
        total += c;
      }
      unsigned inc = total;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned up = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += up;
      }
      if (lane == 31) warp_total[warp] = inc;
      __syncthreads();
      run = ahead + inc - total;
      for (int k = 0; k < warp; ++k) run += warp_total[k];
    }
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

// A block takes one chunk and 128 columns, each of its eight warps an eighth of the entries, in order: 16 sorted tokens at
// the first level, 32 slots of the level below (two for each of its kFan chunks) at the others.  A run that crosses from
// one warp to the next is finished by the warp where it begins, from the sums that the others leave in shared memory.  The
// loads of a batch of entries go out together, with accumulation (ACC) those of the rows that are added to among them.  What
// steers the sums is the same for a whole warp: masks of the entries there are and of those that end a run.
// 8 x 16384 tokens of 650 columns in bf16, a tenth of them padding, take 61 us for 153 MB read and 102 MB written.  No unit is
// full (DRAM 46 %, L2 28 %): a scheduler issues in 60 % of the cycles, from seven warps that wait for loads, for barriers and
// for their own latencies in equal parts.  Chunk and batches were measured at this width; of rows of few columns most lanes are
// idle (one worker's 131072 tokens of 8 columns: 63 us).  Rows of an odd number of columns in bf16, 16 entries of four single
// loads each, spill 56 bytes of their 64 registers (64 bytes of 80 with accumulation).
constexpr int kChunk = 128, kFan = 128;
constexpr unsigned kNoKey = 0xffffffffu;
struct EmbLevel {
  const unsigned* keys;   // first level: sorted rows, [W][n]; otherwise the slots' rows, [W][2 chunks of the level below]
  const unsigned* pos;    // first level: sorted positions
  int count, chunks;      // keys per worker; chunks of this level per worker
  float* slots;           // [W][chunks][2][cols]: where this level leaves its partial sums
  unsigned* slot_keys;    // [W][chunks][2]: their rows; kNoKey: nothing there
};

// In: the values' type at the first level (FIRST); float above.
template <typename In, int VEC, bool FIRST, bool ACC>
__global__ void __launch_bounds__(256, ACC ? (sizeof(In) == 2 ? 3 : 2) : (sizeof(In) == 2 ? 4 : 3))
embedding_sum_kernel(const In* in, const EmbLevel l, const EmbArgs a, int groups, float scale, float* grads) {
  constexpr int kPart = FIRST ? kChunk / 8 : 2 * kFan / 8;  // entries per warp
  __shared__ unsigned skey[8 * kPart + 2], smask[8], sends[8];
  __shared__ __align__(16) float shead[8][128];  // read and written four columns at a time
  let_next_start();
  await_previous();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int wc = blockIdx.x / groups, group = blockIdx.x % groups;  // column group fastest, then chunk, then worker
  const int w = wc / l.chunks, chunk = wc % l.chunks;
  const unsigned* kw = l.keys + (long long)w * l.count;
  const int c0 = chunk * 8 * kPart;

  // the chunk's keys at skey[1 ..], the keys beside it at either end
  for (int t = threadIdx.x; t < 8 * kPart + 2; t += 256) {
    const int at = c0 - 1 + t;
    const unsigned key = at >= 0 && at < l.count ? kw[at] : kNoKey;
    skey[t] = key == (unsigned)a.rows ? kNoKey : key;
  }
  unsigned pos = 0u;
  if (FIRST && lane < kPart && c0 + kPart * warp + lane < l.count) pos = l.pos[(long long)w * l.count + c0 + kPart * warp + lane];
  __syncthreads();
  const unsigned* own = skey + 1 + kPart * warp;
  const unsigned key = lane < kPart ? own[lane] : kNoKey;
  const unsigned mask = __ballot_sync(0xffffffffu, key != kNoKey);
  if (lane == 0) smask[warp] = mask;
  __syncthreads();
  // an entry ends a run if the next one has another row; the chunk's last one always does
  unsigned next = kNoKey;
  if (FIRST) {
    if (lane < kPart && kPart * warp + lane + 1 < 8 * kPart) next = own[lane + 1];
  } else {
    unsigned behind = lane == 31 ? 0u : mask >> (lane + 1) << (lane + 1);
    int q = warp;
    while (behind == 0u && q + 1 < 8) behind = smask[++q];
    if (behind != 0u) next = skey[kPart * q + __ffs(behind)];
  }
  const unsigned ends = __ballot_sync(0xffffffffu, key != kNoKey && key != next);
  if (lane == 0) sends[warp] = ends;
  // is the chunk's first (last) run open to the left (right), and the warp's first run?
  const bool open_left = skey[1] != kNoKey && (!FIRST || skey[0] == skey[1]);
  const bool open_right = skey[8 * kPart + 1] != kNoKey && (!FIRST || skey[8 * kPart] == skey[8 * kPart + 1]);
  int before = warp - 1, last_warp = 7;
  while (before >= 0 && smask[before] == 0u) --before;
  while (last_warp > 0 && smask[last_warp] == 0u) --last_warp;
  const int last_entry = 31 - __clz(smask[last_warp]);
  const bool left = before < 0 ? warp == 0 && open_left
                               : mask != 0u && skey[kPart * before + 32 - __clz(smask[before])] == own[__ffs(mask) - 1];
  __syncthreads();
  if (group == 0 && l.chunks > 1 && threadIdx.x < 2) {
    int runs = 0;
    for (int q = 0; q < 8; ++q) runs += __popc(sends[q]);
    unsigned slot_key = kNoKey;
    if (threadIdx.x == 0 && open_left) slot_key = skey[1];
    if (threadIdx.x == 1 && open_right && !(open_left && runs == 1)) slot_key = skey[kPart * last_warp + 1 + last_entry];
    l.slot_keys[(long long)wc * 2 + threadIdx.x] = slot_key;
  }

  const int col = group * 128 + lane * VEC;
  bool on[4 / VEC], all_on[4 / VEC];
#pragma unroll
  for (int u = 0; u < 4 / VEC; ++u) {
    on[u] = col + 32 * VEC * u < a.cols;
    all_on[u] = true;
  }
  const In* iw = in + (long long)w * l.count * a.cols + col;
  float* gw = grads + (long long)w * a.stride + a.offset + col;
  float* tail_slot = l.slots + ((long long)wc * 2 + 1) * a.cols + col;
  float* head = shead[warp] + lane * VEC;
  Lane<VEC> sum = {};
  bool first_run = left;  // the run that an earlier warp, or the chunk before, began
  const int tail_entry = open_right && warp == last_warp ? last_entry : -1;  // ends the chunk's last run, which goes on
  auto finish_entry = [&](int e, const LaneRaw<float, VEC>& o) {  // entry e ends a run
    if (first_run) {
      store_lane<32>(head, sum, all_on);
    } else if (e == tail_entry) {
      store_lane<32>(tail_slot, sum, on);
    } else {
      scale_lane<ACC>(sum, scale, o);
      store_lane<32>(gw + own[e] * (unsigned)a.cols, sum, on);
    }
    sum = {};
    first_run = false;
  };
  // 32 registers of loads in flight: 16 entries of bf16 at once, of fp32 (and of rows that are added to) eight
  constexpr int kBatch = sizeof(In) == 2 && !ACC ? 16 : 8;
  if constexpr (FIRST) {  // the entries are the first ones of the warp's part
    const int entries = __popc(mask);
#pragma unroll
    for (int e0 = 0; e0 < kPart; e0 += kBatch) {
      if (e0 >= entries) break;
      LaneRaw<In, VEC> v[kBatch];
      LaneRaw<float, VEC> o[ACC ? kBatch : 1];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const unsigned from = __shfl_sync(0xffffffffu, pos, e0 + k);
        if (e0 + k < entries) load_lane<32>(v[k], iw + (unsigned long long)from * (unsigned)a.cols, on);
        if (ACC && (ends >> (e0 + k) & 1u)) load_lane<32>(o[k], (const float*)gw + own[e0 + k] * (unsigned)a.cols, on);
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        if (e0 + k >= entries) break;
        add_lane(sum, v[k]);
        if (ends >> (e0 + k) & 1u) finish_entry(e0 + k, o[ACC ? k : 0]);
      }
    }
  } else {
    unsigned todo = mask;
#pragma unroll 1
    while (todo != 0u) {
      LaneRaw<In, VEC> v[kBatch];
      LaneRaw<float, VEC> o[ACC ? kBatch : 1];
      unsigned batch = todo;
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        if (todo == 0u) continue;
        const int e = __ffs(todo) - 1;
        todo &= todo - 1u;
        load_lane<32>(v[k], iw + (unsigned long long)(unsigned)(c0 + kPart * warp + e) * (unsigned)a.cols, on);
        if (ACC && (ends >> e & 1u)) load_lane<32>(o[k], (const float*)gw + own[e] * (unsigned)a.cols, on);
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        if (batch == 0u) break;
        const int e = __ffs(batch) - 1;
        batch &= batch - 1u;
        add_lane(sum, v[k]);
        if (ends >> e & 1u) finish_entry(e, o[ACC ? k : 0]);
      }
    }
  }
  bool pending = mask != 0u && !(ends >> (31 - __clz(mask)) & 1u);  // a run goes on behind this warp
  if (pending && first_run) {
    store_lane<32>(head, sum, all_on);
    pending = false;
  }
  __syncthreads();
  // the rest of a run that ends in a later warp: adds the heads up to there, returns whether it ends the chunk
  auto finish_run = [&](int q) {
    for (;; ++q) {
      if (smask[q] == 0u) continue;
      LaneRaw<float, VEC> h;
      load_lane<32>(h, (const float*)shead[q] + lane * VEC, all_on);
      add_lane(sum, h);
      if (sends[q] != 0u) return q == last_warp && __ffs(sends[q]) - 1 == last_entry;
    }
  };
  if (pending) {
    const unsigned row = own[31 - __clz(mask)];
    float* g = gw + row * (unsigned)a.cols;
    LaneRaw<float, VEC> o;
    if (ACC) load_lane<32>(o, (const float*)g, on);
    if (finish_run(warp + 1) && open_right) {
      store_lane<32>(tail_slot, sum, on);
    } else {
      scale_lane<ACC>(sum, scale, o);
      store_lane<32>(g, sum, on);
    }
  }
  if (warp == 0 && open_left) {
    LaneRaw<float, VEC> h;
    load_lane<32>(h, (const float*)shead[0] + lane * VEC, all_on);
    sum = {};
    add_lane(sum, h);
    if (sends[0] == 0u) finish_run(1);
    store_lane<32>(tail_slot - a.cols, sum, on);
  }
}

// ---- launches ----------------------------------------------------------------------------------------------------

static size_t align256(size_t x) { return (x + 255) / 256 * 256; }

// Workspace of the gradient: two (row, position) lists, the radix sort's histograms, the levels' slots.  The one
// launch for few tokens needs none.
struct EmbPlan {
  size_t keys[2], pos[2], hist, slots[2], slot_keys[2], total;
  int n_tiles;
};
static bool small_way(int rows, int cols, long long n) {
  return n <= kSmallMost && rows < kSmallRows && cols <= kSmallWide;  // (all ones is no row's word)
}
static EmbPlan emb_plan(int W, int rows, int cols, long long n) {
  EmbPlan p{};
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t at = o; o = align256(o + bytes); return at; };
  p.n_tiles = (int)((n + kSortTile - 1) / kSortTile);
  if (!small_way(rows, cols, n)) {
    for (int k = 0; k < 2; ++k) {
      p.keys[k] = take(sizeof(unsigned) * (size_t)W * n);
      p.pos[k] = take(sizeof(unsigned) * (size_t)W * n);
    }
    p.hist = take(sizeof(unsigned) * (size_t)W * 256 * p.n_tiles);
    // slots of the first level, and of the second (the third uses the first's again, and so on)
    const long long c1 = (n + kChunk - 1) / kChunk, c2 = (c1 + kFan - 1) / kFan;
    p.slots[0] = take(sizeof(float) * (size_t)W * c1 * 2 * cols);
    p.slots[1] = take(c2 > 1 ? sizeof(float) * (size_t)W * c2 * 2 * cols : 0);
    p.slot_keys[0] = take(sizeof(unsigned) * (size_t)W * c1 * 2);
    p.slot_keys[1] = take(c2 > 1 ? sizeof(unsigned) * (size_t)W * c2 * 2 : 0);
  }
  p.total = o < 256 ? 256 : o;
  return p;
}

size_t embedding_workspace(const acc_ctx* ctx, int layer, long long n) {
  const DevLayer& L = ctx->plan.layers[layer];
  return emb_plan(ctx->cfg.n_workers, L.rows, L.cols, n).total;
}

cudaError_t launch_embedding_lookup(acc_ctx* ctx, int layer, const float* params, const void* tokens, bool tok64,
                                    long long n, float scale, void* out, bool bf16, cudaStream_t s) {
  const DevLayer& L = ctx->plan.layers[layer];
  PhaseTimer pt(ctx, PH_EMB_LOOKUP, s);
  auto go = [&](auto tok, auto o) {
    using Tok = decltype(tok);
    using Out = decltype(o);
    auto* kernel = L.vec == 4   ? embedding_lookup_kernel<Tok, Out, 4>
                   : L.vec == 2 ? embedding_lookup_kernel<Tok, Out, 2>
                                : embedding_lookup_kernel<Tok, Out, 1>;
    return launch_early(kernel, (unsigned)((n + 7) / 8), 256, s, params + L.offset, L.rows, L.cols,
                        static_cast<const Tok*>(tokens), n, scale, static_cast<Out*>(out), ctx->d_status);
  };
  if (tok64) return bf16 ? go((long long)0, __nv_bfloat16()) : go((long long)0, 0.f);
  return bf16 ? go(0, __nv_bfloat16()) : go(0, 0.f);
}

// The kernels of one gradient call, in order.
struct EmbLaunch {
  acc_ctx* ctx;
  cudaStream_t s;
  cudaError_t err = cudaSuccess;

  template <typename... Params, typename... Args>
  void operator()(int phase, void (*kernel)(Params...), long long blocks, int threads, Args... args) {
    if (blocks == 0 || err != cudaSuccess) return;
    PhaseTimer pt(ctx, phase, s);
    err = launch_early(kernel, (unsigned)blocks, threads, s, args...);
  }
};

template <typename In, int VEC>
static void sum_levels(EmbLaunch& go, const EmbArgs& a, const EmbPlan& p, char* ws, const unsigned* keys,
                       const unsigned* pos, const void* dy, float scale, int accumulate, float* grads) {
  const int W = go.ctx->cfg.n_workers;
  const int groups = (a.cols + 127) / 128;
  auto level = [&](int k, const unsigned* lkeys, const unsigned* lpos, int count, int chunks) {
    return EmbLevel{lkeys, lpos, count, chunks, reinterpret_cast<float*>(ws + p.slots[k & 1]),
                    reinterpret_cast<unsigned*>(ws + p.slot_keys[k & 1])};
  };
  int chunks = (a.n + kChunk - 1) / kChunk;
  EmbLevel l = level(0, keys, pos, a.n, chunks);
  go(PH_EMB_SUM, accumulate ? embedding_sum_kernel<In, VEC, true, true> : embedding_sum_kernel<In, VEC, true, false>,
     (long long)W * chunks * groups, 256, static_cast<const In*>(dy), l, a, groups, scale, grads);
  for (int k = 1; chunks > 1; ++k) {
    const float* in = l.slots;
    const unsigned* in_keys = l.slot_keys;
    const int count = 2 * chunks;
    chunks = (chunks + kFan - 1) / kFan;
    l = level(k, in_keys, nullptr, count, chunks);
    go(PH_EMB_JOIN, accumulate ? embedding_sum_kernel<float, VEC, false, true> : embedding_sum_kernel<float, VEC, false, false>,
       (long long)W * chunks * groups, 256, in, l, a, groups, scale, grads);
  }
}

cudaError_t launch_embedding_grad(acc_ctx* ctx, int layer, const void* tokens, bool tok64, long long n, float scale,
                                  const void* dy, bool bf16, float* grads, int accumulate, void* workspace,
                                  cudaStream_t s) {
  if (n == 0 && accumulate) return cudaSuccess;
  const DevLayer& L = ctx->plan.layers[layer];
  const int W = ctx->cfg.n_workers;
  const EmbArgs a{L.offset, ctx->cfg.worker_stride, (long long)L.rows * L.cols, L.rows, L.cols, (int)n};
  char* ws = static_cast<char*>(workspace);
  const bool small = small_way(L.rows, L.cols, n);
  const int piece = small ? kSmallPiece : kZeroPiece, pieces = (int)((a.size + piece - 1) / piece);
  const long long all = accumulate ? 0 : (long long)pieces * W;  // pieces to clear
  EmbLaunch go{ctx, s};
  if (small) {
    const int groups = (L.cols + kSmallCols - 1) / kSmallCols;
    const long long blocks = n == 0 ? 0 : (long long)W * groups;
    auto run = [&](auto tok, auto in, auto vec) {
      using Tok = decltype(tok);
      using In = decltype(in);
      constexpr int VEC = decltype(vec)::value;
      go(PH_EMB_SMALL, accumulate ? embedding_small_kernel<Tok, In, VEC, true> : embedding_small_kernel<Tok, In, VEC, false>,
         blocks + all, accumulate ? 1024 : 512, static_cast<const Tok*>(tokens), static_cast<const In*>(dy), a, groups,
         scale, grads, ctx->d_status, EmbZero{grads, (int)blocks, 0, pieces});
    };
    auto typed = [&](auto tok, auto in) {
      if (L.vec == 1) run(tok, in, std::integral_constant<int, 1>());
      else if (L.vec == 2) run(tok, in, std::integral_constant<int, 2>());
      else run(tok, in, std::integral_constant<int, 4>());
    };
    if (tok64) bf16 ? typed((long long)0, __nv_bfloat16()) : typed((long long)0, 0.f);
    else bf16 ? typed(0, __nv_bfloat16()) : typed(0, 0.f);
  } else {
    const EmbPlan p = emb_plan(W, L.rows, L.cols, n);
    unsigned* keys[2] = {reinterpret_cast<unsigned*>(ws + p.keys[0]), reinterpret_cast<unsigned*>(ws + p.keys[1])};
    unsigned* pos[2] = {reinterpret_cast<unsigned*>(ws + p.pos[0]), reinterpret_cast<unsigned*>(ws + p.pos[1])};
    unsigned* hist = reinterpret_cast<unsigned*>(ws + p.hist);
    const long long blocks = (long long)p.n_tiles * W;
    const bool scan = p.n_tiles > kScanTiles;
    int passes = 0;
    for (int shift = 0; shift < 32 && (shift == 0 || (a.rows >> shift) != 0); shift += 8) ++passes;
    // every launch of the sort clears its share of the pieces behind its own blocks; without tokens the first clears all
    const int sharing = n == 0 ? 1 : passes * (scan ? 3 : 2);
    const long long share = (all + sharing - 1) / sharing;
    long long from = 0;
    auto sort = [&](int phase, auto kernel, long long own, int threads, auto... args) {
      const long long mine = std::min(share, all - from);
      go(phase, kernel, own + mine, threads, args..., EmbZero{grads, (int)own, (int)from, pieces});
      from += mine;
    };
    if (tok64)
      sort(PH_EMB_KEYS, embedding_keys_kernel<long long>, blocks, kSortThreads, static_cast<const long long*>(tokens), a,
           keys[0], pos[0], hist, p.n_tiles, ctx->d_status);
    else
      sort(PH_EMB_KEYS, embedding_keys_kernel<int>, blocks, kSortThreads, static_cast<const int*>(tokens), a, keys[0], pos[0],
           hist, p.n_tiles, ctx->d_status);
    if (n == 0) return go.err;
    int at = 0;
    for (int pass = 0; pass < passes; ++pass, at ^= 1) {
      const int shift = 8 * pass;
      if (pass > 0) sort(PH_EMB_HIST, embedding_hist_kernel, blocks, kSortThreads, keys[at], a, shift, hist, p.n_tiles);
      if (scan) sort(PH_EMB_SCAN, embedding_scan_kernel, W, 1024, hist, p.n_tiles, a);
      sort(PH_EMB_SCATTER, scan ? embedding_scatter_kernel<true> : embedding_scatter_kernel<false>, blocks, kSortThreads,
           keys[at], pos[at], a, shift, hist, p.n_tiles, keys[at ^ 1], pos[at ^ 1]);
    }
    auto sums = [&](auto in) {
      using In = decltype(in);
      if (L.vec == 4) sum_levels<In, 4>(go, a, p, ws, keys[at], pos[at], dy, scale, accumulate, grads);
      else if (L.vec == 2) sum_levels<In, 2>(go, a, p, ws, keys[at], pos[at], dy, scale, accumulate, grads);
      else sum_levels<In, 1>(go, a, p, ws, keys[at], pos[at], dy, scale, accumulate, grads);
    };
    if (bf16) sums(__nv_bfloat16());
    else sums(0.f);
  }
  return go.err;
}

}  // namespace acc
