// Weight gradient of a linear layer from a checkpoint of its input: G_w (+)= scale * sum over the tokens t of dy_wt x_wt^T, a
// matrix product on the tensor cores that writes the workers' fp32 gradients.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <type_traits>

#include "acc_async.cuh"
#include "acc_internal.cuh"

namespace acc {

// Two blocks on neighbouring SMs work on one tile of 256 rows of the layer (the product's M, 128 a block) by up to 256 columns
// (N, half of them loaded by each block); a step is 64 tokens (K).  Both operands lie in memory with the tokens outermost, so a
// stage holds them with M (N) contiguous: boxes of 64 elements (128 bytes) x 64 tokens in the 128-byte swizzle, 16-byte chunk c
// of token k at chunk c ^ (k & 7).
constexpr int kM = 128, kK = 64;
constexpr int kBoxBytes = 64 * 128;
constexpr int kABytes = kM / 64 * kBoxBytes;
constexpr int kEpiPitch = 41;  // floats of a row of 8 + 32 finished sums, odd: a column's 32 rows lie in 32 banks
enum { kEpiWarps = 8, kMmaWarp = 8, kDyWarp = 9, kXWarp = 10, kLoadWarp = 12, kLoadWarps = 8 };

// How dy reaches shared memory: bf16 by tensor copies, or (rows that do not start on 16 bytes; fp32) by loads.
enum DyPath { DY_TMA, DY_BF16, DY_F32 };
template <DyPath P> struct LinCfg {
  // fp32 values are three bf16 terms each (8 bits of the 24 apiece), so that the products stay those of fp32
  static constexpr int parts = P == DY_F32 ? 3 : 1;
  // columns of a tile: each of the eight warps that write it holds half of them for 32 rows, a lane's in registers, which the
  // loading warps leave fewer of
  static constexpr int n = P == DY_TMA ? 256 : 128;
  static constexpr int b_bytes = n / 128 * kBoxBytes;
  static constexpr int stage = kABytes * parts + b_bytes;
  static constexpr int stages = P == DY_F32 ? 3 : P == DY_BF16 ? 6 : 5;
  static constexpr int threads = 32 * (P == DY_TMA ? kLoadWarp : kLoadWarp + kLoadWarps);
  static constexpr int smem = stages * stage + kEpiWarps * 32 * kEpiPitch * 4 + 1024;
  // Registers a thread: the sums' warps take what the others give back, within what the block was launched with.
  static constexpr int launch_regs = P == DY_TMA ? 168 : 96, load_regs = 88;
  static constexpr int epi_regs = P == DY_TMA ? 216 : 128, mma_regs = P == DY_TMA ? 56 : 40;
  static_assert(kEpiWarps * epi_regs + 4 * mma_regs + (threads / 32 - kLoadWarp) * load_regs <= threads / 32 * launch_regs, "");
  // Most steps whose sum stays in the tensor core.  It cuts its sums where fp32 adds round: 44 products of 16 tokens in one sum
  // are 8e-7 off, 1024 of them 1e-5.  So a sum ends after 24 products at most (as many of fp32's three terms) and is added to
  // the others in registers.
  static constexpr int chunk = P == DY_F32 ? 2 : 6;
};

struct LinArgs {
  const void* dy;
  long long ld, dy_stride;      // elements between tokens, between workers
  int n, rows, cols;
  float* out;                   // worker w's (split s's) layer at out + (s * W + w) * out_stride
  long long out_stride;
  float scale;
  int accumulate;
  int W, m_tiles, n_tiles, splits, steps, tile_n;  // tile_n: columns of a tile, a multiple of 32
  int* status;
};

struct LinTile { int split, w, m, n, from, to; };  // steps [from, to)
__device__ __forceinline__ LinTile lin_tile(const LinArgs& a, int t) {
  LinTile x;
  x.n = t % a.n_tiles; t /= a.n_tiles;
  x.m = t % a.m_tiles; t /= a.m_tiles;
  x.w = t % a.W;
  x.split = t / a.W;
  x.from = (int)((long long)a.steps * x.split / a.splits);
  x.to = (int)((long long)a.steps * (x.split + 1) / a.splits);
  return x;
}

// The parts of a tile's steps that are summed on their own, as even as they come.
template <int CHUNK> __device__ __forceinline__ int lin_chunks(const LinTile& x) { return (x.to - x.from + CHUNK - 1) / CHUNK; }

// ---- tensor core, tensor memory, the pair of blocks -----------------------------------------------------------------
__device__ __forceinline__ void tmem_alloc(uint32_t* where) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(where)) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t at) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(at));
}
__device__ __forceinline__ void tc_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// One arrival on this barrier in both blocks once the products issued so far are done.
__device__ __forceinline__ void tc_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
                   smem_u32(bar)), "h"((unsigned short)3)
               : "memory");
}
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile(
      "{\n"
      "  .reg .pred p;\n"
      "  setp.ne.u32 p, %4, 0;\n"
      "  tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n"
      "}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((unsigned)add)
      : "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t at, uint32_t* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(at));
}
__device__ __forceinline__ void tmem_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Shared-memory descriptor of an operand whose M (N) is contiguous: 128-byte swizzle, 64 elements of M a box, boxes kBoxBytes
// apart, groups of 8 tokens 1024 bytes apart inside a box.
__device__ __forceinline__ uint64_t operand_desc(uint32_t smem) {
  return (uint64_t)((smem & 0x3ffff) >> 4) | (uint64_t)(kBoxBytes >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 |
         (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// fp32 sums of bf16 products, both operands with M (N) contiguous, M of the pair.
__device__ __forceinline__ uint32_t mma_desc(int n) {
  return 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | 1u << 16 | (uint32_t)(n >> 3) << 17 | (uint32_t)(2 * kM >> 4) << 24;
}
// A copy into this block's stage that counts on the first block's barrier.
__device__ __forceinline__ void tma_load(void* dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
  asm volatile(
      "{\n"
      "  .reg .b32 there;\n"
      "  mapa.shared::cluster.u32 there, %5, 0;\n"
      "  cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4}], [there];\n"
      "}\n" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
      : "memory");
}
// An arrival on the first block's barrier, from either block.
__device__ __forceinline__ void mbar_arrive_first(uint64_t* bar) {
  asm volatile(
      "{\n"
      "  .reg .b32 there;\n"
      "  mapa.shared::cluster.u32 there, %0, 0;\n"
      "  mbarrier.arrive.shared::cluster.b64 _, [there];\n"
      "}\n" ::"r"(smem_u32(bar))
      : "memory");
}
template <int N> __device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
// True in one lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
  unsigned ok;
  asm volatile(
      "{\n"
      "  .reg .pred p;\n"
      "  elect.sync _|p, 0xffffffff;\n"
      "  selp.u32 %0, 1, 0, p;\n"
      "}\n"
      : "=r"(ok));
  return ok != 0;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
struct LinShared {
  uint64_t full[6], empty[6], acc_full[2], acc_empty[2], drain;
  uint32_t tmem;
};

// A wait of a role; when it gives up, the call's status says so and the role ends, and with it, by their own limits, the others.
// (Waits and remote arrivals of block scope: what they order lies in shared memory, which has no copies; the cluster's scope
// costs each a fence of the whole memory, four times the time of a step's products.)
__device__ __forceinline__ bool lin_wait(uint64_t* bar, unsigned parity, int* status) {
  if (mbar_wait_bounded(bar, parity)) return true;
  atomicCAS(status, 0, ACC_ETIMEOUT);
  return false;
}

// A warp's 32 rows of finished sums, `cols` columns of each lane's row held[], times scale, to or onto rows of the layer.
// Blocks of 32 columns turn in shared memory.  A row may start at any element, and a store that ends inside 32 bytes of memory
// costs as much as two: so a row's block begins up to seven columns early, where 32 bytes do, and the block before leaves
// those to it.  Rows eight apart start at the same place within 32 bytes and go together, one address for four of them.  (Rows
// of 650 columns, the writing alone: 2.5 TB/s with blocks from the first column, 3.9 with an address each, 5.2 so.)
// The code stays small -- one copy of the part that writes, for all blocks: unrolled, it cost 30 us of 300 in instruction
// fetches.
template <bool ADD, bool WHOLE>
__device__ __forceinline__ void write_block(uint32_t at, float* out, int start, int ld, int c, int cols, int rows, int lane) {
  const long long step = 8ll * ld;
#pragma unroll WHOLE ? 8 : 1
  for (int k = 0; k < 8; ++k) {
    const int early = (start + k * ld) & 7, col = c - early + lane;
    if ((unsigned)col >= (unsigned)cols) continue;
    const uint32_t from = at + 4 * (k * kEpiPitch + 8 - early + lane);
    float* p = out + (long long)k * ld + col;
    float v[4], old[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v[r]) : "r"(from + 4 * 8 * r * kEpiPitch));
      if (ADD && (WHOLE || k + 8 * r < rows)) old[r] = p[r * step];
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if (WHOLE || k + 8 * r < rows) *p = ADD ? old[r] + v[r] : v[r];
      p += step;
    }
  }
}
template <int HELD>
__device__ __forceinline__ void write_rows(const float (&held)[HELD], float scale, bool add, float* buf, float* out, int ld, int cols,
                                           int rows, int lane) {
  const int start = (int)(reinterpret_cast<uintptr_t>(out) >> 2);
  const uint32_t at = smem_u32(buf);
#pragma unroll 1
  for (int c = 0; c <= HELD && c - 7 < cols; c += 32) {
#pragma unroll
    for (int b = 0; b <= HELD; b += 32) {
      if (b != c) continue;
#pragma unroll
      for (int j = b > 0 ? 0 : 8; j < (b < HELD ? 40 : 8); ++j)
        asm volatile("st.shared.f32 [%0], %1;" ::"r"(at + 4 * (lane * kEpiPitch + j)), "f"(held[b - 8 + j] * scale)
                     : "memory");
    }
    __syncwarp();
    if (rows == 32) {
      if (add) write_block<true, true>(at, out, start, ld, c, cols, rows, lane);
      else write_block<false, true>(at, out, start, ld, c, cols, rows, lane);
    } else {
      if (add) write_block<true, false>(at, out, start, ld, c, cols, rows, lane);
      else write_block<false, false>(at, out, start, ld, c, cols, rows, lane);
    }
    __syncwarp();
  }
}

// ---- dy by loads --------------------------------------------------------------------------------------------------
// The steps of a pair, one after another over its tiles.
struct StepWalk {
  const LinArgs& a;
  int t, by, k;
  LinTile x;
  __device__ __forceinline__ StepWalk(const LinArgs& a, int pair, int pairs) : a(a), t(pair), by(pairs) {
    if (on()) x = lin_tile(a, t), k = x.from;
  }
  __device__ __forceinline__ bool on() const { return t < a.splits * a.W * a.m_tiles * a.n_tiles; }
  __device__ __forceinline__ void next() {
    if (++k < x.to) return;
    t += by;
    if (on()) x = lin_tile(a, t), k = x.from;
  }
};

// A loading warp's share of a step: its box of 64 rows, two of them a lane, of the tokens token0, token0 + 4, ...: 16 lines of
// 128 bytes in a stage.
constexpr int kLines = 16;
struct DyShare {
  int box, token0, lane;
  __device__ __forceinline__ int row(const LinTile& x, int rank) const { return x.m * 2 * kM + rank * kM + box * 64 + 2 * lane; }
  __device__ __forceinline__ uint32_t place(int line) const {
    const int token = token0 + 4 * line;
    return box * kBoxBytes + token * 128 + (((lane >> 2) ^ (token & 7)) << 4) + (lane & 3) * 4;
  }
};
__device__ __forceinline__ void store4(uint32_t at, unsigned v) {
  asm volatile("st.shared.b32 [%0], %1;" ::"r"(at), "r"(v) : "memory");
}

// bf16 rows on 4 bytes: words copied asynchronously, two steps ahead of the step that is handed on.
template <typename Wait, typename Done>
__device__ __forceinline__ void copy_words(const LinArgs& a, StepWalk walk, const DyShare& me, int rank, uint32_t stages, int stage,
                                           int S, Wait wait, Done done) {
  constexpr unsigned kAhead = 2;
  unsigned step = 0, told = 0;
  for (; walk.on(); walk.next(), ++step) {
    if (!wait(step)) break;
    const uint32_t at = stages + step % S * stage;
    const int row = me.row(walk.x, rank), live = 2 * max(0, min(2, a.rows - row)), token0 = walk.k * kK + me.token0;
    const __nv_bfloat16* const from = static_cast<const __nv_bfloat16*>(a.dy) + walk.x.w * a.dy_stride + (live ? row : 0);
#pragma unroll
    for (int i = 0; i < kLines; ++i) {
      const int token = token0 + 4 * i;  // (bytes that are not there arrive as zeros)
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(at + me.place(i)),
                   "l"(__cvta_generic_to_global(token < a.n ? from + token * a.ld : from)), "r"(token < a.n ? live : 0)
                   : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    if (step < kAhead) continue;
    asm volatile("cp.async.wait_group %0;" ::"n"(kAhead) : "memory");
    done(told++);
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  while (told < step) done(told++);
}

// Loads into registers, a step ahead: single bf16 values, or pairs of fp32 that become three terms each.
template <bool F32, bool WIDE> struct DyPair;
template <bool WIDE> struct DyPair<false, WIDE> {
  unsigned short v[2];
  __device__ __forceinline__ void load(const void* dy, long long at, int live) {
    const unsigned short* const p = static_cast<const unsigned short*>(dy) + at;
    v[0] = live > 0 ? p[0] : 0;
    v[1] = live > 1 ? p[1] : 0;
  }
  static constexpr bool special = false;
  __device__ __forceinline__ void watch(float&) const {}
  __device__ __forceinline__ void store(uint32_t at, bool) const { store4(at, v[0] | (unsigned)v[1] << 16); }
};
template <bool WIDE> struct DyPair<true, WIDE> {
  float v[2];
  __device__ __forceinline__ void load(const void* dy, long long at, int live) {
    const float* const p = static_cast<const float*>(dy) + at;
    if (WIDE && live == 2) {
      const float2 x = *reinterpret_cast<const float2*>(p);
      v[0] = x.x; v[1] = x.y;
    } else {
      v[0] = live > 0 ? p[0] : 0.f;
      v[1] = live > 1 ? p[1] : 0.f;
    }
  }
  static constexpr bool special = true;
  __device__ __forceinline__ void watch(float& most) const {
#pragma unroll
    for (int k = 0; k < 2; ++k) asm("max.NaN.f32 %0, %0, %1;" : "+f"(most) : "f"(fabsf(v[k])));
  }
  // Cut, not rounded: each term takes the next 8 bits, and the rest is exact.  An infinity or NaN (`odd`) is the first alone.
  __device__ __forceinline__ void store(uint32_t at, bool odd) const {
    unsigned w[3] = {};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      unsigned b0 = __float_as_uint(v[k]) & 0xffff0000u;
      float r = v[k] - __uint_as_float(b0);
      if (odd && !(fabsf(v[k]) < __builtin_huge_valf())) {
        r = 0.f;
        if (v[k] != v[k]) b0 = 0x7fff0000u;
      }
      const unsigned b1 = __float_as_uint(r) & 0xffff0000u;
      const unsigned b2 = __float_as_uint(r - __uint_as_float(b1));
      w[0] = k ? __byte_perm(w[0], b0, 0x7610) : b0 >> 16;
      w[1] = k ? __byte_perm(w[1], b1, 0x7610) : b1 >> 16;
      w[2] = k ? __byte_perm(w[2], b2, 0x7610) : b2 >> 16;
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) store4(at + q * kABytes, w[q]);
  }
};
template <bool F32, bool WIDE, typename Wait, typename Done>
__device__ __forceinline__ void load_pairs(const LinArgs& a, StepWalk walk, const DyShare& me, int rank, uint32_t stages, int stage,
                                           int S, Wait wait, Done done) {
  DyPair<F32, WIDE> pair[kLines];
  auto fetch = [&]() {
    const int row = me.row(walk.x, rank), live = max(0, min(2, a.rows - row)), token0 = walk.k * kK + me.token0;
    const long long at = walk.x.w * a.dy_stride + row;
#pragma unroll
    for (int i = 0; i < kLines; ++i) {
      const int token = token0 + 4 * i;
      pair[i].load(a.dy, at + token * a.ld, token < a.n ? live : 0);
    }
  };
  if (walk.on()) fetch();
  for (unsigned step = 0; walk.on(); ++step) {
    if (!wait(step)) break;
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < kLines; ++i) pair[i].watch(most);
    const bool odd = DyPair<F32, WIDE>::special && !(most < __builtin_huge_valf());
    const uint32_t at = stages + step % S * stage;
    if (__any_sync(0xffffffffu, odd)) {
#pragma unroll
      for (int i = 0; i < kLines; ++i) pair[i].store(at + me.place(i), true);
    } else {
#pragma unroll
      for (int i = 0; i < kLines; ++i) pair[i].store(at + me.place(i), false);
    }
    done(step);
    walk.next();
    if (walk.on()) fetch();
  }
}

// The blocks of a pair walk over the tiles.  In each, warps 0-7 add up and write the sums of its 128 rows, two warps (half of
// the columns each) for each quarter of them, warps 9 and 10 issue the copies of dy and of the checkpoint, and where dy cannot
// be copied eight more warps load it; the first block's warp 8 issues the products of both.  Two sums in tensor memory: one is
// read while the other grows.  All by this kernel alone, a few launches:
// 8 x 700 tokens into 33278 x 650: 287 us (843 TFLOP/s, 37 % of the memory's rate); 187 us with the
// sums left unwritten, 132 us for the same writing alone: the two meet in the L2 cache, which hands out 2.6 GB of operands
// meanwhile.  8 x 16384 tokens into 4096 x 1024: 882 us, 1246 TFLOP/s; into 2600 x 650, whose tiles are 8 % and 3 % empty and fill
// 3.6 waves of 4: 468 us, 945 TFLOP/s.  Whole calls (decoding too), a thousand behind one another at the power cap: 337-365 us
// and 557-600 us for the first and the last of these.  dy by loads, 33278 x 650: bf16 rows on 4 bytes 835-1070 us, on 2 bytes
// 1010 us, fp32 1880 us.
template <DyPath P, bool WIDE>
__global__ void __launch_bounds__(LinCfg<P>::threads, 1)
linear_grad_kernel(const LinArgs a, const __grid_constant__ CUtensorMap dy_map, const __grid_constant__ CUtensorMap x_map) {
  using Cfg = LinCfg<P>;
  constexpr int S = Cfg::stages;
  extern __shared__ char dynamic[];
  __shared__ LinShared sh;
  char* const stages = dynamic + (1024 - (smem_u32(dynamic) & 1023)) % 1024;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.x & 1, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const int tiles = a.splits * a.W * a.m_tiles * a.n_tiles, half = a.tile_n / 2;
  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(&sh.full[s], 1 + (P == DY_TMA ? 0 : 2 * kLoadWarps));
      mbar_init(&sh.empty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&sh.acc_full[s], 1);
      mbar_init(&sh.acc_empty[s], 2 * kEpiWarps);
    }
    mbar_init(&sh.drain, 1);
    fence_mbar_init();
  }
  // Tensor memory is taken when nothing ahead can still need it, and before the next kernel may start: two kernels on an SM
  // never wait for each other's.
  await_previous();
  if (warp == kMmaWarp) tmem_alloc(&sh.tmem);
  tc_before_sync();
  __syncthreads();
  cluster_sync();
  tc_after_sync();
  let_next_start();
  const uint32_t tmem = sh.tmem;

  if (warp < kEpiWarps) {
    more_registers<Cfg::epi_regs>();
    constexpr int kHeld = Cfg::n / 2;  // columns of a lane's row
    const int quarter = warp & 3, side = warp >> 2;
    float* const buf = reinterpret_cast<float*>(stages + S * Cfg::stage) + warp * 32 * kEpiPitch;
    const uint32_t held_at = tmem + side * half + ((uint32_t)(quarter * 32) << 16);
    unsigned sum = 0;
    bool ok = true;
    for (int t = pair; t < tiles && ok; t += pairs) {
      float held[kHeld];
      auto take = [&](auto add) {
        if (!(ok = lin_wait(&sh.acc_full[sum & 1], (sum >> 1) & 1, a.status))) return;
        tc_after_sync();
#pragma unroll
        for (int c = 0; c < kHeld; c += 32) {  // (the last reads up to 16 columns behind its half, which nobody writes)
          if (c < half) {
            uint32_t v[32];
            tmem_load16(held_at + (sum & 1) * Cfg::n + c, v);
            tmem_load16(held_at + (sum & 1) * Cfg::n + c + 16, v + 16);
            tmem_wait_load();
#pragma unroll
            for (int j = 0; j < 32; ++j)
              held[c + j] = decltype(add)::value ? held[c + j] + __uint_as_float(v[j]) : __uint_as_float(v[j]);
          }
        }
        tc_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive_first(&sh.acc_empty[sum & 1]);
        ++sum;
      };
      int chunks = lin_chunks<Cfg::chunk>(lin_tile(a, t));
      take(std::false_type());
      while (--chunks > 0 && ok) take(std::true_type());
      if (!ok) break;
      const LinTile x = lin_tile(a, t);
      const int row0 = x.m * 2 * kM + rank * kM + quarter * 32, n0 = x.n * a.tile_n + side * half;
      float* const out = a.out + ((long long)x.split * a.W + x.w) * a.out_stride + (long long)row0 * a.cols + n0;
      const int rows = min(32, a.rows - row0), cols = min(half, a.cols - n0);
      if (rows <= 0 || cols <= 0) continue;  // (a tile may end inside the other warp's half)
      write_rows<kHeld>(held, a.scale, a.accumulate, buf, out, a.cols, cols, rows, lane);
    }
  } else if (warp < kLoadWarp) {
    fewer_registers<Cfg::mma_regs>();
    unsigned step = 0;
    bool ok = true;
    if (warp == kMmaWarp && rank == 0) {
      unsigned sum = 0;
      const uint32_t idesc = mma_desc(a.tile_n);
      const bool issuer = elect_one();
      for (int t = pair; t < tiles && ok; t += pairs) {
        const LinTile x = lin_tile(a, t);
        const int chunks = lin_chunks<Cfg::chunk>(x);
        int begin = x.from, end = begin, chunk = 0;
        for (int k = x.from; k < x.to; ++k, ++step) {
          if (k == end) begin = k, end = x.from + (int)((long long)(x.to - x.from) * ++chunk / chunks);
          const unsigned s = step % S, acc = sum & 1;
          const bool first = k == begin, last = k + 1 == end;
          if (first && !(ok = lin_wait(&sh.acc_empty[acc], ((sum >> 1) & 1) ^ 1, a.status))) break;
          if (!(ok = lin_wait(&sh.full[s], (step / S) & 1, a.status))) break;
          tc_after_sync();
          if (issuer) {
            const uint32_t at = smem_u32(stages + s * Cfg::stage);
            const uint64_t b = operand_desc(at + Cfg::parts * kABytes);
#pragma unroll
            for (int part = 0; part < Cfg::parts; ++part) {
              const uint64_t am = operand_desc(at + part * kABytes);
#pragma unroll
              for (int j = 0; j < kK / 16; ++j)
                tc_mma(tmem + acc * Cfg::n, am + j * (2048 >> 4), b + j * (2048 >> 4), idesc, !first || part > 0 || j > 0);
            }
            tc_commit(&sh.empty[s]);
            if (last) tc_commit(&sh.acc_full[acc]);
          }
          sum += last;
        }
      }
      if (!ok && issuer) {  // no product may be under way when the blocks free their tensor memory
        tc_commit(&sh.drain);
        mbar_wait_bounded(&sh.drain, 0);
      }
    } else if ((warp == kDyWarp || warp == kXWarp) && elect_one()) {
      const int boxes = warp == kXWarp ? (half + 63) / 64 : P == DY_TMA ? kM / 64 : 0;
      const unsigned bytes = 2 * ((P == DY_TMA ? kABytes : 0) + (half + 63) / 64 * kBoxBytes);  // of a step, in both blocks
      const CUtensorMap* const map = warp == kXWarp ? &x_map : &dy_map;
      for (int t = pair; t < tiles && ok; t += pairs) {
        const LinTile x = lin_tile(a, t);
        const int at0 = warp == kXWarp ? x.n * a.tile_n + rank * half : x.m * 2 * kM + rank * kM;
        for (int k = x.from; k < x.to; ++k, ++step) {
          const unsigned s = step % S;
          if (!(ok = lin_wait(&sh.empty[s], ((step / S) & 1) ^ 1, a.status))) break;
          if (warp == kDyWarp && rank == 0) mbar_arrive_expect_tx(&sh.full[s], bytes);
          char* const to = stages + s * Cfg::stage + (warp == kXWarp ? Cfg::parts * kABytes : 0);
          for (int b = 0; b < boxes; ++b) tma_load(to + b * kBoxBytes, map, at0 + b * 64, k * kK, x.w, &sh.full[s]);
        }
      }
      if (!ok && warp == kDyWarp && rank == 0)  // both blocks' copies under way end before the blocks do
        for (unsigned j = step < S ? 0 : step - S; j < step; ++j) mbar_wait_bounded(&sh.full[j % S], (j / S) & 1);
    }
  } else {
    fewer_registers<Cfg::load_regs>();
    if constexpr (P != DY_TMA) {
      const int loader = warp - kLoadWarp;
      const DyShare me{loader & 1, loader >> 1, lane};
      const uint32_t at = smem_u32(stages);
      auto wait = [&](unsigned step) { return lin_wait(&sh.empty[step % S], ((step / S) & 1) ^ 1, a.status); };
      auto done = [&](unsigned step) {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive_first(&sh.full[step % S]);
      };
      if constexpr (P == DY_BF16 && WIDE) copy_words(a, StepWalk(a, pair, pairs), me, rank, at, Cfg::stage, S, wait, done);
      else load_pairs<P == DY_F32, WIDE>(a, StepWalk(a, pair, pairs), me, rank, at, Cfg::stage, S, wait, done);
    }
  }
  __syncwarp();
  tc_before_sync();
  __syncthreads();
  cluster_sync();  // the other block may still read this one's stages and arrive on its barriers
  tc_after_sync();
  if (warp == kMmaWarp) tmem_free(tmem);
}

// Few tokens and small layers, where starting the tensor cores is most of the time: a block of 64 rows by 64 columns in fp32,
// dy and the decoded columns in shared memory, eight rows by two columns a thread.
constexpr int kFewTokens = 64, kFewTile = 64;
template <typename T>
__global__ void __launch_bounds__(256) linear_grad_few_kernel(const LinArgs a, const uint8_t* code, const uint8_t* scales) {
  __shared__ __align__(16) float sy[kFewTokens][kFewTile];
  __shared__ __align__(16) float sx[kFewTokens][kFewTile];
  await_previous();
  let_next_start();
  const int tid = threadIdx.x, w = blockIdx.z, row0 = blockIdx.y * kFewTile, col0 = blockIdx.x * kFewTile;
  const int blocks = (a.cols + ACC_CHECKPOINT_BLOCK - 1) / ACC_CHECKPOINT_BLOCK, code_row = blocks * ACC_CHECKPOINT_BLOCK;
  // all loads of a thread go out before the first is waited for
  constexpr int kY = kFewTokens / 4, kX = kFewTokens / 16;
  T y[kY];
  unsigned x[kX], byte[kX];
  const int i = tid & 63, u = 4 * (tid & 15);
#pragma unroll
  for (int k = 0; k < kX; ++k) {
    const int t = (tid >> 4) + 16 * k, c = col0 + u;
    const bool on = t < a.n && c < code_row;
    const long long row = (long long)w * a.n + t;
    x[k] = on ? *reinterpret_cast<const unsigned*>(code + row * code_row + c) : 0u;
    byte[k] = on ? scales[row * blocks + c / ACC_CHECKPOINT_BLOCK] : 0u;
  }
  const T* const dy = static_cast<const T*>(a.dy) + w * a.dy_stride + row0 + i;
#pragma unroll
  for (int k = 0; k < kY; ++k) {
    const int t = (tid >> 6) + 4 * k;
    y[k] = t < a.n && row0 + i < a.rows ? dy[t * a.ld] : T(0.f);
  }
#pragma unroll
  for (int k = 0; k < kX; ++k) {
    const float s = __uint_as_float(byte[k] == 0 ? 0x00400000u : byte[k] == 255 ? 0x7fffffffu : byte[k] << 23);
    float v[4];
#pragma unroll
    for (int h = 0; h < 4; h += 2) {
      unsigned f;
      asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(f) : "h"((unsigned short)(x[k] >> (8 * h))));
      const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&f));
      v[h] = p.x * s;
      v[h + 1] = p.y * s;
    }
    *reinterpret_cast<float4*>(&sx[(tid >> 4) + 16 * k][u]) = make_float4(v[0], v[1], v[2], v[3]);
  }
#pragma unroll
  for (int k = 0; k < kY; ++k) {
    if constexpr (sizeof(T) == 2) sy[(tid >> 6) + 4 * k][i] = __bfloat162float(y[k]);
    else sy[(tid >> 6) + 4 * k][i] = y[k];
  }
  __syncthreads();
  const int lane = tid & 31, r = 8 * (tid >> 5);
  float sum[8][2] = {};
#pragma unroll 8
  for (int t = 0; t < a.n; ++t) {
    const float4 y0 = *reinterpret_cast<const float4*>(&sy[t][r]), y1 = *reinterpret_cast<const float4*>(&sy[t][r + 4]);
    const float yv[8] = {y0.x, y0.y, y0.z, y0.w, y1.x, y1.y, y1.z, y1.w};
    const float x0 = sx[t][lane], x1 = sx[t][lane + 32];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      sum[k][0] = fmaf(yv[k], x0, sum[k][0]);
      sum[k][1] = fmaf(yv[k], x1, sum[k][1]);
    }
  }
  float* const out = a.out + w * a.out_stride + (long long)(row0 + r) * a.cols + col0 + lane;
  float old[8][2];
  if (a.accumulate) {
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        old[k][j] = row0 + r + k < a.rows && col0 + lane + 32 * j < a.cols ? out[(long long)k * a.cols + 32 * j] : 0.f;
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float v = sum[k][j] * a.scale;
      if (row0 + r + k < a.rows && col0 + lane + 32 * j < a.cols)
        out[(long long)k * a.cols + 32 * j] = a.accumulate ? old[k][j] + v : v;
    }
  }
}

// G (+)= scale * the splits' sums, in order.
__global__ void __launch_bounds__(256) linear_join_kernel(const float* part, long long slab, int splits, int W, long long size,
                                                          float* grads, long long stride, float scale, int accumulate) {
  await_previous();
  let_next_start();
  const long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * 4;
  const int w = blockIdx.y;
  if (i >= size) return;
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s = 0; s < splits; ++s) {
    const float4 v = __ldcs(reinterpret_cast<const float4*>(part + ((long long)s * W + w) * slab + i));
    sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
  }
  float* const g = grads + w * stride + i;
  const float v[4] = {sum.x * scale, sum.y * scale, sum.z * scale, sum.w * scale};
  if (i + 4 <= size) {
    float4 o = make_float4(v[0], v[1], v[2], v[3]);
    if (accumulate) {
      const float4 old = *reinterpret_cast<const float4*>(g);
      o.x += old.x; o.y += old.y; o.z += old.z; o.w += old.w;
    }
    *reinterpret_cast<float4*>(g) = o;
  } else {
    for (int k = 0; i + k < size; ++k) g[k] = accumulate ? g[k] + v[k] : v[k];
  }
}

// ---- launches ----------------------------------------------------------------------------------------------------
struct LinPlan {
  int m_tiles, n_tiles, tile_n, steps, splits;
  long long slab;  // floats of a split's sums of one worker
  size_t x_bytes, bytes;  // of the decoded checkpoint; of it and the splits' sums
};
static LinPlan lin_plan(const acc_ctx* ctx, int layer, long long n, int most_n, int parts) {
  const DevLayer& L = ctx->plan.layers[layer];
  const int W = ctx->cfg.n_workers;
  LinPlan p{};
  p.m_tiles = (L.rows + 2 * kM - 1) / (2 * kM);
  p.steps = (int)((n + kK - 1) / kK);
  p.slab = ((long long)L.rows * L.cols + 3) / 4 * 4;
  // Few tiles leave SMs idle: then the tiles get narrower, or the tokens are cut into splits whose sums a second kernel joins.
  // Costs in products of 64 tokens by 256 columns (a quarter of a microsecond): a step of a narrow tile costs what
  // dy's copies take, that of 224 columns; a tile's start and end are 6 of its width and 2, the second launch 8 and its traffic.
  const long long pairs = ctx->sm_count / 2;
  const int least = (L.cols + most_n - 1) / most_n;
  double best = -1.0;
  // (a wide layer has tiles enough: a few counts above the least are weighed, not all)
  for (int nt = least; nt <= std::min(4 * least, least + 12) && (nt == least || L.cols / nt >= 32); ++nt) {
    const int tile_n = ((L.cols + nt - 1) / nt + 31) / 32 * 32, n_tiles = (L.cols + tile_n - 1) / tile_n;
    const long long tiles = (long long)W * p.m_tiles * n_tiles;
    const double each = tile_n / 256.0, step = std::max(each, most_n * 0.875 / 256.0);
    for (int s = 1; s <= 32 && (s == 1 || p.steps / s >= 4); ++s) {
      const double waves = (double)((tiles * s + pairs - 1) / pairs), traffic = (s + 1.0) * W * p.slab * 4.0 / 1.6e6;
      const double cost = waves * ((p.steps + s - 1) / s * step * parts + 6 * each + 2) + (s > 1 ? 8 + traffic : 0.0);
      if (best < 0 || cost < best) {
        best = cost;
        p.splits = s;
        p.tile_n = tile_n;
        p.n_tiles = n_tiles;
      }
    }
  }
  const long long row = (L.cols + ACC_CHECKPOINT_BLOCK - 1) / ACC_CHECKPOINT_BLOCK * ACC_CHECKPOINT_BLOCK;
  p.x_bytes = ((size_t)(2 * row * n * W) + 255) / 256 * 256;
  p.bytes = p.x_bytes + (p.splits > 1 ? sizeof(float) * (size_t)p.splits * W * p.slab : 0);
  if (p.bytes < 256) p.bytes = 256;
  return p;
}
// Whether the kernel for few tokens takes the call: its sums cost 2 W n rows cols operations at the fp32 units' rate, the tensor
// cores' way two launches and their start (columns: 650).  On the GPU, 35 tokens into 2600 rows: 7.9 us against 13.0; 64 tokens
// into 1200: 6.6 and 9.4; into 2400: 9.2 and 8.0; 2 tokens into 33278: 34 and 37.
static bool few_way(const acc_ctx* ctx, int layer, long long n) {
  const DevLayer& L = ctx->plan.layers[layer];
  return n <= kFewTokens && (double)ctx->cfg.n_workers * n * L.rows * L.cols <= 7e7 && L.rows <= 65535 * kFewTile;
}
template <DyPath P> static LinPlan lin_plan(const acc_ctx* ctx, int layer, long long n) {
  return lin_plan(ctx, layer, n, LinCfg<P>::n, LinCfg<P>::parts);
}
size_t linear_grad_workspace(const acc_ctx* ctx, int layer, long long n) {
  LinWorkspace& last = ctx->linear_workspace;  // (the same question from call to call: 400 plans to weigh for many tokens)
  {
    std::lock_guard<std::mutex> hold(last.lock);
    if (last.layer == layer && last.n == n) return last.bytes;
  }
  const size_t bytes = few_way(ctx, layer, n) ? 256 :
      std::max(lin_plan<DY_TMA>(ctx, layer, n).bytes,
               std::max(lin_plan<DY_BF16>(ctx, layer, n).bytes, lin_plan<DY_F32>(ctx, layer, n).bytes));
  std::lock_guard<std::mutex> hold(last.lock);
  last.layer = layer;
  last.n = n;
  last.bytes = bytes;
  return bytes;
}

template <DyPath P, bool WIDE> static cudaError_t lin_prepare() {
  // (a block launched with fewer registers than it deals out would wait for them for good)
  cudaFuncAttributes f;
  cudaError_t e = cudaFuncGetAttributes(&f, linear_grad_kernel<P, WIDE>);
  if (e == cudaSuccess && f.numRegs < LinCfg<P>::launch_regs) e = cudaErrorInvalidConfiguration;
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(linear_grad_kernel<P, WIDE>, cudaFuncAttributeMaxDynamicSharedMemorySize, LinCfg<P>::smem);
}
cudaError_t prepare_linear() {
  cudaError_t e = lin_prepare<DY_TMA, true>();
  if (e == cudaSuccess) e = lin_prepare<DY_BF16, true>();
  if (e == cudaSuccess) e = lin_prepare<DY_BF16, false>();
  if (e == cudaSuccess) e = lin_prepare<DY_F32, true>();
  if (e == cudaSuccess) e = lin_prepare<DY_F32, false>();
  return e;
}

// The driver's tensor-map encoder, through the runtime (the library is not linked against the driver's).
using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeTiled encode_tiled() {
  static const EncodeTiled f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      p = nullptr;
    }
    return reinterpret_cast<EncodeTiled>(p);
  }();
  return f;
}

// Map of [W][n] rows of `width` bf16 values, ld apart, workers `stride` apart (each a multiple of 8 where there are several;
// a dimension of one has no stride of its own, and any that spans it does); false for strides beyond a map's range.
static bool bf16_map(CUtensorMap* map, const void* p, long long width, long long n, long long W, long long ld, long long stride) {
  const long long row = n == 1 ? (width + 7) / 8 * 8 : ld, worker = W == 1 ? row * n : stride;
  const cuuint64_t dims[3] = {(cuuint64_t)width, (cuuint64_t)n, (cuuint64_t)W};
  const cuuint64_t strides[2] = {(cuuint64_t)row * 2, (cuuint64_t)worker * 2};
  const cuuint32_t box[3] = {64, kK, 1}, one[3] = {1, 1, 1};
  return encode_tiled()(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(p), dims, strides, box, one,
                        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t launch_linear_grad(acc_ctx* ctx, int layer, const void* dy, bool bf16, long long n, long long ld,
                               long long dy_stride, float scale, const uint8_t* code, const uint8_t* scales, float* grads,
                               int accumulate, void* workspace, cudaStream_t s) {
  const DevLayer& L = ctx->plan.layers[layer];
  const int W = ctx->cfg.n_workers;
  float* const layer0 = grads + L.offset;
  const long long stride = ctx->cfg.worker_stride, size = (long long)L.rows * L.cols;
  if (n == 0) {
    if (accumulate) return cudaSuccess;
    cudaError_t e = cudaSuccess;
    for (int w = 0; w < W && e == cudaSuccess; ++w) e = cudaMemsetAsync(layer0 + w * stride, 0, sizeof(float) * size, s);
    return e;
  }
  if (few_way(ctx, layer, n)) {
    LinArgs a{};
    a.dy = dy; a.ld = ld; a.dy_stride = dy_stride;
    a.n = (int)n; a.rows = L.rows; a.cols = L.cols;
    a.out = layer0; a.out_stride = stride; a.scale = scale; a.accumulate = accumulate;
    PhaseTimer pt(ctx, PH_LINEAR_FEW, s);
    return launch_early(bf16 ? linear_grad_few_kernel<__nv_bfloat16> : linear_grad_few_kernel<float>,
                        dim3((L.cols + kFewTile - 1) / kFewTile, (L.rows + kFewTile - 1) / kFewTile, W), 256, s, a, code, scales);
  }
  if (ctx->linear_ready != cudaSuccess) return ctx->linear_ready;
  if (encode_tiled() == nullptr) return cudaErrorNotSupported;
  // The checkpoint as bf16, exactly, once for all tiles: a tile's own decoding costs the SM more than its products do (64 tokens
  // x 224 columns: 2400 warp instructions for 448 cycles of the tensor core).
  const int row = (L.cols + ACC_CHECKPOINT_BLOCK - 1) / ACC_CHECKPOINT_BLOCK * ACC_CHECKPOINT_BLOCK;
  const uintptr_t address = reinterpret_cast<uintptr_t>(dy);
  CUtensorMap x_map{}, dy_map{};
  if (!bf16_map(&x_map, workspace, row, n, W, row, row * n)) return cudaErrorInvalidValue;
  const bool tma = bf16 && address % 16 == 0 && (n == 1 || ld % 8 == 0) && (W == 1 || dy_stride % 8 == 0) &&
                   bf16_map(&dy_map, dy, L.rows, n, W, ld, dy_stride);
  cudaError_t e = launch_checkpoint(ctx, false, workspace, true, n * W, row, row, nullptr, false, const_cast<uint8_t*>(code),
                                    const_cast<uint8_t*>(scales), s);
  if (e != cudaSuccess) return e;
  const LinPlan p = tma    ? lin_plan<DY_TMA>(ctx, layer, n)
                    : bf16 ? lin_plan<DY_BF16>(ctx, layer, n)
                           : lin_plan<DY_F32>(ctx, layer, n);
  const bool split = p.splits > 1;
  float* const sums = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.x_bytes);
  LinArgs a{};
  a.dy = dy; a.ld = ld; a.dy_stride = dy_stride;
  a.n = (int)n; a.rows = L.rows; a.cols = L.cols;
  a.out = split ? sums : layer0;
  a.out_stride = split ? p.slab : stride;
  a.scale = split ? 1.f : scale;
  a.accumulate = split ? 0 : accumulate;
  a.W = W; a.m_tiles = p.m_tiles; a.n_tiles = p.n_tiles; a.splits = p.splits; a.steps = p.steps; a.tile_n = p.tile_n;
  a.status = ctx->d_status;
  const long long tiles = (long long)p.splits * W * p.m_tiles * p.n_tiles;
  const unsigned grid = 2 * (unsigned)std::min<long long>(tiles, ctx->sm_count / 2);
  {
    PhaseTimer pt(ctx, PH_LINEAR_GRAD, s);
    auto go = [&](auto path, auto wide) {
      constexpr DyPath P = decltype(path)::value;
      return launch_early_as(linear_grad_kernel<P, decltype(wide)::value>, grid, LinCfg<P>::threads, LinCfg<P>::smem, 2, s, a,
                             dy_map, x_map);
    };
    using Tma = std::integral_constant<DyPath, DY_TMA>;
    using Bf16 = std::integral_constant<DyPath, DY_BF16>;
    using F32 = std::integral_constant<DyPath, DY_F32>;
    // pairs of values, where every row starts on one
    const int size = bf16 ? 2 : 4;
    const uintptr_t each = address | (uintptr_t)(n > 1 ? ld : 0) * size | (uintptr_t)(W > 1 ? dy_stride : 0) * size;
    const bool wide = each % (2 * size) == 0;
    if (tma) e = go(Tma(), std::true_type());
    else if (bf16) e = wide ? go(Bf16(), std::true_type()) : go(Bf16(), std::false_type());
    else e = wide ? go(F32(), std::true_type()) : go(F32(), std::false_type());
  }
  if (e != cudaSuccess || !split) return e;
  PhaseTimer pt(ctx, PH_LINEAR_JOIN, s);
  return launch_early(linear_join_kernel, dim3((unsigned)((size + 1023) / 1024), (unsigned)W), 256, s,
                      static_cast<const float*>(sums), p.slab, p.splits, W, size, layer0, stride, scale, accumulate);
}

}  // namespace acc
