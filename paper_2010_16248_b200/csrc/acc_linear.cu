// Weight gradient of a linear layer from a checkpoint of its input: G_w (+)= scale * sum over the tokens t of dy_wt x_wt^T, a
// matrix product on the tensor cores that reads the 8-bit codes and writes the workers' fp32 gradients.
#include <cuda.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <type_traits>

#include "acc_async.cuh"
#include "acc_internal.cuh"

namespace acc {

// A tile is 128 rows of the layer (the product's M) by up to 256 columns (N); a step is 64 tokens (K).  Both operands lie in
// memory with the tokens outermost, so a stage holds them with M (N) contiguous: boxes of 64 elements (128 bytes) x 64 tokens
// in the 128-byte swizzle, 16-byte chunk c of token k at chunk c ^ (k & 7).
constexpr int kM = 128, kN = 256, kK = 64;
constexpr int kBoxBytes = 64 * 128;
constexpr int kABytes = kM / 64 * kBoxBytes, kBBytes = kN / 64 * kBoxBytes;
constexpr int kEpiPitch = 33;

enum { kEpiWarps = 4, kMmaWarp = 4, kTmaWarp = 5, kDecodeWarp = 6, kDecodeGroups = 2, kGroupWarps = 4, kLoadWarp = 14, kLoadWarps = 4 };

// How dy reaches shared memory: bf16 by tensor copies, or (rows that do not start on 16 bytes; fp32) by loads.
enum DyPath { DY_TMA, DY_BF16, DY_F32 };
template <DyPath P> struct LinCfg {
  // fp32 values are three bf16 terms each (8 bits of the 24 apiece), so that the products stay those of fp32
  static constexpr int parts = P == DY_F32 ? 3 : 1;
  static constexpr int stage = kABytes * parts + kBBytes;
  static constexpr int stages = P == DY_F32 ? 2 : 4;
  static constexpr int threads = 32 * (P == DY_TMA ? kLoadWarp : kLoadWarp + kLoadWarps);
  static constexpr int smem = stages * stage + kEpiWarps * 32 * kEpiPitch * 4 + 1024;
};

struct LinArgs {
  const void* dy;
  long long ld, dy_stride;      // elements between tokens, between workers
  int n, rows, cols;
  const uint4* code;            // [W][n] rows of code_row pieces of 16 codes
  const uint8_t* scales;        // [W][n][blocks]
  int code_row, blocks;
  float* out;                   // worker w's (split s's) layer at out + (s * W + w) * out_stride
  long long out_stride;
  float scale;
  int accumulate;
  int W, m_tiles, n_tiles, splits, steps, tile_n;  // tile_n: columns of a tile, a multiple of 16
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

// ---- tensor core, tensor memory ----------------------------------------------------------------------------------
__device__ __forceinline__ void tmem_alloc(uint32_t* where) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(where)) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t at) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(at));
}
__device__ __forceinline__ void tc_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile(
      "{\n"
      "  .reg .pred p;\n"
      "  setp.ne.u32 p, %4, 0;\n"
      "  tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n"
      "}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((unsigned)add)
      : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t at, uint32_t* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, "
      "%18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]),
        "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]),
        "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(at));
}
__device__ __forceinline__ void tmem_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Shared-memory descriptor of an operand whose M (N) is contiguous: 128-byte swizzle, 64 elements of M a box, boxes kBoxBytes
// apart, groups of 8 tokens 1024 bytes apart inside a box.
__device__ __forceinline__ uint64_t operand_desc(uint32_t smem) {
  return (uint64_t)((smem & 0x3ffff) >> 4) | (uint64_t)(kBoxBytes >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 |
         (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// fp32 sums of bf16 products, both operands with M (N) contiguous.
__device__ __forceinline__ uint32_t mma_desc(int n) {
  return 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | 1u << 16 | (uint32_t)(n >> 3) << 17 | (uint32_t)(kM >> 4) << 24;
}
__device__ __forceinline__ void tma_load(void* dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::
                   "r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
               : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void store16(char* p, const uint4& v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(smem_u32(p)), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// ---- codes -> bf16 -----------------------------------------------------------------------------------------------
__device__ __forceinline__ unsigned mul_bf16x2(unsigned a, unsigned b) {
  unsigned r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// Sixteen codes times their scale, exactly: a code's exponent and mantissa, moved to where bf16 has them, stand for the value
// times 2^-120 (subnormal codes become subnormal there), and the two factors are powers of two.
__device__ __forceinline__ void decode16(const uint4& c, unsigned byte, uint4& lo, uint4& hi) {
  const unsigned s = byte == 0 ? 0x0040u : byte == 255 ? 0x7fffu : byte << 7, s2 = s | s << 16;
  const unsigned w[4] = {c.x, c.y, c.z, c.w};
  unsigned o[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const unsigned x = __byte_perm(w[k >> 1], 0, k & 1 ? 0x3424 : 0x1404);
    o[k] = mul_bf16x2(mul_bf16x2((x & 0x80008000u) | ((x >> 4) & 0x07f007f0u), 0x7b807b80u), s2);
  }
  lo = make_uint4(o[0], o[1], o[2], o[3]);
  hi = make_uint4(o[4], o[5], o[6], o[7]);
}

struct LinShared {
  uint64_t full[4], empty[4], acc_full[2], acc_empty[2], drain;
  uint32_t tmem;
};

// A wait of a role; when it gives up, the call's status says so and the role ends, and with it, by their own limits, the others.
__device__ __forceinline__ bool lin_wait(uint64_t* bar, unsigned parity, int* status) {
  if (mbar_wait_bounded(bar, parity)) return true;
  atomicCAS(status, 0, ACC_ETIMEOUT);
  return false;
}

// dy's values of one token and 8 rows as bf16 terms.
template <DyPath P, bool WIDE>
__device__ __forceinline__ void load_dy8(const LinArgs& a, long long at, int left, uint4* part) {
  if constexpr (P == DY_BF16) {
    const unsigned short* p = static_cast<const unsigned short*>(a.dy) + at;
    unsigned w[4] = {};
    if (left >= 8) {
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = WIDE ? reinterpret_cast<const unsigned*>(p)[k] : p[2 * k] | (unsigned)p[2 * k + 1] << 16;
    } else {
      for (int k = 0; k < left; ++k) w[k >> 1] |= (unsigned)p[k] << (16 * (k & 1));
    }
    part[0] = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
    const float* p = static_cast<const float*>(a.dy) + at;
    float v[8] = {};
    if (left >= 8) {
      if (WIDE) {
        const float4 x = reinterpret_cast<const float4*>(p)[0], y = reinterpret_cast<const float4*>(p)[1];
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = p[k];
      }
    } else {
      for (int k = 0; k < left; ++k) v[k] = p[k];
    }
    unsigned w[3][4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma unroll
      for (int j = 0; j < 3; ++j) w[j][k] = 0;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        // cut, not rounded: each term takes the next 8 bits, and the rest is exact; an infinity or NaN is the first term alone
        const float x = v[2 * k + h];
        const unsigned b0 = __float_as_uint(x) & 0xffff0000u;
        const bool fine = (b0 & 0x7f800000u) != 0x7f800000u;
        const float r0 = fine ? x - __uint_as_float(b0) : 0.f;
        const unsigned b1 = __float_as_uint(r0) & 0xffff0000u;
        const unsigned b2 = __float_as_uint(r0 - __uint_as_float(b1)) & 0xffff0000u;
        const unsigned first = fine ? b0 : (__float_as_uint(x) & 0x7fffffffu) > 0x7f800000u ? 0x7fff0000u : b0;
        w[0][k] |= h ? first : first >> 16;
        w[1][k] |= h ? b1 : b1 >> 16;
        w[2][k] |= h ? b2 : b2 >> 16;
      }
    }
#pragma unroll
    for (int j = 0; j < 3; ++j) part[j] = make_uint4(w[j][0], w[j][1], w[j][2], w[j][3]);
  }
}

// One block per SM walks over the tiles.  Warps 0-3 write finished tiles, warp 4 issues the products, warp 5 the copies of
// dy, two groups of four warps decode the checkpoint's codes for alternate steps (a group's loads of its next step are under
// way while the other decodes), and where dy cannot be copied four more warps load it.  Two accumulators in tensor memory: a
// tile is written while the next is summed.
template <DyPath P, bool WIDE>
__global__ void __launch_bounds__(LinCfg<P>::threads, 1) linear_grad_kernel(const LinArgs a, const __grid_constant__ CUtensorMap map) {
  using Cfg = LinCfg<P>;
  constexpr int S = Cfg::stages;
  extern __shared__ char dynamic[];
  __shared__ LinShared sh;
  char* const stages = dynamic + (1024 - (smem_u32(dynamic) & 1023)) % 1024;
  float* const epi = reinterpret_cast<float*>(stages + S * Cfg::stage);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int tiles = a.splits * a.W * a.m_tiles * a.n_tiles;
  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(&sh.full[s], kGroupWarps + (P == DY_TMA ? 1 : kLoadWarps));
      mbar_init(&sh.empty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&sh.acc_full[s], 1);
      mbar_init(&sh.acc_empty[s], kEpiWarps);
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
  tc_after_sync();
  let_next_start();
  const uint32_t tmem = sh.tmem;

  if (warp < kEpiWarps) {
    float* const buf = epi + warp * 32 * kEpiPitch;
    unsigned i = 0;
    for (int t = blockIdx.x; t < tiles; t += gridDim.x, ++i) {
      const LinTile x = lin_tile(a, t);
      const unsigned acc = i & 1;
      if (!lin_wait(&sh.acc_full[acc], (i >> 1) & 1, a.status)) break;
      tc_after_sync();
      const int row0 = x.m * kM + warp * 32, n0 = x.n * a.tile_n;
      float* const out = a.out + ((long long)x.split * a.W + x.w) * a.out_stride + (long long)row0 * a.cols + n0;
      const int rows = min(32, a.rows - row0), cols = min(a.tile_n, a.cols - n0);
      for (int c = 0; c < cols; c += 32) {
        uint32_t v[32];
        tmem_load32(tmem + acc * kN + c + ((uint32_t)(warp * 32) << 16), v);
        tmem_wait_load();
#pragma unroll
        for (int k = 0; k < 32; ++k) buf[lane * kEpiPitch + k] = __uint_as_float(v[k]) * a.scale;
        __syncwarp();
        if (c + lane < cols) {
          float* const p = out + c + lane;
          if (a.accumulate) {
            for (int r = 0; r < rows; r += 8) {  // loads of a batch first
              float old[8];
#pragma unroll
              for (int k = 0; k < 8; ++k)
                if (r + k < rows) old[k] = p[(long long)(r + k) * a.cols];
#pragma unroll
              for (int k = 0; k < 8; ++k)
                if (r + k < rows) p[(long long)(r + k) * a.cols] = old[k] + buf[(r + k) * kEpiPitch + lane];
            }
          } else {
#pragma unroll 8
            for (int r = 0; r < rows; ++r) p[(long long)r * a.cols] = buf[r * kEpiPitch + lane];
          }
        }
        __syncwarp();
      }
      tc_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.acc_empty[acc]);
    }
  } else if (warp == kMmaWarp) {
    if (lane == 0) {
      unsigned step = 0, i = 0;
      const uint32_t idesc = mma_desc(a.tile_n);
      bool ok = true;
      for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x, ++i) {
        const LinTile x = lin_tile(a, t);
        const unsigned acc = i & 1;
        if (!(ok = lin_wait(&sh.acc_empty[acc], ((i >> 1) & 1) ^ 1, a.status))) break;
        tc_after_sync();
        for (int k = x.from; k < x.to; ++k, ++step) {
          const unsigned s = step % S;
          if (!(ok = lin_wait(&sh.full[s], (step / S) & 1, a.status))) break;
          tc_after_sync();
          const uint32_t at = smem_u32(stages + s * Cfg::stage);
          const uint64_t b = operand_desc(at + Cfg::parts * kABytes);
#pragma unroll
          for (int part = 0; part < Cfg::parts; ++part) {
            const uint64_t am = operand_desc(at + part * kABytes);
#pragma unroll
            for (int j = 0; j < kK / 16; ++j)
              tc_mma(tmem + acc * kN, am + j * (2048 >> 4), b + j * (2048 >> 4), idesc, k > x.from || part > 0 || j > 0);
          }
          tc_commit(&sh.empty[s]);
        }
        if (ok) tc_commit(&sh.acc_full[acc]);
      }
      if (!ok) {  // nothing of this block's may be in flight when it frees its tensor memory
        tc_commit(&sh.drain);
        mbar_wait_bounded(&sh.drain, 0);
      }
    }
    __syncwarp();
  } else if (warp == kTmaWarp) {
    if (P == DY_TMA && lane == 0) {
      unsigned step = 0;
      bool ok = true;
      for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
        const LinTile x = lin_tile(a, t);
        for (int k = x.from; k < x.to; ++k, ++step) {
          const unsigned s = step % S;
          if (!(ok = lin_wait(&sh.empty[s], ((step / S) & 1) ^ 1, a.status))) break;
          char* const at = stages + s * Cfg::stage;
          mbar_arrive_expect_tx(&sh.full[s], kABytes);
          for (int b = 0; b < kM / 64; ++b) tma_load(at + b * kBoxBytes, &map, x.m * kM + b * 64, k * kK, x.w, &sh.full[s]);
        }
      }
      if (!ok)  // copies under way end before the block does
        for (unsigned j = step < S ? 0 : step - S; j < step; ++j) mbar_wait_bounded(&sh.full[j % S], (j / S) & 1);
    }
    __syncwarp();
  } else if (warp < kLoadWarp) {
    const int group = (warp - kDecodeWarp) / kGroupWarps, tid = threadIdx.x - 32 * (kDecodeWarp + group * kGroupWarps);
    const int piece = tid & 15, token0 = tid >> 4;  // 16 codes; tokens token0, token0 + 8, ... of a step
    uint4 code[8];
    unsigned byte[8];
    // this group's next step: tile, step inside it, number among all
    int t = blockIdx.x, k = 0;
    unsigned step = 0;
    LinTile x{};
    auto settle = [&]() {  // moves on to the next tile until step k lies inside one
      while (t < tiles) {
        x = lin_tile(a, t);
        if (x.from + k < x.to) return;
        k -= x.to - x.from;
        t += gridDim.x;
      }
    };
    auto fetch = [&]() {
      const int col = x.n * a.tile_n + piece * 16;  // pieces behind the tile or the row are zeros
      const bool on = piece * 16 < a.tile_n && (col >> 4) < a.code_row;
      const int token = (x.from + k) * kK + token0;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        code[u] = make_uint4(0, 0, 0, 0);
        byte[u] = 0;
        if (on && token + 8 * u < a.n) {
          const long long row = (long long)x.w * a.n + token + 8 * u;
          code[u] = a.code[row * a.code_row + (col >> 4)];
          byte[u] = a.scales[row * a.blocks + (col >> 5)];
        }
      }
    };
    k = group;
    step = group;
    settle();
    if (t < tiles) fetch();
    while (t < tiles) {
      const unsigned s = step % S;
      if (!lin_wait(&sh.empty[s], ((step / S) & 1) ^ 1, a.status)) break;
      char* const at = stages + s * Cfg::stage + Cfg::parts * kABytes + (piece >> 2) * kBoxBytes;
      if (piece * 16 < a.tile_n) {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          uint4 lo, hi;
          decode16(code[u], byte[u], lo, hi);
          const int token = token0 + 8 * u, chunk = 2 * (piece & 3);
          char* const line = at + token * 128;
          // (neighbouring boxes' lanes begin with opposite halves: their chunks lie in the same banks)
          const bool swap = piece & 4;
          store16(line + (((chunk + swap) ^ (token & 7)) << 4), swap ? hi : lo);
          store16(line + (((chunk + !swap) ^ (token & 7)) << 4), swap ? lo : hi);
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.full[s]);
      k += kDecodeGroups;
      step += kDecodeGroups;
      settle();
      if (t < tiles) fetch();
    }
  } else {
    const int tid = threadIdx.x - 32 * kLoadWarp, chunk = tid & 15, token0 = tid >> 4;
    unsigned step = 0;
    bool ok = true;
    for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
      const LinTile x = lin_tile(a, t);
      const int row = x.m * kM + chunk * 8, left = a.rows - row;
      for (int k = x.from; k < x.to; ++k, ++step) {
        const unsigned s = step % S;
        if (!(ok = lin_wait(&sh.empty[s], ((step / S) & 1) ^ 1, a.status))) break;
        char* const at = stages + s * Cfg::stage + (chunk >> 3) * kBoxBytes;
#pragma unroll 1
        for (int u = 0; u < 8; u += 4) {
          uint4 part[4][Cfg::parts];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int token = k * kK + token0 + 8 * (u + j);
            if (token < a.n && left > 0) {
              load_dy8<P, WIDE>(a, x.w * a.dy_stride + token * a.ld + row, left, part[j]);
            } else {
              for (int q = 0; q < Cfg::parts; ++q) part[j][q] = make_uint4(0, 0, 0, 0);
            }
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int token = token0 + 8 * (u + j);
#pragma unroll
            for (int q = 0; q < Cfg::parts; ++q)
              store16(at + q * kABytes + token * 128 + (((chunk & 7) ^ (token & 7)) << 4), part[j][q]);
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.full[s]);
      }
    }
  }
  __syncwarp();
  tc_before_sync();
  __syncthreads();
  tc_after_sync();
  if (warp == kMmaWarp) tmem_free(tmem);
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
  size_t bytes;
};
static LinPlan lin_plan(const acc_ctx* ctx, int layer, long long n) {
  const DevLayer& L = ctx->plan.layers[layer];
  const int W = ctx->cfg.n_workers;
  LinPlan p{};
  p.m_tiles = (L.rows + kM - 1) / kM;
  p.n_tiles = (L.cols + kN - 1) / kN;
  p.tile_n = ((L.cols + p.n_tiles - 1) / p.n_tiles + 15) / 16 * 16;
  p.steps = (int)((n + kK - 1) / kK);
  p.slab = ((long long)L.rows * L.cols + 3) / 4 * 4;
  // Few tiles leave SMs idle: the tokens are then cut into splits, whose sums a second kernel joins.  Costs in steps of 64
  // tokens (a quarter of a microsecond): a tile's start and end 6, the second launch 8, its traffic at the memory's rate.
  const long long tiles = (long long)W * p.m_tiles * p.n_tiles, sms = ctx->sm_count;
  double best = 0;
  for (int s = 1; s <= 32 && (s == 1 || p.steps / s >= 4); ++s) {
    const double waves = (double)((tiles * s + sms - 1) / sms), traffic = (s + 1.0) * W * p.slab * 4.0 / 1.6e6;
    const double cost = waves * ((p.steps + s - 1) / s + 6) + (s > 1 ? 8 + traffic : 0.0);
    if (s == 1 || cost < best) { best = cost; p.splits = s; }
  }
  p.bytes = p.splits > 1 ? sizeof(float) * (size_t)p.splits * W * p.slab : 0;
  if (p.bytes < 256) p.bytes = 256;
  return p;
}
size_t linear_grad_workspace(const acc_ctx* ctx, int layer, long long n) { return lin_plan(ctx, layer, n).bytes; }

template <DyPath P, bool WIDE> static cudaError_t lin_prepare() {
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
  const LinPlan p = lin_plan(ctx, layer, n);
  const bool split = p.splits > 1;
  const int blocks = (L.cols + ACC_CHECKPOINT_BLOCK - 1) / ACC_CHECKPOINT_BLOCK;
  LinArgs a{};
  a.dy = dy; a.ld = ld; a.dy_stride = dy_stride;
  a.n = (int)n; a.rows = L.rows; a.cols = L.cols;
  a.code = reinterpret_cast<const uint4*>(code); a.scales = scales;
  a.code_row = blocks * 2; a.blocks = blocks;
  a.out = split ? static_cast<float*>(workspace) : layer0;
  a.out_stride = split ? p.slab : stride;
  a.scale = split ? 1.f : scale;
  a.accumulate = split ? 0 : accumulate;
  a.W = W; a.m_tiles = p.m_tiles; a.n_tiles = p.n_tiles; a.splits = p.splits; a.steps = p.steps; a.tile_n = p.tile_n;
  a.status = ctx->d_status;
  const uintptr_t address = reinterpret_cast<uintptr_t>(dy);
  CUtensorMap map{};
  bool tma = bf16 && address % 16 == 0 && (n == 1 || ld % 8 == 0) && (W == 1 || dy_stride % 8 == 0);
  if (tma) {
    // (a dimension of one has no stride of its own: any multiple of 16 bytes that spans it)
    const long long row = n == 1 ? (L.rows + 7) / 8 * 8 : ld, worker = W == 1 ? row * n : dy_stride;
    const cuuint64_t dims[3] = {(cuuint64_t)L.rows, (cuuint64_t)n, (cuuint64_t)W};
    const cuuint64_t strides[2] = {(cuuint64_t)row * 2, (cuuint64_t)worker * 2};
    const cuuint32_t box[3] = {64, kK, 1}, one[3] = {1, 1, 1};
    const EncodeTiled encode = encode_tiled();
    if (encode == nullptr) return cudaErrorNotSupported;
    if (encode(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(dy), dims, strides, box, one,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      tma = false;  // strides beyond a map's range take the other way
  }
  const long long tiles = (long long)p.splits * W * p.m_tiles * p.n_tiles;
  const unsigned grid = (unsigned)std::min<long long>(tiles, ctx->sm_count);
  cudaError_t e;
  {
    PhaseTimer pt(ctx, PH_LINEAR_GRAD, s);
    auto go = [&](auto path, auto wide) {
      constexpr DyPath P = decltype(path)::value;
      return launch_early_as(linear_grad_kernel<P, decltype(wide)::value>, grid, LinCfg<P>::threads, LinCfg<P>::smem, 1, s, a, map);
    };
    using Tma = std::integral_constant<DyPath, DY_TMA>;
    using Bf16 = std::integral_constant<DyPath, DY_BF16>;
    using F32 = std::integral_constant<DyPath, DY_F32>;
    // words of two bf16, vectors of four floats, where every row starts on one
    const uintptr_t each = address | (uintptr_t)(n > 1 ? ld : 0) * (bf16 ? 2 : 4) | (uintptr_t)(W > 1 ? dy_stride : 0) * (bf16 ? 2 : 4);
    const bool wide = each % (bf16 ? 4 : 16) == 0;
    if (tma) e = go(Tma(), std::true_type());
    else if (bf16) e = wide ? go(Bf16(), std::true_type()) : go(Bf16(), std::false_type());
    else e = wide ? go(F32(), std::true_type()) : go(F32(), std::false_type());
  }
  if (e != cudaSuccess || !split) return e;
  PhaseTimer pt(ctx, PH_LINEAR_JOIN, s);
  return launch_early(linear_join_kernel, dim3((unsigned)((size + 1023) / 1024), (unsigned)W), 256, s,
                      static_cast<const float*>(workspace), p.slab, p.splits, W, size, layer0, stride, scale, accumulate);
}

}  // namespace acc
