// Tensor-core products of 8-bit operands with a power-of-two scale for each 128 values along the contraction:
// out[i, j] = sum_k A(i, k) B(j, k), float32 accumulation, bf16 out.  Three forms:
//   linear   Y = act(X W^T + b): both operands with the contraction in their rows (K-major);
//   input    dX = dY W: the weight's rows are the contraction (MN-major B), so the forward's 8-bit values and scales serve here
//            too and no transposed copy is kept;
//   weight   dW = (dY^T X) * Mask: both operands MN-major, contraction over the tokens.
// The scales go into the tensor core (tcgen05.mma kind::mxf8f6f4.block_scale): it multiplies every product of a row by the
// row's scale, so nothing has to leave tensor memory between the blocks of 128.  The instruction wants a scale for each 32 values; the
// four instructions of a 128-deep stage are given the same one.  Scales of four stages make the four bytes of a 32-bit column
// of tensor memory: a warp collects them from the caller's arrays (any row and block stride, see Operand), 16 bytes per lane,
// and one tcgen05.cp per 128 rows brings them over, in the order of the instructions that read them.
//
// Roles: warps 0 and 10 TMA producers of A and B, warp 11 the scales, warp 1 issues, warps 2..9 epilogue, as in
// bsp_linear_tc.cu.  All waits are bounded.
#include "bsp_fp8.cuh"
#include "bsp_fp8_gemm.cuh"
#include "bsp_tc.cuh"

namespace bsp {
using namespace tc;
using namespace fp8;

namespace {

constexpr int kFp8Threads = 384;
constexpr int kScaleStages = 3;                    // groups of four stages whose scales are on their way
constexpr int kScaleTile = 512;                    // bytes: 128 rows x 4 blocks

template <int BN>
struct Fp8Cfg {
  static constexpr int kStageA = kBlockM * kBlock;
  static constexpr int kStageB = BN * kBlock;
  static constexpr int kStage = kStageA + kStageB;
  static constexpr int kTilesB = (BN + 127) / 128;
  static constexpr int kScaleGroup = (1 + kTilesB) * kScaleTile;
  static constexpr int kFixed = 1024 + kEpiBytes + kScaleStages * kScaleGroup + 2 * BN * 2 + 256;
  static constexpr int kStages = (kSmemLimit - kFixed) / kStage > 8 ? 8 : (kSmemLimit - kFixed) / kStage;
  static constexpr int kSmemBytes = kStages * kStage + kFixed;
  static constexpr int kScaleCols = 4 + 4 * kTilesB;                   // tensor memory columns of one group's scales
  static constexpr int kTmemCols = 2 * BN + 2 * kScaleCols <= 256 ? 256 : 512;
};

// A load without a branch around it, zero where it does not take place: the loads of a group of scales have to be in flight together
// (one after the other, 0.4 us each, they had bound the whole kernel: 8192 x 4096 x 4096 130 us, and its weight gradient 241).
__device__ __forceinline__ uint32_t load_word_if(const void* p, bool there) {
  uint32_t v;
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %2, 0;\n\tmov.b32 %0, 0;\n\t@p ld.global.b32 %0, [%1];\n\t}" : "=r"(v) : "l"(p), "r"(there ? 1u : 0u));
  return v;
}
// Scales of a group of four blocks (from `block0` on) of 128 rows (from `row0` on): load() asks for them, word by word, finish()
// makes of them the four blocks of a row as a word.  Arrays begin anywhere: four bytes at an address that is no multiple of four
// come from two words (aligned words that hold a byte of the array are read whole).
// What a lane gets: the rows l, l + 32, l + 64, l + 96; of an operand whose scales lie along its rows (MN-major) the rows 4 l to 4 l + 3.
// Scales that do not exist may be anything: no instruction, or no output that exists, uses them.
struct Scales {
  uint32_t lo[4], hi[4];

  __device__ __forceinline__ void load_bytes(int i, const uint8_t* p, int exist) {
    const uint32_t off = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p) & 3u);
    lo[i] = load_word_if(p - off, exist > 0);
    hi[i] = load_word_if(p - off + 4, off != 0u && exist > 4 - static_cast<int>(off));
  }
  __device__ __forceinline__ uint32_t bytes(int i, const uint8_t* p) const {
    return __funnelshift_r(lo[i], hi[i], 8u * static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p) & 3u));
  }
  __device__ __forceinline__ void load(const Operand& O, int row0, int block0, int blocks, int lane) {
    if (O.s_shift != 0) {
      // one scale for 128 rows: at most two different ones per block, eight bytes that as many lanes fetch
      const int first = row0 >> O.s_shift, last = (O.rows - 1) >> O.s_shift;
      const int r = min(first + ((lane >> 2) & 1), last), b = min(block0 + (lane & 3), blocks - 1);
      lo[0] = ld_global(O.s + r * O.s_row + b * O.s_k);
    } else if (O.mn) {
      const int r = row0 + 4 * lane;
#pragma unroll
      for (int b = 0; b < 4; ++b) load_bytes(b, O.s + (block0 + b) * O.s_k + r, block0 + b < blocks ? O.rows - r : 0);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int r = row0 + lane + 32 * q;
        load_bytes(q, O.s + r * O.s_row + block0, r < O.rows ? blocks - block0 : 0);
      }
    }
  }
  __device__ __forceinline__ uint4 finish(const Operand& O, int row0, int block0, int lane) const {
    if (O.s_shift != 0) {
      uint32_t w[2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
        w[i] = __shfl_sync(0xffffffffu, lo[0], 4 * i) | (__shfl_sync(0xffffffffu, lo[0], 4 * i + 1) << 8) |
               (__shfl_sync(0xffffffffu, lo[0], 4 * i + 2) << 16) | (__shfl_sync(0xffffffffu, lo[0], 4 * i + 3) << 24);
      auto word = [&](int q) { return (row0 + lane + 32 * q) >> O.s_shift == row0 >> O.s_shift ? w[0] : w[1]; };
      return make_uint4(word(0), word(1), word(2), word(3));
    }
    uint32_t x[4];
    if (O.mn) {
#pragma unroll
      for (int b = 0; b < 4; ++b) x[b] = bytes(b, O.s + (block0 + b) * O.s_k + row0 + 4 * lane);
      const uint32_t t0 = __byte_perm(x[0], x[1], 0x5140), t1 = __byte_perm(x[2], x[3], 0x5140);
      const uint32_t t2 = __byte_perm(x[0], x[1], 0x7362), t3 = __byte_perm(x[2], x[3], 0x7362);
      return make_uint4(__byte_perm(t0, t1, 0x5410), __byte_perm(t0, t1, 0x7632), __byte_perm(t2, t3, 0x5410), __byte_perm(t2, t3, 0x7632));
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) x[q] = bytes(q, O.s + (row0 + lane + 32 * q) * O.s_row + block0);
    return make_uint4(x[0], x[1], x[2], x[3]);
  }
};
// To the tile of 512 bytes that the tensor core reads: row r at 16 (r % 32) + 4 (r / 32).
__device__ __forceinline__ void store_scales(const Operand& O, uint32_t dst, uint4 w, int lane) {
  if (O.mn && O.s_shift == 0) {
    const uint32_t at = dst + 16u * ((4 * lane) & 31) + 4u * (lane >> 3);
    asm volatile("st.shared.b32 [%0], %1;" ::"r"(at), "r"(w.x));
    asm volatile("st.shared.b32 [%0], %1;" ::"r"(at + 16u), "r"(w.y));
    asm volatile("st.shared.b32 [%0], %1;" ::"r"(at + 32u), "r"(w.z));
    asm volatile("st.shared.b32 [%0], %1;" ::"r"(at + 48u), "r"(w.w));
  } else {
    st_shared_v4(dst + 16u * lane, w.x, w.y, w.z, w.w);
  }
}

// 512 bytes of scales (32 rows of 16 bytes: no swizzle, groups of eight rows 128 bytes apart) to four columns of tensor memory,
// for all four quarters of its lanes.
__device__ __forceinline__ uint64_t scale_desc(uint32_t smem_addr) {
  return static_cast<uint64_t>((smem_addr & 0x3ffff) >> 4) | (static_cast<uint64_t>(1) << 16) | (static_cast<uint64_t>(128 >> 4) << 32) |
         (static_cast<uint64_t>(1) << 46);
}
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint32_t smem_addr) {
  asm volatile(
      "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t}" ::"r"(taddr), "l"(scale_desc(smem_addr))
      : "memory");
}
// One pipeline stage: four K = 32 steps under the same scales, then the commit that frees the stage.
template <int STEP_A, int STEP_B>
__device__ __forceinline__ void mma_stage_scaled(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate,
                                                 uint32_t free_bar, uint32_t sfa, uint32_t sfb) {
  asm volatile(
      "{\n\t.reg .pred p, t, e;\n\t.reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.eq.b32 t, 0, 0;\n\t"
      "add.s64 a1, %1, %8;\n\tadd.s64 a2, a1, %8;\n\tadd.s64 a3, a2, %8;\n\t"
      "add.s64 b1, %2, %9;\n\tadd.s64 b2, b1, %9;\n\tadd.s64 b3, b2, %9;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%6], [%7], p;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a1, b1, %3, [%6], [%7], t;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a2, b2, %3, [%6], [%7], t;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a3, b3, %3, [%6], [%7], t;\n\t"
      "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%5];\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(free_bar), "r"(sfa), "r"(sfb), "n"(STEP_A), "n"(STEP_B)
      : "memory");
}
// MN-major tile of 8-bit values: atoms of 8 contraction rows x 128 bytes, 1024 bytes apart along the contraction; 16 KB (128
// contraction rows) from one group of 128 values along M / N to the next.
constexpr int kGroupMn = 128 * kBlock;
__device__ __forceinline__ uint64_t smem_desc_mn8(uint32_t smem_addr) {
  return static_cast<uint64_t>((smem_addr & 0x3ffff) >> 4) | (static_cast<uint64_t>(kGroupMn >> 4) << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) |
         (static_cast<uint64_t>(1) << 46) | (static_cast<uint64_t>(2) << 61);
}
// Instruction descriptor: formats of A and B (bits 7 and 10), MN-major A and B (15, 16), N (17), power-of-two scales (23), M (27);
// the bytes of the scales' columns that a stage reads go to bits 29 (A) and 4 (B).
__host__ __device__ constexpr uint32_t idesc_scaled(int a_fmt, int b_fmt, bool a_mn, bool b_mn, int m, int n) {
  return (static_cast<uint32_t>(a_fmt) << 7) | (static_cast<uint32_t>(b_fmt) << 10) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) |
         (static_cast<uint32_t>(n >> 3) << 17) | (1u << 23) | (static_cast<uint32_t>(m >> 7) << 27);
}

struct Fp8Params {
  Operand A, B;
  int contraction;
  int a_bytes;               // bytes of one A copy: fewer than 128 rows where the matrix has fewer
  int b_bytes, width;        // pairs: bytes of one B copy, columns of a tile
  uint32_t idesc;
  int act;
  const uint16_t* bias;      // [B.rows], or null
  const uint8_t* keep;       // flags [A.rows / block, B.rows] of the output, or null
  int block, keep_wide;      // eight flags at a time
  uint16_t* Y;               // where the output's rows are not whole 16-byte pieces (the copy engine writes no less), else null
  int ldy;
  int* status;
};

// Mask flags of eight outputs, a byte each.
__device__ __forceinline__ uint2 output_flags(const Fp8Params& P, int r, int n) {
  if (r >= P.A.rows || n >= P.B.rows) return make_uint2(0u, 0u);
  const uint8_t* f = P.keep + static_cast<size_t>(r / P.block) * P.B.rows + n;
  if (P.keep_wide) return ld_global(reinterpret_cast<const uint2*>(f));            // (then the output's width is a multiple of 8)
  uint2 k = make_uint2(0u, 0u);
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (n + e < P.B.rows) (e < 4 ? k.x : k.y) |= static_cast<uint32_t>(ld_global(f + e)) << (8 * (e & 3));
  return k;
}

// A piece of 32 columns of this warp's 32 rows from the staging buffer, a row at a time.
__device__ __forceinline__ void store_piece_rows(const Fp8Params& P, uint32_t buf, int warp_row, int m0, int col, int lane) {
  __syncwarp();
  for (int r = warp_row; r < warp_row + 32 && m0 + r < P.A.rows; ++r) {
    uint16_t v;
    asm volatile("ld.shared.b16 %0, [%1];" : "=h"(v) : "r"(buf + 64u * r + ((((lane >> 3) ^ (r >> 1)) & 3) << 4) + 2u * (lane & 7)));
    if (col + lane < P.B.rows) P.Y[static_cast<size_t>(m0 + r) * P.ldy + col + lane] = v;
  }
}

template <int BN, bool kAMn, bool kBMn>
__global__ void __launch_bounds__(kFp8Threads, 1)
gemm_fp8_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                const __grid_constant__ CUtensorMap map_y, const __grid_constant__ Fp8Params P) {
  using Cfg = Fp8Cfg<BN>;
  constexpr int S = Cfg::kStages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  // [S operand stages][epilogue staging buffers][scales][bias of two tiles][mbarriers, TMEM base]
  const uint32_t smem_base = smem_u32(smem);
  constexpr int kScalesOff = S * Cfg::kStage + kEpiBytes;
  uint16_t* s_bias = reinterpret_cast<uint16_t*>(smem + kScalesOff + kScaleStages * Cfg::kScaleGroup);
  uint64_t* bars = reinterpret_cast<uint64_t*>(reinterpret_cast<uint8_t*>(s_bias) + 2 * BN * 2);
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(bars + 2 * S + 4 + 2 * kScaleStages);
  volatile uint32_t* timed_out = tmem_holder + 1;     // set by a role whose wait expired
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t bar_base = smem_u32(bars);
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (S + s); };
  auto acc_full_bar = [&](int a) { return bar_base + 8u * (2 * S + a); };
  auto acc_empty_bar = [&](int a) { return bar_base + 8u * (2 * S + 2 + a); };
  auto scale_full_bar = [&](int s) { return bar_base + 8u * (2 * S + 4 + s); };
  auto scale_empty_bar = [&](int s) { return bar_base + 8u * (2 * S + 4 + kScaleStages + s); };

  if (threadIdx.x == 0) {
    *timed_out = 0u;
    for (int s = 0; s < S; ++s) { mbar_init(full_bar(s), 2); mbar_init(empty_bar(s), 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(acc_full_bar(a), 1); mbar_init(acc_empty_bar(a), 8); }
    for (int s = 0; s < kScaleStages; ++s) { mbar_init(scale_full_bar(s), 1); mbar_init(scale_empty_bar(s), 1); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_holder)),
                 "r"(static_cast<uint32_t>(Cfg::kTmemCols)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tcgen05_fence_before();
  __syncthreads();
  tcgen05_fence_after();
  const uint32_t tmem_base = *tmem_holder;
  pdl_wait();
  pdl_launch_dependents();

  const int rows = P.A.rows, cols = P.B.rows;
  const int m_tiles = (rows + kBlockM - 1) / kBlockM;
  const int n_tiles = (cols + BN - 1) / BN;
  const int total_tiles = m_tiles * n_tiles;
  const int k_blocks = blocks_of(P.contraction);

  if (warp == 0) {
    // ---------------------------------------------------------------- TMA producer of A
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int tile = blockIdx.x; tile < total_tiles && ok; tile += gridDim.x) {
      const int m0 = (tile / n_tiles) * kBlockM;
      for (int kb = 0; kb < k_blocks; ++kb) {
        if (!mbar_wait_warp(empty_bar(stage), phase ^ 1u, P.status)) { ok = false; break; }
        const uint32_t dst = smem_base + stage * Cfg::kStage;
        tma_stage_load(dst, &map_a, kAMn ? m0 : kb * kBlock, kAMn ? kb * kBlock : m0, full_bar(stage), static_cast<uint32_t>(P.a_bytes));
        if (++stage == S) { stage = 0; phase ^= 1u; }
      }
    }
    if (!ok && lane == 0) record_timeout(P.status, timed_out);
  } else if (warp == 10) {
    // ---------------------------------------------------------------- TMA producer of B
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int tile = blockIdx.x; tile < total_tiles && ok; tile += gridDim.x) {
      const int n0 = (tile % n_tiles) * BN;
      for (int kb = 0; kb < k_blocks; ++kb) {
        if (!mbar_wait_warp(empty_bar(stage), phase ^ 1u, P.status)) { ok = false; break; }
        const uint32_t dst = smem_base + stage * Cfg::kStage + Cfg::kStageA;
        tma_stage_load(dst, &map_b, kBMn ? n0 : kb * kBlock, kBMn ? kb * kBlock : n0, full_bar(stage), Cfg::kStageB);
        if constexpr (kBMn) {
#pragma unroll
          for (int g = 1; g < BN / 128; ++g) tma_load_2d_elect(dst + g * kGroupMn, &map_b, n0 + 128 * g, kb * kBlock, full_bar(stage));
        }
        if (++stage == S) { stage = 0; phase ^= 1u; }
      }
    }
    if (!ok && lane == 0) record_timeout(P.status, timed_out);
  } else if (warp == 11) {
    // ---------------------------------------------------------------- scales
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int tile = blockIdx.x; tile < total_tiles && ok; tile += gridDim.x) {
      const int m0 = (tile / n_tiles) * kBlockM, n0 = (tile % n_tiles) * BN;
      for (int kb = 0; kb < k_blocks; kb += 4) {
        Scales a, b[Cfg::kTilesB];
        a.load(P.A, m0, kb, k_blocks, lane);
#pragma unroll
        for (int i = 0; i < Cfg::kTilesB; ++i) b[i].load(P.B, n0 + 128 * i, kb, k_blocks, lane);
        if (!mbar_wait_warp(scale_empty_bar(stage), phase ^ 1u, P.status)) { ok = false; break; }
        const uint32_t dst = smem_base + kScalesOff + stage * Cfg::kScaleGroup;
        store_scales(P.A, dst, a.finish(P.A, m0, kb, lane), lane);
#pragma unroll
        for (int i = 0; i < Cfg::kTilesB; ++i) store_scales(P.B, dst + (1 + i) * kScaleTile, b[i].finish(P.B, n0 + 128 * i, kb, lane), lane);
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(scale_full_bar(stage));
        if (++stage == kScaleStages) { stage = 0; phase ^= 1u; }
      }
    }
    if (!ok && lane == 0) record_timeout(P.status, timed_out);
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMA issuer
    int stage = 0, scale_stage = 0;
    uint32_t phase = 0, scale_phase = 0, scale_buf = 0;
    uint32_t acc_phase[2] = {0u, 0u};
    int acc = 0;
    bool ok = true;
    for (int tile = blockIdx.x; tile < total_tiles && ok; tile += gridDim.x) {
      if (!mbar_wait_warp(acc_empty_bar(acc), acc_phase[acc] ^ 1u, P.status)) { ok = false; break; }
      tcgen05_fence_after();
      const uint32_t d_tmem = tmem_base + static_cast<uint32_t>(acc * BN);
      uint32_t sfa = 0u;
      for (int kb = 0; kb < k_blocks; ++kb) {
        if ((kb & 3) == 0) {
          // the next four blocks' scales (two sets of columns in turn: the instructions before still read the other one)
          if (!mbar_wait_warp(scale_full_bar(scale_stage), scale_phase, P.status)) { ok = false; break; }
          tcgen05_fence_after();
          const uint32_t src = smem_base + kScalesOff + scale_stage * Cfg::kScaleGroup;
          sfa = tmem_base + static_cast<uint32_t>(2 * BN) + scale_buf * Cfg::kScaleCols;
          scale_buf ^= 1u;
#pragma unroll
          for (int i = 0; i < 1 + Cfg::kTilesB; ++i) copy_scales(sfa + 4u * i, src + i * kScaleTile);
          tcgen05_commit_elect(scale_empty_bar(scale_stage));
          if (++scale_stage == kScaleStages) { scale_stage = 0; scale_phase ^= 1u; }
        }
        if (!mbar_wait_warp(full_bar(stage), phase, P.status)) { ok = false; break; }
        tcgen05_fence_after();
        const uint32_t a_addr = smem_base + stage * Cfg::kStage, b_addr = a_addr + Cfg::kStageA;
        const uint32_t idesc = P.idesc | (static_cast<uint32_t>(kb & 3) << 29) | (static_cast<uint32_t>(kb & 3) << 4);
        mma_stage_scaled<kAMn ? 256 : 2, kBMn ? 256 : 2>(d_tmem, kAMn ? smem_desc_mn8(a_addr) : smem_desc_sw128(a_addr),
                                                         kBMn ? smem_desc_mn8(b_addr) : smem_desc_sw128(b_addr), idesc, kb != 0 ? 1u : 0u,
                                                         empty_bar(stage), sfa, sfa + 4u);
        if (++stage == S) { stage = 0; phase ^= 1u; }
      }
      if (!ok) break;
      tcgen05_commit_elect(acc_full_bar(acc));
      acc_phase[acc] ^= 1u;
      acc ^= 1;
    }
    if (!ok && lane == 0) record_timeout(P.status, timed_out);
  } else {
    // ---------------------------------------------------------------- epilogue
    const int group = (warp - 2) >> 2;
    const int quad = warp & 3;
    const int row = quad * 32 + lane;
    const int epi_tid = threadIdx.x - 64;
    const bool issuer = (epi_tid & 127) == 0;
    const uint32_t buf0 = smem_base + S * Cfg::kStage + group * 2 * kEpiStage;
    uint32_t my_piece = 0;
    const uint32_t row_off = static_cast<uint32_t>(row) * 64u;
    const uint32_t row_xor = static_cast<uint32_t>((row >> 1) & 3);
    uint32_t acc_phase[2] = {0u, 0u};
    int acc = 0;
    bool ok = true;
    for (int tile = blockIdx.x; tile < total_tiles && ok; tile += gridDim.x) {
      const int m0 = (tile / n_tiles) * kBlockM, n0 = (tile % n_tiles) * BN;
      for (int c = epi_tid; c < BN; c += 256)
        s_bias[acc * BN + c] = (P.bias != nullptr && n0 + c < cols) ? ld_global(P.bias + n0 + c) : static_cast<uint16_t>(0);
      epilogue_sync_all();
      // all 256 threads take the same decision, so nobody is left alone at a named barrier below
      if (!epilogue_all_ok(mbar_wait(acc_full_bar(acc), acc_phase[acc], P.status))) { ok = false; break; }
      tcgen05_fence_after();
      const uint32_t taddr = tmem_base + (static_cast<uint32_t>(quad * 32) << 16) + static_cast<uint32_t>(acc * BN);
      const int pieces = (min(BN, cols - n0) + kEpiCols - 1) / kEpiCols;
      bool released = false;
#pragma unroll 1
      for (int pc = group; pc < pieces; pc += 2) {
        const int c0 = pc * kEpiCols;
        const uint32_t buf = buf0 + (my_piece & 1u) * kEpiStage;
        ++my_piece;
        uint2 flags[kEpiCols / 8];
        if (P.keep != nullptr) {
#pragma unroll
          for (int j = 0; j < kEpiCols / 8; ++j) flags[j] = output_flags(P, m0 + row, n0 + c0 + 8 * j);
        }
        EpiloguePiece piece;
        piece_load(taddr + c0, smem_u32(s_bias + acc * BN + c0), piece);
        if (P.keep != nullptr) {
#pragma unroll
          for (int i = 0; i < kEpiCols; ++i)
            if ((((i & 4 ? flags[i >> 3].y : flags[i >> 3].x) >> (8 * (i & 3))) & 0xffu) == 0u) piece.v[i] = 0u;
        }
        if (issuer) tma_store_wait_read<1>();
        group_sync(group);
        if (pc + 2 >= pieces) {
          tcgen05_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(acc_empty_bar(acc));
          released = true;
        }
        piece_store(piece, P.act, buf + row_off, row_xor);
        if (P.Y != nullptr) {
          store_piece_rows(P, buf, quad * 32, m0, n0 + c0, lane);
        } else {
          fence_async_smem();
          group_sync(group);
          if (issuer) tma_store_2d(&map_y, n0 + c0, m0, buf);
        }
      }
      if (!released) {
        tcgen05_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(acc_empty_bar(acc));
      }
      acc_phase[acc] ^= 1u;
      acc ^= 1;
    }
    if (issuer) tma_store_wait_read<0>();
    if (!ok && lane == 0) record_timeout(P.status, timed_out);
  }

  tcgen05_fence_before();
  __syncthreads();
  quiet_period(timed_out);
  if (warp == 1) {
    tcgen05_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(static_cast<uint32_t>(Cfg::kTmemCols)) : "memory");
  }
}

// ------------------------------------------------------------------------------------------ CTA pairs
// Two CTAs of a cluster share a tile of 256 x w outputs, as in bsp_linear_tc2.cu: each loads its own 128 rows of A and half of the
// w rows of B, and the instructions of the leader (cta_group::2) read both.  8-bit operands are multiplied twice as fast as
// bf16 ones, so the path from L2 binds sooner: a 128-deep stage of a 128 x 128 tile is 32 KB, 0.3 us at the 115 bytes per ns
// that an SM gets, for 0.14 us of tensor work; a CTA of a 256 x 256 pair has the same 32 KB for 0.28 us.
// The width is the launch's (choose_pair): up to 240 two accumulators fit tensor memory beside the scales; wider tiles have one, which
// the epilogue empties into registers before it does anything else (0.3 us).
// Every CTA holds the scales of its own rows of A and of all rows of B of the tile.
constexpr int kPairStage = 2 * kBlockM * kBlock;           // 128 rows of A, up to 128 of B
constexpr int kPairStages = 6;
constexpr int kPairEpi = 2 * kEpiStage;                    // one staging buffer for each epilogue group
constexpr int kPairScaleGroup = 3 * kScaleTile;
constexpr int kPairMaxW = 256;
constexpr int kPairSmem = 1024 + kPairStages * kPairStage + kPairEpi + kScaleStages * kPairScaleGroup + 2 * kPairMaxW * 2 + 256;
constexpr int kPairScaleCols = 12;
static_assert(kPairSmem <= kSmemLimit, "shared memory");
__host__ __device__ constexpr int pair_accumulators(int w) { return 2 * w + 2 * kPairScaleCols <= 512 ? 2 : 1; }

__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar_leader, uint32_t bar_own, uint32_t arm) {
  asm volatile(
      "{\n\t.reg .pred e, a;\n\telect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.and.u32 a, %6, 0, e;\n\t"
      "@a mbarrier.arrive.expect_tx.shared::cta.b64 _, [%5], %6;\n\t"
      "@e cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar_leader), "r"(bar_own), "r"(arm)
      : "memory");
}
// Commits to the same barrier of both CTAs.
__device__ __forceinline__ void commit_both(uint32_t bar_own, uint32_t bar_peer) {
  asm volatile(
      "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t"
      "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%1];\n\t}" ::"r"(bar_own), "r"(bar_peer)
      : "memory");
}
__device__ __forceinline__ void copy_scales_pair(uint32_t taddr, uint32_t smem_addr) {
  asm volatile(
      "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;\n\t}" ::"r"(taddr), "l"(scale_desc(smem_addr))
      : "memory");
}
template <int STEP_A, int STEP_B>
__device__ __forceinline__ void mma_stage_scaled_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate,
                                                      uint32_t free_own, uint32_t free_peer, uint32_t sfa, uint32_t sfb) {
  asm volatile(
      "{\n\t.reg .pred p, t, e;\n\t.reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.eq.b32 t, 0, 0;\n\t"
      "add.s64 a1, %1, %9;\n\tadd.s64 a2, a1, %9;\n\tadd.s64 a3, a2, %9;\n\t"
      "add.s64 b1, %2, %10;\n\tadd.s64 b2, b1, %10;\n\tadd.s64 b3, b2, %10;\n\t"
      "@e tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%7], [%8], p;\n\t"
      "@e tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a1, b1, %3, [%7], [%8], t;\n\t"
      "@e tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a2, b2, %3, [%7], [%8], t;\n\t"
      "@e tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a3, b3, %3, [%7], [%8], t;\n\t"
      "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%5];\n\t"
      "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%6];\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(free_own), "r"(free_peer), "r"(sfa), "r"(sfb), "n"(STEP_A), "n"(STEP_B)
      : "memory");
}
__device__ __forceinline__ void mbar_arrive_remote(uint32_t bar_cluster) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar_cluster) : "memory");
}
// The same where it hands over what this CTA has written to its own shared memory (behind a fence to the copies that read it).
__device__ __forceinline__ void mbar_arrive_remote_release(uint32_t bar_cluster) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar_cluster) : "memory");
}

// A warp's wait that sees what the other CTA wrote before such an arrival.
__device__ __forceinline__ bool mbar_try_cluster(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool mbar_wait_cluster(uint32_t bar, uint32_t parity, const int* status) {
  if (__all_sync(0xffffffffu, mbar_try_cluster(bar, parity))) return true;
  const unsigned long long limit = wait_limit_ns(status);
  const unsigned long long start = global_timer_ns();
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 256; ++i)
      if (__all_sync(0xffffffffu, mbar_try_cluster(bar, parity))) return true;
    if (__any_sync(0xffffffffu, global_timer_ns() - start > limit)) return false;
  }
}

template <bool kAMn, bool kBMn>
__global__ void __launch_bounds__(kFp8Threads, 1)
gemm_fp8_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                     const __grid_constant__ CUtensorMap map_y, const __grid_constant__ Fp8Params P) {
  constexpr int S = kPairStages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  // [S operand stages][epilogue staging buffers][scales][bias of two tiles][mbarriers, TMEM base]
  const uint32_t smem_base = smem_u32(smem);
  constexpr int kScalesOff = S * kPairStage + kPairEpi;
  uint16_t* s_bias = reinterpret_cast<uint16_t*>(smem + kScalesOff + kScaleStages * kPairScaleGroup);
  uint64_t* bars = reinterpret_cast<uint64_t*>(reinterpret_cast<uint8_t*>(s_bias) + 2 * kPairMaxW * 2);
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(bars + 2 * S + 4 + 2 * kScaleStages);
  volatile uint32_t* timed_out = tmem_holder + 1;     // set by a role of this CTA whose wait expired
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();               // 0 = leader of the pair
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
  const uint32_t bar_base = smem_u32(bars);
  auto full_bar = [&](int s) { return bar_base + 8u * s; };                       // used in the leader only
  auto empty_bar = [&](int s) { return bar_base + 8u * (S + s); };                // one per CTA
  auto acc_full_bar = [&](int a) { return bar_base + 8u * (2 * S + a); };         // one per CTA
  auto acc_empty_bar = [&](int a) { return bar_base + 8u * (2 * S + 2 + a); };    // used in the leader only
  auto scale_full_bar = [&](int s) { return bar_base + 8u * (2 * S + 4 + s); };   // used in the leader only
  auto scale_empty_bar = [&](int s) { return bar_base + 8u * (2 * S + 4 + kScaleStages + s); };   // one per CTA

  if (threadIdx.x == 0) {
    *timed_out = 0u;
    for (int s = 0; s < S; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(acc_full_bar(a), 1); mbar_init(acc_empty_bar(a), 16); }   // 8 warps x 2 CTAs
    for (int s = 0; s < kScaleStages; ++s) { mbar_init(scale_full_bar(s), 4); mbar_init(scale_empty_bar(s), 1); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {   // the same warp in both CTAs, same destination offset
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_holder)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tcgen05_fence_before();
  __syncthreads();
  cluster_arrive_relaxed();      // this CTA's barriers exist (fenced above) and its tensor memory is allocated
  tcgen05_fence_after();
  const uint32_t tmem_base = *tmem_holder;
  pdl_wait();
  pdl_launch_dependents();
  cluster_wait();                // and so do the other's, before anything signals across the pair

  const int rows = P.A.rows, cols = P.B.rows, w = P.width;
  const int m_tiles = (rows - 1) / 256 + 1;
  const int n_tiles = (cols - 1) / w + 1;
  const int total_tiles = m_tiles * n_tiles;
  const int k_blocks = blocks_of(P.contraction);
  const int accs = pair_accumulators(w);
  const int tiles_b = (w + 127) >> 7;                  // sets of 128 rows of B with scales

  if (warp == 0) {
    // ---------------------------------------------------------------- TMA producer (both CTAs)
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int tile = pair; tile < total_tiles && ok; tile += n_pairs) {
      const int m0 = (tile / n_tiles) * 256 + static_cast<int>(rank) * kBlockM, n0 = (tile % n_tiles) * w + static_cast<int>(rank) * (w / 2);
      for (int kb = 0; kb < k_blocks; ++kb) {
        if (!mbar_wait_warp(empty_bar(stage), phase ^ 1u, P.status)) { ok = false; break; }
        const uint32_t dst = smem_base + stage * kPairStage, leader_full = map_to_cta(full_bar(stage), 0);
        tma_load_pair(dst, &map_a, kAMn ? m0 : kb * kBlock, kAMn ? kb * kBlock : m0, leader_full, full_bar(stage),
                      rank == 0 ? 2u * static_cast<uint32_t>(kBlockM * kBlock + P.b_bytes) : 0u);       // both CTAs' bytes
        tma_load_pair(dst + kBlockM * kBlock, &map_b, kBMn ? n0 : kb * kBlock, kBMn ? kb * kBlock : n0, leader_full, full_bar(stage), 0u);
        if (++stage == S) { stage = 0; phase ^= 1u; }
      }
    }
    // the leader's commits that free the last stages arrive here while this CTA still exists
    for (int i = 0; i < S && ok; ++i) {
      ok = mbar_wait_warp(empty_bar(stage), phase ^ 1u, P.status);
      if (++stage == S) { stage = 0; phase ^= 1u; }
    }
    if (!ok && lane == 0) record_timeout(P.status, timed_out);
  } else if (warp >= 10) {
    // ---------------------------------------------------------------- scales (both CTAs): warp 10 its own rows of A, warp 11 all rows of B
    const bool for_a = warp == 10;
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    int tile = pair, kb = 0;
    Scales s0, s1;
    int m0, n0;
    auto fetch = [&] {
      m0 = (tile / n_tiles) * 256 + static_cast<int>(rank) * kBlockM;
      n0 = (tile % n_tiles) * w;
      if (for_a) {
        s0.load(P.A, m0, kb, k_blocks, lane);
      } else {
        s0.load(P.B, n0, kb, k_blocks, lane);
        if (tiles_b > 1) s1.load(P.B, n0 + 128, kb, k_blocks, lane);
      }
    };
    if (tile < total_tiles) fetch();
    while (tile < total_tiles) {
      if (!mbar_wait_warp(scale_empty_bar(stage), phase ^ 1u, P.status)) { ok = false; break; }
      const uint32_t dst = smem_base + kScalesOff + stage * kPairScaleGroup;
      if (for_a) {
        store_scales(P.A, dst, s0.finish(P.A, m0, kb, lane), lane);
      } else {
        store_scales(P.B, dst + kScaleTile, s0.finish(P.B, n0, kb, lane), lane);
        if (tiles_b > 1) store_scales(P.B, dst + 2 * kScaleTile, s1.finish(P.B, n0 + 128, kb, lane), lane);
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive_remote_release(map_to_cta(scale_full_bar(stage), 0));
      if (++stage == kScaleStages) { stage = 0; phase ^= 1u; }
      kb += 4;
      if (kb >= k_blocks) { kb = 0; tile += n_pairs; }
      if (tile < total_tiles) fetch();                 // (in flight while the next group waits for its place)
    }
    for (int i = 0; i < kScaleStages && ok; ++i) {     // as for the stages
      ok = mbar_wait_warp(scale_empty_bar(stage), phase ^ 1u, P.status);
      if (++stage == kScaleStages) { stage = 0; phase ^= 1u; }
    }
    if (!ok && lane == 0) record_timeout(P.status, timed_out);
  } else if (warp == 1 && rank == 0) {
    // ---------------------------------------------------------------- MMA issuer (leader CTA only)
    int stage = 0, scale_stage = 0;
    uint32_t phase = 0, scale_phase = 0, scale_buf = 0, acc_phases = 0;
    int acc = 0;
    bool ok = true;
    for (int tile = pair; tile < total_tiles && ok; tile += n_pairs) {
      if (!mbar_wait_warp(acc_empty_bar(acc), ((acc_phases >> acc) & 1u) ^ 1u, P.status)) { ok = false; break; }
      tcgen05_fence_after();
      const uint32_t d_tmem = tmem_base + static_cast<uint32_t>(acc * w);
      uint32_t sfa = 0u;
      for (int kb = 0; kb < k_blocks; ++kb) {
        if ((kb & 3) == 0) {
          // the next four blocks' scales (two sets of columns in turn: the instructions before still read the other one)
          if (!mbar_wait_cluster(scale_full_bar(scale_stage), scale_phase, P.status)) { ok = false; break; }
          tcgen05_fence_after();
          const uint32_t src = smem_base + kScalesOff + scale_stage * kPairScaleGroup;
          sfa = tmem_base + 512u - 2u * kPairScaleCols + scale_buf * kPairScaleCols;
          scale_buf ^= 1u;
          for (int i = 0; i <= tiles_b; ++i) copy_scales_pair(sfa + 4u * i, src + i * kScaleTile);
          commit_both(scale_empty_bar(scale_stage), map_to_cta(scale_empty_bar(scale_stage), 1));
          if (++scale_stage == kScaleStages) { scale_stage = 0; scale_phase ^= 1u; }
        }
        if (!mbar_wait_warp(full_bar(stage), phase, P.status)) { ok = false; break; }
        tcgen05_fence_after();
        const uint32_t a_addr = smem_base + stage * kPairStage, b_addr = a_addr + kBlockM * kBlock;
        const uint32_t idesc = P.idesc | (static_cast<uint32_t>(kb & 3) << 29) | (static_cast<uint32_t>(kb & 3) << 4);
        mma_stage_scaled_pair<kAMn ? 256 : 2, kBMn ? 256 : 2>(d_tmem, kAMn ? smem_desc_mn8(a_addr) : smem_desc_sw128(a_addr),
                                                              kBMn ? smem_desc_mn8(b_addr) : smem_desc_sw128(b_addr), idesc, kb != 0 ? 1u : 0u,
                                                              empty_bar(stage), map_to_cta(empty_bar(stage), 1), sfa, sfa + 4u);
        if (++stage == S) { stage = 0; phase ^= 1u; }
      }
      if (!ok) break;
      commit_both(acc_full_bar(acc), map_to_cta(acc_full_bar(acc), 1));
      acc_phases ^= 1u << acc;
      if (accs == 2) acc ^= 1;
    }
    if (!ok && lane == 0) record_timeout(P.status, timed_out);
  } else if (warp >= 2 && warp < 10) {
    // ---------------------------------------------------------------- epilogue of this CTA's 128 rows
    const int group = (warp - 2) >> 2;
    const int quad = warp & 3;
    const int row = quad * 32 + lane;
    const int epi_tid = threadIdx.x - 64;
    const bool issuer = (epi_tid & 127) == 0;
    const uint32_t buf = smem_base + S * kPairStage + group * kEpiStage;
    const uint32_t row_off = static_cast<uint32_t>(row) * 64u;
    const uint32_t row_xor = static_cast<uint32_t>((row >> 1) & 3);
    constexpr int kPieces = kPairMaxW / kEpiCols / 2;            // of a tile that a group takes, at most
    uint32_t acc_phases = 0, bias_buf = 0;
    int acc = 0;
    bool ok = true;
    for (int tile = pair; tile < total_tiles && ok; tile += n_pairs) {
      const int m0 = (tile / n_tiles) * 256 + static_cast<int>(rank) * kBlockM, n0 = (tile % n_tiles) * w;
      for (int c = epi_tid; c < w; c += 256)
        s_bias[bias_buf * kPairMaxW + c] = (P.bias != nullptr && n0 + c < cols) ? ld_global(P.bias + n0 + c) : static_cast<uint16_t>(0);
      epilogue_sync_all();
      // all 256 threads take the same decision, so nobody is left alone at a named barrier below
      if (!epilogue_all_ok(mbar_wait(acc_full_bar(acc), (acc_phases >> acc) & 1u, P.status))) { ok = false; break; }
      tcgen05_fence_after();
      const uint32_t taddr = tmem_base + (static_cast<uint32_t>(quad * 32) << 16) + static_cast<uint32_t>(acc * w);
      const int pieces = (min(w, cols - n0) + kEpiCols - 1) / kEpiCols;
      // (the last piece of a tile whose width is no multiple of 32 begins early: both write the same values)
      auto first_col = [&](int pc) { return min(pc * kEpiCols, w - kEpiCols); };
      uint32_t v[kPieces][32];
#pragma unroll
      for (int i = 0; i < kPieces; ++i)
        if (group + 2 * i < pieces) tmem_load_32cols(taddr + first_col(group + 2 * i), v[i]);
      tmem_load_wait();
#pragma unroll
      for (int i = 0; i < kPieces; ++i) tmem_loaded<32>(v[i]);
      // (the last accumulators are not waited for again: no arrival that could come when the leader has left)
      if (tile + accs * n_pairs < total_tiles) {
        tcgen05_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_remote(map_to_cta(acc_empty_bar(acc), 0));
      }
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        const int pc = group + 2 * i;
        if (pc >= pieces) break;
        const int c0 = first_col(pc);
        if (P.keep != nullptr) {
#pragma unroll
          for (int j = 0; j < kEpiCols / 8; ++j) {
            const uint2 f = output_flags(P, m0 + row, n0 + c0 + 8 * j);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if ((((e < 4 ? f.x : f.y) >> (8 * (e & 3))) & 0xffu) == 0u) v[i][8 * j + e] = 0u;
          }
        }
        EpiloguePiece piece;
#pragma unroll
        for (int e = 0; e < 32; ++e) piece.v[e] = v[i][e];
#pragma unroll
        for (int j = 0; j < 4; ++j) piece.bias[j] = ld_shared_v4(smem_u32(s_bias + bias_buf * kPairMaxW + c0) + 16u * j);
        if (issuer) tma_store_wait_read<0>();    // the store before has read this buffer
        group_sync(group);
        piece_store(piece, P.act, buf + row_off, row_xor);
        if (P.Y != nullptr) {
          store_piece_rows(P, buf, quad * 32, m0, n0 + c0, lane);
        } else {
          fence_async_smem();
          group_sync(group);
          if (issuer) tma_store_2d(&map_y, n0 + c0, m0, buf);
        }
      }
      acc_phases ^= 1u << acc;
      if (accs == 2) acc ^= 1;
      bias_buf ^= 1u;
    }
    if (issuer) tma_store_wait_read<0>();
    if (!ok && lane == 0) record_timeout(P.status, timed_out);
  }

  tcgen05_fence_before();
  __syncthreads();
  quiet_period(timed_out);
  // neither CTA leaves, or frees its tensor memory, while the other may still touch them (nothing is in flight between them by now)
  cluster_arrive_relaxed();
  cluster_wait();
  if (warp == 1) {
    tcgen05_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
  }
}

// 8-bit matrix [outer, inner], boxes of 128 x box_outer, 128-byte swizzle; what lies outside reads as zero.
bool make_map8(CUtensorMap* map, const void* base, uint64_t inner, uint64_t outer, uint64_t ld, uint32_t box_outer) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {inner, outer};
  const cuuint64_t strides[1] = {ld};
  const cuuint32_t box[2] = {kBlock, box_outer};
  const cuuint32_t elem[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The driver's encoder wants a current context, which a thread that has only asked the runtime for facts does not have.
bool make_current() {
  int device = 0;
  return cudaGetDevice(&device) == cudaSuccess && cudaSetDevice(device) == cudaSuccess;
}

template <int BN, bool kAMn, bool kBMn>
int launch(const Product& p, TcDevice* dev, cudaStream_t s) {
  using Cfg = Fp8Cfg<BN>;
  static_assert(Cfg::kStages >= 4 && Cfg::kStage % 1024 == 0 && (!kBMn || BN % 128 == 0), "stages");
  static OncePerDevice once;
  BSP_TRY(allow_dynamic_smem(once, gemm_fp8_kernel<BN, kAMn, kBMn>, Cfg::kSmemBytes));
  CUtensorMap map_a, map_b, map_y;
  const bool whole = aligned_to(p.Y, 16) && p.ldy % 8 == 0 && p.B.rows % 8 == 0;
  if (!(whole ? make_map(&map_y, p.Y, p.B.rows, p.A.rows, p.ldy, kBlockM, kEpiCols) : make_current())) return BSP_ERR_CUDA;
  if (!whole) map_y = CUtensorMap{};
  const int a_rows = kAMn ? kBlock : copy_rows(p.A.rows);
  if (!(kAMn ? make_map8(&map_a, p.A.q, p.A.rows, p.contraction, p.A.ld, kBlock) : make_map8(&map_a, p.A.q, p.contraction, p.A.rows, p.A.ld, a_rows)) ||
      !(kBMn ? make_map8(&map_b, p.B.q, p.B.rows, p.contraction, p.B.ld, kBlock) : make_map8(&map_b, p.B.q, p.contraction, p.B.rows, p.B.ld, BN)))
    return BSP_ERR_CUDA;
  const Fp8Params P{p.A, p.B, p.contraction, a_rows * kBlock, 0, BN, idesc_scaled(p.A.fmt, p.B.fmt, kAMn, kBMn, kBlockM, BN), p.act, p.bias, p.keep, p.block,
                    aligned_to(p.keep, 8) && p.B.rows % 8 == 0, whole ? nullptr : p.Y, p.ldy, dev->status};
  const long long tiles = static_cast<long long>((p.A.rows + kBlockM - 1) / kBlockM) * ((p.B.rows + BN - 1) / BN);
  BSP_CUDA_TRY(launch_pdl(gemm_fp8_kernel<BN, kAMn, kBMn>, dim3(tiles < dev->sms ? static_cast<unsigned>(tiles) : dev->sms), dim3(kFp8Threads),
                          Cfg::kSmemBytes, s, map_a, map_b, map_y, P));
  return BSP_OK;
}

template <bool kAMn, bool kBMn>
int launch_pair(const Product& p, int w, TcDevice* dev, cudaStream_t s) {
  static OncePerDevice once;
  BSP_TRY(allow_dynamic_smem(once, gemm_fp8_pair_kernel<kAMn, kBMn>, kPairSmem));
  CUtensorMap map_a, map_b, map_y;
  const bool whole = aligned_to(p.Y, 16) && p.ldy % 8 == 0 && p.B.rows % 8 == 0;
  if (!(whole ? make_map(&map_y, p.Y, p.B.rows, p.A.rows, p.ldy, kBlockM, kEpiCols) : make_current())) return BSP_ERR_CUDA;
  if (!whole) map_y = CUtensorMap{};
  const int b_rows = kBMn ? kBlock : w / 2;
  if (!(kAMn ? make_map8(&map_a, p.A.q, p.A.rows, p.contraction, p.A.ld, kBlock) : make_map8(&map_a, p.A.q, p.contraction, p.A.rows, p.A.ld, kBlockM)) ||
      !(kBMn ? make_map8(&map_b, p.B.q, p.B.rows, p.contraction, p.B.ld, kBlock) : make_map8(&map_b, p.B.q, p.contraction, p.B.rows, p.B.ld, b_rows)))
    return BSP_ERR_CUDA;
  const Fp8Params P{p.A, p.B, p.contraction, kBlockM * kBlock, b_rows * kBlock, w, idesc_scaled(p.A.fmt, p.B.fmt, kAMn, kBMn, 256, w), p.act, p.bias,
                    p.keep, p.block, aligned_to(p.keep, 8) && p.B.rows % 8 == 0, whole ? nullptr : p.Y, p.ldy, dev->status};
  const long long tiles = static_cast<long long>((p.A.rows - 1) / 256 + 1) * ((p.B.rows - 1) / w + 1);
  const int pairs = tiles < dev->sms / 2 ? static_cast<int>(tiles) : dev->sms / 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * pairs);
  cfg.blockDim = dim3(kFp8Threads);
  cfg.dynamicSmemBytes = kPairSmem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  BSP_CUDA_TRY(cudaLaunchKernelEx(&cfg, gemm_fp8_pair_kernel<kAMn, kBMn>, map_a, map_b, map_y, P));
  return BSP_OK;
}

// Width of the pairs' tiles for an output of rows x cols, with its estimated time in ns: waves of tiles, a stage of each bound by
// the tensor cores or by the path from L2.
int choose_pair(int rows, int cols, int k_blocks, bool b_mn, int sms, double* ns) {
  int best = 0;
  for (const int w : {64, 96, 128, 160, 192, 224, 240, 256}) {
    if (b_mn && w % 32 != 0) continue;              // (half a tile's columns begin at a multiple of 16 bytes)
    const long long tiles = static_cast<long long>((rows - 1) / 256 + 1) * ((cols - 1) / w + 1);
    const long long waves = (tiles + sms / 2 - 1) / (sms / 2);
    const double stage = fmax(1.1 * w, (16384 + (b_mn ? 16384 : 64 * w)) / 115.0);
    const double t = waves * (k_blocks * stage + (pair_accumulators(w) == 2 ? 0.0 : 500.0)) + 6.0 * w;
    if (best == 0 || t < *ns) { best = w; *ns = t; }
  }
  return best;
}

}  // namespace

namespace fp8 {

bool tensor_core_ok(const Product& p) {
  const long long tiles = static_cast<long long>((p.A.rows + kBlockM - 1) / kBlockM) * ((p.B.rows + 127) / 128);
  return aligned_to(p.A.q, 16) && p.A.ld % 16 == 0 && aligned_to(p.B.q, 16) && p.B.ld % 16 == 0 && tiles <= 0x7fffffffLL;
}

int launch_tensor_core(const Product& p, cudaStream_t s) {
  TcDevice* dev = tc_device();
  if (dev == nullptr) return BSP_ERR_CUDA;
  if (p.A.rows > kBlockM) {
    double ns = 0.0;
    const int w = choose_pair(p.A.rows, p.B.rows, blocks_of(p.contraction), p.B.mn, dev->sms, &ns);
    return p.A.mn ? launch_pair<true, true>(p, w, dev, s) : p.B.mn ? launch_pair<false, true>(p, w, dev, s) : launch_pair<false, false>(p, w, dev, s);
  }
  if (p.A.mn) return launch<128, true, true>(p, dev, s);
  if (p.B.mn) return launch<128, false, true>(p, dev, s);
  return launch<128, false, false>(p, dev, s);
}

}  // namespace fp8
}  // namespace bsp
