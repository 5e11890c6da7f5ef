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

// Scales of a group of four blocks (from `block0` on) of 128 rows (from `row0` on): lane l fetches those of rows l, l + 32, ...
// as the 32-bit words of its 16 bytes.  What does not exist is 1.
__device__ __forceinline__ uint4 fetch_scales(const Operand& O, int row0, int block0, int blocks, int lane) {
  uint32_t w[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int r = row0 + lane + 32 * q;
    const uint8_t* p = O.s + static_cast<long long>(r >> O.s_shift) * O.s_row + static_cast<long long>(block0) * O.s_k;
    w[q] = 0u;
#pragma unroll
    for (int b = 0; b < 4; ++b)
      w[q] |= (r < O.rows && block0 + b < blocks ? static_cast<uint32_t>(ld_global(p + b * O.s_k)) : 127u) << (8 * b);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
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
__host__ __device__ constexpr uint32_t idesc_scaled(int a_fmt, int b_fmt, bool a_mn, bool b_mn, int n) {
  return (static_cast<uint32_t>(a_fmt) << 7) | (static_cast<uint32_t>(b_fmt) << 10) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) |
         (static_cast<uint32_t>(n >> 3) << 17) | (1u << 23) | (static_cast<uint32_t>(kBlockM >> 7) << 27);
}

struct Fp8Params {
  Operand A, B;
  int contraction;
  int a_bytes;               // bytes of one A copy: fewer than 128 rows where the matrix has fewer
  uint32_t idesc;
  int act;
  const uint16_t* bias;      // [B.rows], or null
  const uint8_t* keep;       // flags [A.rows / block, B.rows] of the output, or null
  int block, keep_wide;      // eight flags at a time
  uint16_t* Y;               // where the output's rows are not whole 16-byte pieces (the copy engine writes no less), else null
  int ldy;
  int* status;
};

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
        const uint4 a = fetch_scales(P.A, m0, kb, k_blocks, lane);
        uint4 b[Cfg::kTilesB];
#pragma unroll
        for (int i = 0; i < Cfg::kTilesB; ++i) b[i] = fetch_scales(P.B, n0 + 128 * i, kb, k_blocks, lane);
        if (!mbar_wait_warp(scale_empty_bar(stage), phase ^ 1u, P.status)) { ok = false; break; }
        const uint32_t dst = smem_base + kScalesOff + stage * Cfg::kScaleGroup + 16u * lane;
        st_shared_v4(dst, a.x, a.y, a.z, a.w);
#pragma unroll
        for (int i = 0; i < Cfg::kTilesB; ++i) st_shared_v4(dst + (1 + i) * kScaleTile, b[i].x, b[i].y, b[i].z, b[i].w);
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
          for (int j = 0; j < kEpiCols / 8; ++j) {
            const int n = n0 + c0 + 8 * j;
            flags[j] = make_uint2(0x01010101u, 0x01010101u);
            if (m0 + row < rows && n < cols) {
              const uint8_t* f = P.keep + static_cast<size_t>((m0 + row) / P.block) * cols + n;
              if (P.keep_wide) {                       // (then cols is a multiple of 8)
                flags[j] = ld_global(reinterpret_cast<const uint2*>(f));
              } else {
                flags[j] = make_uint2(0u, 0u);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                  if (n + e < cols) (e < 4 ? flags[j].x : flags[j].y) |= static_cast<uint32_t>(ld_global(f + e)) << (8 * (e & 3));
              }
            }
          }
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
  const Fp8Params P{p.A, p.B, p.contraction, a_rows * kBlock, idesc_scaled(p.A.fmt, p.B.fmt, kAMn, kBMn, BN), p.act, p.bias, p.keep, p.block,
                    aligned_to(p.keep, 8) && p.B.rows % 8 == 0, whole ? nullptr : p.Y, p.ldy, dev->status};
  const long long tiles = static_cast<long long>((p.A.rows + kBlockM - 1) / kBlockM) * ((p.B.rows + BN - 1) / BN);
  BSP_CUDA_TRY(launch_pdl(gemm_fp8_kernel<BN, kAMn, kBMn>, dim3(tiles < dev->sms ? static_cast<unsigned>(tiles) : dev->sms), dim3(kFp8Threads),
                          Cfg::kSmemBytes, s, map_a, map_b, map_y, P));
  return BSP_OK;
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
  if (p.A.mn) return launch<128, true, true>(p, dev, s);
  if (p.B.mn) return launch<128, false, true>(p, dev, s);
  return launch<128, false, false>(p, dev, s);
}

}  // namespace fp8
}  // namespace bsp
