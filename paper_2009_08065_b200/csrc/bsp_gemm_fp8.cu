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
#include <algorithm>

#include "bsp_fp8_tc.cuh"

namespace bsp {
using namespace tc;
using namespace fp8;

namespace {

constexpr int kWarpEpi = 32 * kEpiCols * 2;        // an epilogue warp's 32 rows x 32 columns

struct Fp8Params {
  Operand A, B;
  int contraction;
  int a_bytes, b_bytes;      // of one copy
  int width;                 // columns of a tile
  uint32_t idesc;
  int act;
  const uint16_t* bias;      // [B.rows], or null
  const uint8_t* keep;       // flags [A.rows / block, B.rows] of the output, or null
  int block, keep_wide;      // eight flags at a time
  uint16_t* Y;
  int ldy, y_wide;           // 16-byte stores
  int* status;
};

// 32 rows x 32 columns of the output by one warp, a row of accumulators per lane: mask, bias, activation, rounding, then through the
// warp's own 2 KB of shared memory, so that four lanes store 64 neighbouring bytes of a row.  (By the copy engine a piece took 0.8 us
// behind its fence, two barriers of four warps and the wait for the buffer: 4 us of a 256-wide tile; this way there is
// nothing to wait for.)
__device__ __forceinline__ void finish_piece(const Fp8Params& P, uint32_t (&v)[32], uint32_t bias_smem, uint32_t buf, int row0, int col0, int lane) {
  if (P.keep != nullptr) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint2 f = output_flags(P, row0 + lane, col0 + 8 * j);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if ((((e < 4 ? f.x : f.y) >> (8 * (e & 3))) & 0xffu) == 0u) v[8 * j + e] = 0u;
    }
  }
  EpiloguePiece piece;
#pragma unroll
  for (int e = 0; e < 32; ++e) piece.v[e] = v[e];
#pragma unroll
  for (int j = 0; j < 4; ++j) piece.bias[j] = ld_shared_v4(bias_smem + 16u * j);
  __syncwarp();                                    // the piece before has been read
  piece_store(piece, P.act, buf + 64u * lane, static_cast<uint32_t>((lane >> 1) & 3));
  __syncwarp();
  const int chunk = lane & 3, n = min(8, P.B.rows - (col0 + 8 * chunk));       // columns of this lane that exist
  uint4 q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 8 * i + (lane >> 2);
    q[i] = ld_shared_v4(buf + 64u * r + (((chunk ^ (r >> 1)) & 3) << 4));
  }
  uint16_t* dst = P.Y + static_cast<size_t>(row0 + (lane >> 2)) * P.ldy + col0 + 8 * chunk;
  const int rows = P.A.rows - row0 - (lane >> 2);      // rows from this lane's first one on
  if (P.y_wide && n == 8) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (8 * i < rows) *reinterpret_cast<uint4*>(dst + static_cast<size_t>(8 * i) * P.ldy) = q[i];
  } else {
#pragma unroll 1
    for (int i = 0; i < 4 && 8 * i < rows; ++i) {
      const uint4 v = i == 0 ? q[0] : i == 1 ? q[1] : i == 2 ? q[2] : q[3];
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n) dst[static_cast<size_t>(8 * i) * P.ldy + e] = static_cast<uint16_t>(w[e >> 1] >> (16 * (e & 1)));
    }
  }
  __syncwarp();                                    // (what follows reads tensor memory, which takes the whole warp at once)
}

// Two CTAs of a cluster share a tile of 256 x w outputs, as in bsp_linear_tc2.cu: each loads its own 128 rows of A and half of the
// w rows of B, and the instructions of the leader (cta_group::2) read both.  8-bit operands are multiplied twice as fast as
// bf16 ones, so the path from L2 binds sooner: a 128-deep stage of a 128 x 128 tile of one CTA is 32 KB, 0.3 us at the 115 bytes per ns
// that an SM gets, for 0.14 us of tensor work; a CTA of a 256 x 256 pair has the same 32 KB for 0.28 us.
// The width is the launch's (choose_width): up to 240 two accumulators fit tensor memory beside the scales; a wider tile has one.
// Every CTA holds the scales of its own rows of A and of all rows of B of the tile.
// Roles per CTA: warps 0 and 11 TMA producers of A and B (completion is counted on the leader's mbarrier), warp 10 the scales, warp 1 of
// the LEADER issues the MMAs and commits to both CTAs' barriers, warps 2 to 9 epilogue of the CTA's own 128 rows: two groups of four.  (With GELU
// the epilogue binds, 4096 x 4096 x 1024 18.3 us without and 22.3 with it, by the latency of its chain: 38 % of issue slots; with three groups the same.)
// 384 threads of up to 140 registers leave room on the SM for a CTA of the quantiser (bsp_fp8_quantize.cu), which therefore starts
// while these run, and these while it runs.  No TMA multicast is used.  All mbarrier waits are bounded.
constexpr int kFp8Threads = 384;
constexpr int kEpiWarps = 8, kEpiGroups = kEpiWarps / 4;
constexpr int kPairStage = 2 * kBlockM * kBlock;           // 128 rows of A, up to 128 of B
constexpr int kPairStages = 6;
constexpr int kPairEpi = kEpiWarps * kWarpEpi;
constexpr int kPairScaleGroup = 3 * kScaleTile;            // of four stages
constexpr int kSlotGroups = 2, kScaleSlots = 2;            // groups that are handed over together; how many such hand-overs are on their way
constexpr int kPairMaxW = 256;
constexpr int kPairSmem = 1024 + kPairStages * kPairStage + kPairEpi + kScaleSlots * kSlotGroups * kPairScaleGroup + 2 * kPairMaxW * 2 + 256;
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
__device__ __forceinline__ void commit_both(uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t.reg .b16 m;\n\telect.sync _|e, 0xffffffff;\n\tmov.b16 m, 3;\n\t"
      "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], m;\n\t}" ::"r"(bar)
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
                                                      uint32_t free_bar, uint32_t sfa, uint32_t sfb) {
  asm volatile(
      "{\n\t.reg .pred p, t, e;\n\t.reg .b16 m;\n\tmov.b16 m, 3;\n\t.reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.eq.b32 t, 0, 0;\n\t"
      "add.s64 a1, %1, %8;\n\tadd.s64 a2, a1, %8;\n\tadd.s64 a3, a2, %8;\n\t"
      "add.s64 b1, %2, %9;\n\tadd.s64 b2, b1, %9;\n\tadd.s64 b3, b2, %9;\n\t"
      "@e tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%6], [%7], p;\n\t"
      "@e tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a1, b1, %3, [%6], [%7], t;\n\t"
      "@e tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a2, b2, %3, [%6], [%7], t;\n\t"
      "@e tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], a3, b3, %3, [%6], [%7], t;\n\t"
      "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%5], m;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(free_bar), "r"(sfa), "r"(sfb), "n"(STEP_A), "n"(STEP_B)
      : "memory");
}
// An arrival on a barrier of the leader.  What it reports is complete: reads of tensor memory behind a tcgen05 fence, or scales that
// this CTA has written to its own shared memory, behind the fence towards the unit that reads them there.  (Ordering everything
// else as well, .release.cluster, took 1 us.)
__device__ __forceinline__ void mbar_arrive_remote(uint32_t bar_cluster) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar_cluster) : "memory");
}

// Named barriers of the epilogue warps; the second with an AND reduction: whether all of their waits succeeded.
__device__ __forceinline__ void epilogue_meet() {
  __syncwarp();
  asm volatile("bar.sync 3, %0;" ::"n"(32 * kEpiWarps) : "memory");
}
__device__ __forceinline__ bool epilogue_agree(bool ok) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %1, 0;\n\t"
      "barrier.cta.red.and.pred q, 4, %2, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"(ok ? 1u : 0u), "n"(32 * kEpiWarps)
      : "memory");
  return r != 0u;
}

// The value is computed before anything that follows, not where it is first used.
__device__ __forceinline__ void keep_here(int& x) { asm volatile("" : "+r"(x)); }

template <bool kAMn, bool kBMn>
__global__ void __launch_bounds__(kFp8Threads, 1)
gemm_fp8_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                     const __grid_constant__ Fp8Params P) {
  constexpr int S = kPairStages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  // [S operand stages][epilogue staging buffers][scales][bias of two tiles][mbarriers, TMEM base]
  const uint32_t smem_base = smem_u32(smem);
  constexpr int kScalesOff = S * kPairStage + kPairEpi;
  uint16_t* s_bias = reinterpret_cast<uint16_t*>(smem + kScalesOff + kScaleSlots * kSlotGroups * kPairScaleGroup);
  uint64_t* bars = reinterpret_cast<uint64_t*>(reinterpret_cast<uint8_t*>(s_bias) + 2 * kPairMaxW * 2);
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(bars + 2 * S + 4 + 2 * kScaleSlots);
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
  auto scale_empty_bar = [&](int s) { return bar_base + 8u * (2 * S + 4 + kScaleSlots + s); };   // one per CTA

  if (threadIdx.x == 0) {
    *timed_out = 0u;
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_a)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_b)) : "memory");
    for (int s = 0; s < S; ++s) { mbar_init(full_bar(s), 2); mbar_init(empty_bar(s), 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(acc_full_bar(a), 1); mbar_init(acc_empty_bar(a), 2 * kEpiWarps); }
    for (int s = 0; s < kScaleSlots; ++s) { mbar_init(scale_full_bar(s), 2); mbar_init(scale_empty_bar(s), 1); }
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
  const int rows = P.A.rows, cols = P.B.rows, w = P.width;
  const int m_tiles = (rows - 1) / 256 + 1;
  const int n_tiles = (cols - 1) / w + 1;
  const int total_tiles = m_tiles * n_tiles;
  const int k_blocks = blocks_of(P.contraction);
  const int accs = pair_accumulators(w);
  const int tiles_b = (w + 127) >> 7;                  // sets of 128 rows of B with scales
  // Before this returns nothing of global memory is touched, and nothing signalled across the pair.  Each role calls it where it has computed
  // all it can: the kernel before is mostly still running, and what comes behind it costs up to 0.5 us in instructions that are not cached yet.
  auto begin_work = [&] {
    pdl_wait();
    pdl_launch_dependents();
    cluster_wait();              // the other CTA's barriers exist, and its tensor memory is allocated
  };

  if (warp == 0 || warp == 11) {
    // ---------------------------------------------------------------- TMA producers (both CTAs): warp 0 of A, warp 11 of B
    const bool for_a = warp == 0;
    const CUtensorMap* map = for_a ? &map_a : &map_b;
    const uint32_t at = for_a ? 0u : static_cast<uint32_t>(kBlockM * kBlock);
    const uint32_t arm = rank == 0 ? 2u * static_cast<uint32_t>(for_a ? P.a_bytes : P.b_bytes) : 0u;      // both CTAs' bytes
    const bool mn = for_a ? kAMn : kBMn;
    const uint32_t leader_full = map_to_cta(full_bar(0), 0);
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    auto first_row = [&](int tile) {
      return for_a ? (tile / n_tiles) * 256 + static_cast<int>(rank) * kBlockM : (tile % n_tiles) * w + static_cast<int>(rank) * (w / 2);
    };
    int row0 = first_row(pair);
    keep_here(row0);
    begin_work();
    for (int tile = pair; tile < total_tiles && ok; tile += n_pairs) {
      if (tile != pair) row0 = first_row(tile);
      for (int kb = 0; kb < k_blocks; ++kb) {
        if (!mbar_wait_warp(empty_bar(stage), phase ^ 1u, P.status)) { ok = false; break; }
        tma_load_pair(smem_base + stage * kPairStage + at, map, mn ? row0 : kb * kBlock, mn ? kb * kBlock : row0, leader_full + 8u * stage,
                      full_bar(stage), arm);
        if (++stage == S) { stage = 0; phase ^= 1u; }
      }
    }
    // the leader's commits that free the last stages arrive here while this CTA still exists
    for (int i = 0; i < S && ok; ++i) {
      ok = mbar_wait_warp(empty_bar(stage), phase ^ 1u, P.status);
      if (++stage == S) { stage = 0; phase ^= 1u; }
    }
    if (!ok && lane == 0) record_timeout(P.status, timed_out);
  } else if (warp == 10) {
    // ---------------------------------------------------------------- scales (both CTAs: its own rows of A, all rows of B)
    // A turn's loads take 0.7 us and more, so it carries the scales of eight stages; the very first one of four.
    const uint32_t leader_scale_full = map_to_cta(scale_full_bar(0), 0);
    int slot = 0;
    uint32_t phase = 0;
    bool ok = true;
    int m0 = (pair / n_tiles) * 256 + static_cast<int>(rank) * kBlockM, n0 = (pair % n_tiles) * w;
    keep_here(m0);
    keep_here(n0);
    begin_work();
    for (int tile = pair; tile < total_tiles && ok; tile += n_pairs) {
      if (tile != pair) {
        m0 = (tile / n_tiles) * 256 + static_cast<int>(rank) * kBlockM;
        n0 = (tile % n_tiles) * w;
      }
      for (int kb = 0; kb < k_blocks;) {
        const bool begin = tile == pair && kb == 0;
        const int n = min(begin ? 4 : 4 * kSlotGroups, k_blocks - kb);
        ScalesA<kAMn> x;
        ScalesB<kAMn> y, z;
        x.load(P.A, m0, kb, n, lane);
        y.load(P.B, n0, kb, n, lane);
        if (tiles_b > 1) z.load(P.B, n0 + 128, kb, n, lane);
        ok = mbar_wait_warp(scale_empty_bar(slot), phase ^ 1u, P.status);
        if (!ok) break;
        uint32_t dst = smem_base + kScalesOff + slot * kSlotGroups * kPairScaleGroup;
        if (begin) dst += (kSlotGroups - 1) * kPairScaleGroup;
#pragma unroll
        for (int g = 0; g < kSlotGroups; ++g, dst += kPairScaleGroup) {
          if (4 * g >= n) continue;
          x.store(P.A, m0, kb, g, dst, lane);
          y.store(P.B, n0, kb, g, dst + kScaleTile, lane);
          if (tiles_b > 1) z.store(P.B, n0 + 128, kb, g, dst + 2 * kScaleTile, lane);
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive_remote(leader_scale_full + 8u * slot);
        if (++slot == kScaleSlots) { slot = 0; phase ^= 1u; }
        kb += n;
      }
    }
    for (int i = 0; i < kScaleSlots && ok; ++i) {      // as for the stages
      ok = mbar_wait_warp(scale_empty_bar(slot), phase ^ 1u, P.status);
      if (++slot == kScaleSlots) { slot = 0; phase ^= 1u; }
    }
    if (!ok && lane == 0) record_timeout(P.status, timed_out);
  } else if (warp == 1 && rank == 0) {
    // ---------------------------------------------------------------- MMA issuer (leader CTA only)
    int stage = 0, slot = 0;
    uint32_t phase = 0, slot_phase = 0, scale_buf = 0, acc_phases = 0;
    int acc = 0;
    bool ok = true;
    // The scales of the four blocks from kb on, to the set of columns that the four blocks before do not read; two stages ahead of the
    // instructions that read them, which would otherwise wait for the copy.
    auto bring_scales = [&](bool first_tile, int kb) {
      const int group = ((kb >> 2) + (first_tile ? kSlotGroups - 1 : 0)) & (kSlotGroups - 1);      // (the first turn is one group)
      if (group == 0 || kb == 0) {
        if (!mbar_wait_warp(scale_full_bar(slot), slot_phase, P.status)) return false;
        tcgen05_fence_after();
      }
      const uint32_t src = smem_base + kScalesOff + (slot * kSlotGroups + group) * kPairScaleGroup;
      scale_buf ^= kPairScaleCols;
      const uint32_t dst = tmem_base + 512u - 2u * kPairScaleCols + scale_buf;
      for (int i = 0; i <= tiles_b; ++i) copy_scales_pair(dst + 4u * i, src + i * kScaleTile);
      if (group == kSlotGroups - 1 || kb + 4 >= k_blocks) {
        commit_both(scale_empty_bar(slot));
        if (++slot == kScaleSlots) { slot = 0; slot_phase ^= 1u; }
      }
      return true;
    };
    begin_work();
    for (int tile = pair; tile < total_tiles && ok; tile += n_pairs) {
      ok = bring_scales(tile == pair, 0);
      if (!ok) break;
      if (!mbar_wait_warp(acc_empty_bar(acc), ((acc_phases >> acc) & 1u) ^ 1u, P.status)) { ok = false; break; }
      tcgen05_fence_after();
      const uint32_t d_tmem = tmem_base + static_cast<uint32_t>(acc * w);
      uint32_t sfa = 0u;
      bool ready = false;
      for (int kb = 0; kb < k_blocks; ++kb) {
        if ((kb & 3) == 0) sfa = tmem_base + 512u - 2u * kPairScaleCols + scale_buf;
        if (!mbar_wait_probed(ready, full_bar(stage), phase, P.status)) { ok = false; break; }
        tcgen05_fence_after();
        const int next = stage + 1 == S ? 0 : stage + 1;
        const uint32_t next_phase = next ? phase : phase ^ 1u;
        ready = kb + 1 < k_blocks && mbar_try_wait(full_bar(next), next_phase);
        const uint32_t a_addr = smem_base + stage * kPairStage, b_addr = a_addr + kBlockM * kBlock;
        const uint32_t idesc = P.idesc | (static_cast<uint32_t>(kb & 3) << 29) | (static_cast<uint32_t>(kb & 3) << 4);
        mma_stage_scaled_pair<kAMn ? 256 : 2, kBMn ? 256 : 2>(d_tmem, kAMn ? smem_desc_mn8(a_addr) : smem_desc_sw128(a_addr),
                                                              kBMn ? smem_desc_mn8(b_addr) : smem_desc_sw128(b_addr), idesc, kb != 0 ? 1u : 0u,
                                                              empty_bar(stage), sfa, sfa + 4u);
        stage = next;
        phase = next_phase;
        if ((kb & 3) == 1 && kb + 3 < k_blocks && !bring_scales(tile == pair, kb + 3)) { ok = false; break; }
      }
      if (!ok) break;
      commit_both(acc_full_bar(acc));
      acc_phases ^= 1u << acc;
      if (accs == 2) acc ^= 1;
    }
    if (!ok && lane == 0) record_timeout(P.status, timed_out);
  } else if (warp >= 2) {
    // ---------------------------------------------------------------- epilogue of this CTA's 128 rows
    const int number = warp - 2;                                 // 0 to 7
    const int group = number >> 2;
    const int quad = warp & 3;                                   // the quarter of tensor memory that the warp may read
    const int epi_tid = number * 32 + lane;
    const uint32_t buf = smem_base + S * kPairStage + number * kWarpEpi;
    uint32_t acc_phases = 0, bias_buf = 0;
    int acc = 0;
    bool ok = true;
    // The first turn works on no tile: it brings the body's instructions to the caches (1500 cycles of the first piece) while there is
    // nothing else to do, and stores nothing.
    for (int tile = pair - n_pairs; tile < total_tiles && ok; tile += n_pairs) {
      const bool dry = tile < pair;
      const int m0 = dry ? rows : (tile / n_tiles) * 256 + static_cast<int>(rank) * kBlockM, n0 = dry ? 0 : (tile % n_tiles) * w;
      for (int c = epi_tid; c < w; c += 32 * kEpiWarps)
        s_bias[bias_buf * kPairMaxW + c] = (P.bias != nullptr && !dry && n0 + c < cols) ? ld_global(P.bias + n0 + c) : static_cast<uint16_t>(0);
      epilogue_meet();
      // all epilogue threads take the same decision, so nobody is left alone at a named barrier below
      if (!epilogue_agree(dry || mbar_wait(acc_full_bar(acc), (acc_phases >> acc) & 1u, P.status))) { ok = false; break; }
      tcgen05_fence_after();
      const uint32_t taddr = tmem_base + (static_cast<uint32_t>(quad * 32) << 16) + static_cast<uint32_t>(acc * w);
      const int pieces = dry ? kEpiGroups : (min(w, cols - n0) + kEpiCols - 1) / kEpiCols;
      // (the last piece of a tile whose width is no multiple of 32 begins early: both write the same values)
      auto first_col = [&](int pc) { return min(pc * kEpiCols, w - kEpiCols); };
      // One body for all pieces, the next one's accumulators on their way while a piece is finished.  (Unrolled, with all pieces in registers
      // before the first was finished, the accumulator was free sooner, but a piece took 1800 cycles, most of them for
      // instructions that no cache held yet.)
      uint32_t next[32];
      if (group < pieces) tmem_load_32cols(taddr + first_col(group), next);
      tmem_load_wait();
#pragma unroll 1
      for (int pc = group; pc < pieces; pc += kEpiGroups) {
        tmem_loaded<32>(next);
        uint32_t v[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = next[e];
        if (pc + kEpiGroups < pieces) tmem_load_32cols(taddr + first_col(pc + kEpiGroups), next);
        finish_piece(P, v, smem_u32(s_bias + bias_buf * kPairMaxW + first_col(pc)), buf, m0 + quad * 32, n0 + first_col(pc), lane);
        tmem_load_wait();
      }
      if (dry) {
        begin_work();
        continue;
      }
      // (the last accumulators are not waited for again: no arrival that could come when the leader has left)
      if (tile + accs * n_pairs < total_tiles) {
        tcgen05_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_remote(map_to_cta(acc_empty_bar(acc), 0));
      }
      acc_phases ^= 1u << acc;
      if (accs == 2) acc ^= 1;
      bias_buf ^= 1u;
    }
    if (!ok && lane == 0) record_timeout(P.status, timed_out);
  } else {
    begin_work();                                       // (warp 1 of the other CTA has nothing else to do)
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

template <bool kAMn, bool kBMn>
int launch_pair(const Product& p, int w, TcDevice* dev, cudaStream_t s) {
  static OncePerDevice once;
  BSP_TRY(allow_dynamic_smem(once, gemm_fp8_pair_kernel<kAMn, kBMn>, kPairSmem));
  CUtensorMap map_a, map_b;
  const int a_rows = kAMn ? kBlock : box_rows(p.A.rows, kBlockM), b_rows = kBMn ? kBlock : box_rows(p.B.rows, w / 2);
  if (!(kAMn ? make_map8(&map_a, p.A.q, p.A.rows, p.contraction, p.A.ld, kBlock) : make_map8(&map_a, p.A.q, p.contraction, p.A.rows, p.A.ld, a_rows)) ||
      !(kBMn ? make_map8(&map_b, p.B.q, p.B.rows, p.contraction, p.B.ld, kBlock) : make_map8(&map_b, p.B.q, p.contraction, p.B.rows, p.B.ld, b_rows)))
    return BSP_ERR_CUDA;
  const Fp8Params P{p.A, p.B, p.contraction, a_rows * kBlock, b_rows * kBlock, w, idesc_scaled(p.A.fmt, p.B.fmt, kAMn, kBMn, 256, w), p.act, p.bias,
                    p.keep, p.block, aligned_to(p.keep, 8) && p.B.rows % 8 == 0, p.Y, p.ldy, aligned_to(p.Y, 16) && p.ldy % 8 == 0, dev->status};
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
  BSP_CUDA_TRY(cudaLaunchKernelEx(&cfg, gemm_fp8_pair_kernel<kAMn, kBMn>, map_a, map_b, P));
  return BSP_OK;
}

// Width of the tiles by their estimated time: waves of tiles, each with its stages' time and what the stores of the tile before keep of it, or
// with GELU the epilogue's where that is longer; a tile of 256 columns, with its one accumulator, has its epilogue behind its
// stages.  Microseconds of a stage measured on layers of 480 to 4096 features: a call alone, and in one of 30 us and more, where the
// power limit takes a quarter of the clock.  Weights that lie the other way round, and column forms, are copied in whole boxes of 128 columns however
// many are used, and from anything but multiples of 64 bytes slower: fewer widths.  Measured / best width: 4096 x 4096 x 1024 18.3 / 17.9 us (with GELU 22.3 / 22.3),
// 4096 x 1024 x 4096 15.7 / 15.7, 16384 x 1024 x 4096 59.2 / 58.8, 1003 x 2128 x 928 6.4 / 6.4, 1024 x 1024 x 4096 9.4 / 9.4.
int choose_width(const Product& p, int sms, double* us) {
  struct Width { int w; double alone, among; };
  constexpr Width kKMajor[] = {{64, 0.165, 0.194}, {96, 0.166, 0.21}, {128, 0.1875, 0.256}, {160, 0.20, 0.257}, {192, 0.23, 0.293}, {240, 0.28, 0.35}, {256, 0.33, 0.42}};
  constexpr Width kMnMajor[] = {{64, 0.22, 0.26}, {128, 0.23, 0.27}, {192, 0.24, 0.30}, {256, 0.33, 0.42}};
  const Width* widths = p.B.mn ? kMnMajor : kKMajor;
  const int count = p.B.mn ? sizeof(kMnMajor) / sizeof(Width) : sizeof(kKMajor) / sizeof(Width);
  const int k_blocks = blocks_of(p.contraction);
  const bool gelu = p.act == BSP_ACT_GELU;
  int best = 0;
  long long pairs = 0;
  double least = 0.0;
  for (const bool among : {false, true}) {
    least = 0.0;
    best = 0;
    for (int i = 0; i < count; ++i) {
      const int w = widths[i].w;
      const long long tiles = static_cast<long long>((p.A.rows - 1) / 256 + 1) * ((p.B.rows - 1) / w + 1);
      const long long waves = (tiles + sms / 2 - 1) / (sms / 2);
      const double stages = k_blocks * (among ? widths[i].among : widths[i].alone), last = w * (gelu ? 0.0125 : 0.0075);
      const double wave = pair_accumulators(w) == 1 ? stages + w * (gelu ? 0.011 : 0.007) : gelu ? fmax(stages + 0.004 * w, 0.6 + 0.0152 * w) : stages + 0.004 * w;
      const double t = (waves - 1) * wave + stages + last;
      if (best == 0 || t < least) { best = w; least = t; pairs = std::min<long long>(tiles, sms / 2); }
    }
    if (least < 30.0) break;
  }
  *us = least + 2.6 + 0.012 * static_cast<double>(pairs) + (p.A.mn ? 1.0 : 0.0);      // (launch and first operands)
  return best;
}

}  // namespace

namespace fp8 {

bool tensor_core_ok(const Product& p) {
  const long long tiles = static_cast<long long>((p.A.rows - 1) / 256 + 1) * ((p.B.rows - 1) / 64 + 1);
  return aligned_to(p.A.q, 16) && p.A.ld % 16 == 0 && aligned_to(p.B.q, 16) && p.B.ld % 16 == 0 && tiles <= 0x7fffffffLL;
}

int launch_tensor_core(const Product& p, cudaStream_t s) {
  TcDevice* dev = tc_device();
  if (dev == nullptr) return BSP_ERR_CUDA;
  double pairs_us = 0.0, split_us = 0.0;
  const int w = choose_width(p, dev->sms, &pairs_us), c = choose_split(p, *dev, &split_us);
  if (c != 0 && split_us < pairs_us) return launch_split(p, c, dev, s);
  return p.A.mn ? launch_pair<true, true>(p, w, dev, s) : p.B.mn ? launch_pair<false, true>(p, w, dev, s) : launch_pair<false, false>(p, w, dev, s);
}

}  // namespace fp8
}  // namespace bsp
