// Products of 8-bit operands with fewer output tiles than SMs (see bsp_gemm_fp8.cu for the three forms and their scales, and
// bsp_gemm_split.cu for the same idea on bf16 operands): a cluster of C CTAs shares one tile of 128 x 64 outputs, CTA r multiplies the r-th
// part of the contraction, and the partial tiles are added through distributed shared memory, in rank order.
// With C = 1 the tile has a CTA of its own, which still starts and ends sooner than a pair's.  A CTA has at most 32 blocks of 128 of the
// contraction; their scales travel in turns of eight blocks and stay in tensor memory, where each turn has columns of its own.
// A CTA: warps 0 and 10 TMA producers of the two operands, warp 11 the scales, warp 1 the MMAs, warps 2 to 9 the exchange and the
// epilogue, in two groups of four.  Each CTA owns 64 / C columns of the tile; the others send it theirs as float32 straight from tensor memory
// (st.async), counted on an mbarrier.
// What bounds it is the chain of dependent steps: launch, first operands, two exchanges of a few KB.  Against the pairs of
// bsp_gemm_fp8.cu (us): see choose_split.
// All waits are bounded.  A CTA whose wait ran out stays until the rest of its cluster has left: what they were still
// going to send arrives in memory that exists.
#include "bsp_fp8_tc.cuh"

namespace bsp {
using namespace tc;
using namespace fp8;

namespace {

constexpr int kSplit8Threads = 384;
constexpr int kTileN = 64;
constexpr int kMostStages = 8;
constexpr int kTurn = 8, kMostTurns = 4;             // blocks whose scales travel together; a CTA has at most 32
constexpr uint32_t kTmemCols = 128;                  // 64 of the accumulator, 8 for the scales of each four blocks
static_assert(kTileN + 8 * kTurn / 4 * kMostTurns <= static_cast<int>(kTmemCols), "tensor memory");

struct Split8Params {
  Operand A, B;
  int n_tiles, k_blocks, stages;
  int a_bytes, b_bytes;      // of one copy
  int recv_off, tail_off;    // offsets of the receive buffers and of scales, mbarriers and bias
  uint32_t idesc;
  int act;
  const uint16_t* bias;      // [B.rows], or null
  const uint8_t* keep;       // flags [A.rows / block, B.rows] of the output, or null
  int block, keep_wide;
  uint16_t* Y;
  int ldy, y_wide;
  int* status;
};

__device__ __forceinline__ void copy_scales(uint32_t taddr, uint32_t smem_addr) {
  asm volatile(
      "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t}" ::"r"(taddr), "l"(scale_desc(smem_addr))
      : "memory");
}
// A block of 128 of the contraction: four steps under the same scales, then the commit that frees the stage.
template <int STEP_A, int STEP_B>
__device__ __forceinline__ void mma_block_scaled(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate,
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

// Bytes of a stage: 128 rows of A, and 64 rows of B or, where B's rows are the contraction, whole boxes of 128 columns.
__host__ __device__ constexpr int stage_b(bool b_mn) { return (b_mn ? 128 : kTileN) * kBlock; }
__host__ __device__ constexpr int stage_bytes(bool b_mn) { return kBlockM * kBlock + stage_b(b_mn); }
constexpr int kScalesOf = 2 * kScaleTile;            // of four blocks: A's, B's
constexpr int kScalesAll = kScalesOf * kTurn / 4 * kMostTurns;
constexpr int kBars = 256, kTail = kScalesAll + kBars + 4 * kTileN;        // scales, mbarriers and a flag, bias
static_assert((2 * kMostStages + 2 + kMostTurns) * 8 + 8 <= kBars, "mbarriers");

template <bool kAMn, bool kBMn, int C>
__global__ void __launch_bounds__(kSplit8Threads, 1)
gemm_fp8_split_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                      const __grid_constant__ Split8Params P) {
  constexpr int kStage = stage_bytes(kBMn);
  constexpr int W = kTileN / C;                        // columns a CTA owns: [rank * W, +W) of the tile
  constexpr int U = W >= 16 ? W / 2 : 8;               // of these, the columns of one epilogue group (W = 8: group 0 only)
  constexpr uint32_t kSlot = kBlockM * W * 4;          // receive buffer of one source CTA
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  // [8] full, [8] empty, accumulator, received, [4] scales
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + P.tail_off + kScalesAll);
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(bars + 2 * kMostStages + 2 + kMostTurns);
  volatile uint32_t* timed_out = tmem_holder + 1;
  float* s_bias = reinterpret_cast<float*>(smem + P.tail_off + kScalesAll + kBars);      // [W]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t smem_base = smem_u32(smem), bar_base = smem_u32(bars), scales = smem_base + static_cast<uint32_t>(P.tail_off);
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (kMostStages + s); };
  const uint32_t acc_bar = bar_base + 16u * kMostStages, recv_bar = acc_bar + 8u;
  auto scale_bar = [&](int t) { return acc_bar + 16u + 8u * t; };
  const uint32_t rank = cluster_rank();
  const int tile = static_cast<int>(blockIdx.x) / C;
  const int m0 = (tile / P.n_tiles) * kBlockM, n0 = (tile % P.n_tiles) * kTileN;
  const int rows = P.A.rows, cols = P.B.rows;
  const int quads = (min(kBlockM, rows - m0) + 31) >> 5;     // quarters of the tile with rows that exist
  const int kb0 = P.k_blocks * static_cast<int>(rank) / C, n_blocks = P.k_blocks * (static_cast<int>(rank) + 1) / C - kb0;     // 1 to 32
  const int S = P.stages, ahead = min(S, n_blocks);    // stages that are filled without waiting for one to be free

  // The producers fill the first stages before the CTA meets; the signal to dependents is left to the warp that allocates tensor memory,
  // behind the allocation (see bsp_gemm_split.cu).
  ScalesA<kAMn> scales_a;
  ScalesB<kAMn> scales_b;
  auto load_a = [&](int i, int stage) {
    const int k = (kb0 + i) * kBlock;
    tma_stage_load(smem_base + stage * kStage, &map_a, kAMn ? m0 : k, kAMn ? k : m0, full_bar(stage), P.a_bytes);
  };
  auto load_b = [&](int i, int stage) {
    const int k = (kb0 + i) * kBlock;
    tma_stage_load(smem_base + stage * kStage + kBlockM * kBlock, &map_b, kBMn ? n0 : k, kBMn ? k : n0, full_bar(stage), P.b_bytes);
  };
  if (warp == 0) {
    // a lane for each barrier: all in one go
    if (lane < 2 * kMostStages + 2 + kMostTurns) mbar_init(bar_base + 8u * lane, lane < kMostStages ? 2 : 1);
    if (lane == 0) *timed_out = 0u;
    if (C > 1 && lane == 2 * kMostStages + 1)
      mbar_arrive_expect_tx(recv_bar, static_cast<uint32_t>((C - 1) * quads * 32 * W * 4));   // what the others will send
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    asm volatile("bar.arrive 6, 64;" ::: "memory");    // the mbarriers exist
    pdl_wait();
    for (int i = 0; i < ahead; ++i) load_a(i, i);
  } else if (warp == 10) {
    if (lane == 0) {
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_b)) : "memory");
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_a)) : "memory");
    }
    __syncwarp();
    asm volatile("bar.sync 6, 64;" ::: "memory");
    pdl_wait();
    for (int i = 0; i < ahead; ++i) load_b(i, i);
  } else if (warp == 11) {
    pdl_wait();
    scales_a.load(P.A, m0, kb0, min(kTurn, n_blocks), lane);
    scales_b.load(P.B, n0, kb0, min(kTurn, n_blocks), lane);
  } else if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_holder)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    pdl_wait();
    pdl_launch_dependents();
  }
  tcgen05_fence_before();
  __syncthreads();
  tcgen05_fence_after();
  const uint32_t tmem_base = *tmem_holder;
  cluster_arrive_relaxed();                            // this CTA runs and its mbarriers exist (fenced above)
  if (warp >= 2 && warp < 10) pdl_wait();

  if (warp == 0 || warp == 10) {
    // ---------------------------------------------------------------- TMA producers of A and B, further stages
    int stage = ahead == S ? 0 : ahead;
    uint32_t phase = 0;                                // of the first time a stage is freed
    bool ok = true;
    for (int i = ahead; i < n_blocks; ++i) {
      if (!mbar_wait_warp(empty_bar(stage), phase, P.status)) { ok = false; break; }
      if (warp == 0) load_a(i, stage);
      else load_b(i, stage);
      if (++stage == S) { stage = 0; phase ^= 1u; }
    }
    if (!ok && lane == 0) record_timeout(P.status, timed_out);
  } else if (warp == 11) {
    // ---------------------------------------------------------------- scales
    for (int first = 0; first < n_blocks; first += kTurn) {
      const int n = min(kTurn, n_blocks - first);
      if (first > 0) {
        scales_a.load(P.A, m0, kb0 + first, n, lane);
        scales_b.load(P.B, n0, kb0 + first, n, lane);
      }
#pragma unroll
      for (int g = 0; g < kTurn / 4; ++g) {
        if (4 * g >= n) continue;
        const uint32_t dst = scales + (first / 4 + g) * kScalesOf;
        scales_a.store(P.A, m0, kb0 + first, g, dst, lane);
        scales_b.store(P.B, n0, kb0 + first, g, dst + kScaleTile, lane);
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(scale_bar(first / kTurn));
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMAs
    bool ok = true, ready = false;
    int stage = 0;
    uint32_t phase = 0;
    for (int i = 0; i < n_blocks; ++i) {
      if (i % kTurn == 0) {
        if (!mbar_wait_warp(scale_bar(i / kTurn), 0u, P.status)) { ok = false; break; }
        tcgen05_fence_after();
        for (int g = i / 4; g < i / 4 + kTurn / 4 && 4 * g < n_blocks; ++g) {
          copy_scales(tmem_base + kTileN + 8u * g, scales + g * kScalesOf);
          copy_scales(tmem_base + kTileN + 8u * g + 4u, scales + g * kScalesOf + kScaleTile);
        }
      }
      if (!mbar_wait_probed(ready, full_bar(stage), phase, P.status)) { ok = false; break; }
      tcgen05_fence_after();
      const int next = stage + 1 == S ? 0 : stage + 1;
      const uint32_t next_phase = next ? phase : phase ^ 1u;
      ready = i + 1 < n_blocks && mbar_try_wait(full_bar(next), next_phase);
      const uint32_t a_addr = smem_base + stage * kStage, b_addr = a_addr + kBlockM * kBlock, sf = tmem_base + kTileN + 8u * (i >> 2);
      const uint32_t idesc = P.idesc | (static_cast<uint32_t>(i & 3) << 29) | (static_cast<uint32_t>(i & 3) << 4);
      mma_block_scaled<kAMn ? 256 : 2, kBMn ? 256 : 2>(tmem_base, kAMn ? smem_desc_mn8(a_addr) : smem_desc_sw128(a_addr),
                                                       kBMn ? smem_desc_mn8(b_addr) : smem_desc_sw128(b_addr), idesc, i != 0 ? 1u : 0u,
                                                       empty_bar(stage), sf, sf + 4u);
      stage = next;
      phase = next_phase;
    }
    if (ok) tcgen05_commit_elect(acc_bar);
    else if (lane == 0) record_timeout(P.status, timed_out);
  }
  __syncwarp();
  const bool epilogue = warp >= 2 && warp < 10;
  const int group = (warp - 2) >> 2, quad = warp & 3;
  const int row = quad * 32 + lane, m = m0 + row;
  const bool mine = epilogue && group * U < W;         // this warp's group has columns
  const bool live = quad < quads;                      // this warp's rows exist
  const int c0 = group * U;                            // its first column of the CTA's
  const int n_own = n0 + static_cast<int>(rank) * W + c0;
  bool ok = true;
  uint2 flags[U / 8];
  if (epilogue) {
    const int c = static_cast<int>(threadIdx.x) - 64, n = n0 + static_cast<int>(rank) * W + c;
    if (c < W) s_bias[c] = P.bias != nullptr && n < cols ? bf16_bits_to_float(ld_global(P.bias + n)) : 0.0f;
#pragma unroll
    for (int u = 0; u < U / 8; ++u) flags[u] = P.keep != nullptr && mine ? output_flags(P, m, n_own + 8 * u) : make_uint2(0x01010101u, 0x01010101u);
    ok = __all_sync(0xffffffffu, mbar_wait(acc_bar, 0u, P.status));
    if (!ok && lane == 0) record_timeout(P.status, timed_out);
    tcgen05_fence_after();
  }
  __syncwarp();
  cluster_wait();                                      // the others run

  const uint32_t taddr = tmem_base + (static_cast<uint32_t>(quad * 32) << 16);
  // receive buffer of a CTA: [source, own rank left out][4-column group][row][4 floats]
  const uint32_t recv_at = smem_base + static_cast<uint32_t>(P.recv_off) + static_cast<uint32_t>(c0 >> 2) * (kBlockM * 16u) + static_cast<uint32_t>(row) * 16u;
  if (C > 1 && mine && live && ok) {
    // ---------------------------------------------------------------- partial columns to their owners
    uint32_t v[C > 1 ? C - 1 : 1][U];
#pragma unroll
    for (int o = 1; o < C; ++o) tmem_load_cols<U>(taddr + ((rank + o) % C) * W + c0, v[o - 1]);
    tmem_load_wait();
#pragma unroll
    for (int o = 1; o < C; ++o) {
      tmem_loaded<U>(v[o - 1]);
      const uint32_t q = (rank + o) % C, slot = rank < q ? rank : rank - 1;
      const uint32_t dst = map_to_cta(recv_at + slot * kSlot, q), bar = map_to_cta(recv_bar, q);
#pragma unroll
      for (int j = 0; j < U / 4; ++j)
        st_async_v4(dst + j * (kBlockM * 16u), bar, v[o - 1][4 * j], v[o - 1][4 * j + 1], v[o - 1][4 * j + 2], v[o - 1][4 * j + 3]);
    }
  }
  __syncwarp();

  // ---------------------------------------------------------------- this CTA's columns
  if (epilogue) {
    epilogue_sync_all();                               // s_bias is complete
    if (C > 1 && !mbar_wait_warp(recv_bar, 0u, P.status)) {     // (one answer for the warp, which lane 0 records)
      if (lane == 0) record_timeout(P.status, timed_out);
      ok = false;
    }
    ok = __all_sync(0xffffffffu, ok) && live;
  }
  if (mine && ok) {
    uint32_t own[U];
    tmem_load_cols<U>(taddr + rank * W + c0, own);
    tmem_load_wait();
    tmem_loaded<U>(own);
    float f[U];
#pragma unroll
    for (int i = 0; i < U; ++i) f[i] = __uint_as_float(own[i]);
#pragma unroll
    for (int src = 0; src < C - 1; ++src) {            // own part first, then the others in rank order
      uint4 a[U / 4];
#pragma unroll
      for (int j = 0; j < U / 4; ++j) a[j] = ld_shared_v4(recv_at + src * kSlot + j * (kBlockM * 16u));
#pragma unroll
      for (int j = 0; j < U / 4; ++j) {
        f[4 * j] += __uint_as_float(a[j].x);
        f[4 * j + 1] += __uint_as_float(a[j].y);
        f[4 * j + 2] += __uint_as_float(a[j].z);
        f[4 * j + 3] += __uint_as_float(a[j].w);
      }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) f[i] += s_bias[c0 + i];
    if (P.act == BSP_ACT_GELU) {
#pragma unroll
      for (int i = 0; i < U; i += 2) gelu_erf_pair(f[i], f[i + 1]);
    }
#pragma unroll
    for (int i = 0; i < U; ++i)
      if ((((i & 4 ? flags[i >> 3].y : flags[i >> 3].x) >> (8 * (i & 3))) & 0xffu) == 0u) f[i] = 0.0f;
    uint32_t o[U / 2];
#pragma unroll
    for (int i = 0; i < U / 2; ++i) o[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
    if (m < rows) {
      uint16_t* out = P.Y + static_cast<size_t>(m) * P.ldy + n_own;
#pragma unroll
      for (int u = 0; u < U / 8; ++u) {
        if (P.y_wide && n_own + 8 * u + 8 <= cols) {
          *reinterpret_cast<uint4*>(out + 8 * u) = make_uint4(o[4 * u], o[4 * u + 1], o[4 * u + 2], o[4 * u + 3]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (n_own + 8 * u + e < cols) out[8 * u + e] = static_cast<uint16_t>(o[4 * u + (e >> 1)] >> (16 * (e & 1)));
        }
      }
    }
  }

  tcgen05_fence_before();
  __syncthreads();
  quiet_period(timed_out);
  if (*timed_out != 0u) {                              // (the same for every thread) until every other CTA has left, or waits here too
    cluster_arrive();
    cluster_wait();
  }
  if (warp == 1) {
    tcgen05_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
  }
}

template <bool kAMn, bool kBMn, int C>
int launch_split8(const Product& p, TcDevice* dev, cudaStream_t s) {
  static OncePerDevice once;
  auto kernel = gemm_fp8_split_kernel<kAMn, kBMn, C>;
  BSP_TRY(allow_dynamic_smem(once, kernel, kSmemLimit));
  CUtensorMap map_a, map_b;
  const int a_rows = kAMn ? kBlock : box_rows(p.A.rows, kBlockM), b_rows = kBMn ? kBlock : box_rows(p.B.rows, kTileN);
  if (!(kAMn ? make_map8(&map_a, p.A.q, p.A.rows, p.contraction, p.A.ld, kBlock) : make_map8(&map_a, p.A.q, p.contraction, p.A.rows, p.A.ld, a_rows)) ||
      !(kBMn ? make_map8(&map_b, p.B.q, p.B.rows, p.contraction, p.B.ld, kBlock) : make_map8(&map_b, p.B.q, p.contraction, p.B.rows, p.B.ld, b_rows)))
    return BSP_ERR_CUDA;
  constexpr int kReceive = (C - 1) * kBlockM * (kTileN / C) * 4;
  constexpr int kFit = (kSmemLimit - 1024 - kTail - kReceive) / stage_bytes(kBMn) < kMostStages ? (kSmemLimit - 1024 - kTail - kReceive) / stage_bytes(kBMn)
                                                                                                : kMostStages;
  const int k_blocks = blocks_of(p.contraction), n_tiles = (p.B.rows - 1) / kTileN + 1;
  const int each = (k_blocks - 1) / C + 1, stages = each < kFit ? each : kFit;
  const int recv_off = stages * stage_bytes(kBMn);
  int tail_off = recv_off + kReceive;
  if (tail_off < kSmemLimit / 2 + 1024) tail_off = kSmemLimit / 2 + 1024;                // one CTA per SM
  const Split8Params P{p.A, p.B, n_tiles, k_blocks, stages, a_rows * kBlock, b_rows * kBlock, recv_off, tail_off, idesc_scaled(p.A.fmt, p.B.fmt, kAMn, kBMn, kBlockM, kTileN), p.act, p.bias,
                       p.keep, p.block, aligned_to(p.keep, 8) && p.B.rows % 8 == 0, p.Y, p.ldy, aligned_to(p.Y, 16) && p.ldy % 8 == 0, dev->status};
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(((p.A.rows - 1) / kBlockM + 1) * n_tiles * C);
  cfg.blockDim = dim3(kSplit8Threads);
  cfg.dynamicSmemBytes = tail_off + kTail + 1024;      // (1024: alignment)
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  BSP_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, map_a, map_b, P));
  return BSP_OK;
}
template <bool kAMn, bool kBMn>
int launch_split8_c(const Product& p, int c, TcDevice* dev, cudaStream_t s) {
  return c == 1 ? launch_split8<kAMn, kBMn, 1>(p, dev, s) : c == 2 ? launch_split8<kAMn, kBMn, 2>(p, dev, s) : c == 4 ? launch_split8<kAMn, kBMn, 4>(p, dev, s) : launch_split8<kAMn, kBMn, 8>(p, dev, s);
}

}  // namespace

namespace fp8 {

// CTAs to a tile whose launch takes the least time, and that time (us); 0: none.  Only grids that run at once are considered.  A part per kernel,
// one per quarter of a tile that has rows, one per block of 128 of a CTA's part and one per CTA, fitted to layers of 256 to 4096
// features and 17 to 2048 tokens, each a launch among others of its kind with operands in L2.  Measured, pairs / split C ways: 1024 x 1024 with 128 tokens 4.65 /
// 4.96, 3.98, 3.76 us (C = 1, 2, 4), 1024 outputs x 4096 inputs 8.3 / 9.5, 6.6, 5.2, 4096 x 4096 9.3 / 9.7, 7.1; 4096 x 1024, 256 tokens 5.4 / 5.4; a
// weight gradient of 1024 x 1024 from 1003 tokens 6.8 / 5.6.
int choose_split(const Product& p, const TcDevice& dev, double* us) {
  static const double fixed[4] = {3.0, 2.43, 2.45, 2.48}, per_quarter[4] = {0.1, 0.17, 0.21, 0.22}, per_block[4] = {0.192, 0.218, 0.235, 0.235};
  const int k_blocks = blocks_of(p.contraction), quarters = p.A.rows >= kBlockM ? 4 : (p.A.rows + 31) / 32;
  const long long tiles = static_cast<long long>((p.A.rows - 1) / kBlockM + 1) * ((p.B.rows - 1) / kTileN + 1);
  int best = 0;
  for (int i = 0; i < 4; ++i) {
    const int c = 1 << i, each = (k_blocks - 1) / c + 1;
    if (c > k_blocks || each > kTurn * kMostTurns || tiles * c > (i == 0 ? dev.sms : dev.split_ctas[i - 1])) continue;
    const double t = fixed[i] + quarters * per_quarter[i] + each * per_block[i] + 0.003 * static_cast<double>(tiles * c);
    if (best == 0 || t < *us) { best = c; *us = t; }
  }
  return best;
}

int launch_split(const Product& p, int c, TcDevice* dev, cudaStream_t s) {
  return p.A.mn ? launch_split8_c<true, true>(p, c, dev, s) : p.B.mn ? launch_split8_c<false, true>(p, c, dev, s) : launch_split8_c<false, false>(p, c, dev, s);
}

}  // namespace fp8
}  // namespace bsp
