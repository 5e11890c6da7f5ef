// bsp_linear_fp8 for few tokens, in one launch: the activations are brought to 8 bits on their way into the product.
//
// With a few tokens a layer is a pass over its weight (4 MB for 1024 x 4096: 0.65 us of HBM), and what counts is how few dependent
// steps there are from launch to result.  A CTA takes 16 outputs; its warps share the contraction, a block of 128 at a time.  A
// lane's weights are 16-byte pieces straight from global memory in the order in which mma.sync (m16n8k32, e4m3) takes them: which of
// the contraction's indices a lane holds is free as long as both operands agree, so lane 4 g + t holds k = 64 h + 16 t ... + 15 (h = 0, 1) of rows g and g
// + 8 of W, and of token g of X, and nothing passes through shared memory.  The same lane quantises its 32 values of the token (the block's largest
// magnitude is a reduction over four lanes).  Each block's product is multiplied by its two scales into float32 sums; the warps'
// sums meet in shared memory at the end, in a fixed order.
// The legacy tensor instruction is enough here: 16 x 8 outputs a warp leave it idle most of the time, and tcgen05's 128-row tiles would need the
// operands in shared memory first.
// Times, the weight in L2: 1 token, 1024 -> 4096 with GELU 2.6 us; 13 tokens, 4096 -> 1024 4.2 us.  What bounds it is the chain of dependent steps: launch
// and first loads, one block's arithmetic, the meeting of the sums.  Where it ends: few_is_faster (bsp_linear_fp8.cu).
#include "bsp_fp8_gemm.cuh"
#include "bsp_tc.cuh"

namespace bsp {
using namespace fp8;

namespace {

constexpr int kFewRows = 16;                 // outputs per CTA
constexpr int kFewMaxWarps = 16;
// Clusters of 2 or 4 CTAs share the contraction of 16 outputs while they are at most this many CTAs and each has this many blocks of 128.
constexpr int kFewCtas = 296, kFewLeastBlocks = 8;

struct FewArgs {
  const uint8_t* W;
  int ldw;
  const uint8_t* S;
  int lds, n_out, k_in;
  const void* X;             // bf16, or 8 bits with the scales XS
  int tokens, ldx, wide;     // 16-byte loads of bf16 X
  const uint8_t* XS;
  int ldxs;
  const uint16_t* bias;
  int act;
  uint16_t* Y;
  int ldy;
};

// e4m3 weights times activations of either format.
template <int FMT>
__device__ __forceinline__ void mma_fp8(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if (FMT == BSP_FP8_E4M3)
    asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e5m2.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Sixteen 8-bit values from column k on, zeros where the row has ended.
__device__ __forceinline__ uint4 byte_piece(const uint8_t* row, int k, int k_in, bool exists) {
  if (!exists || k >= k_in) return make_uint4(0u, 0u, 0u, 0u);
  if (k + 16 <= k_in) return ld_global(reinterpret_cast<const uint4*>(row + k));
  uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (k + i < k_in) w[i >> 2] |= static_cast<uint32_t>(ld_global(row + k + i)) << (8 * (i & 3));
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// Eight activations from column k on.
__device__ __forceinline__ uint4 token_piece(const uint16_t* row, int k, int k_in, bool exists, int wide) {
  if (!exists || k >= k_in) return make_uint4(0u, 0u, 0u, 0u);
  if (wide && k + 8 <= k_in) return ld_global(reinterpret_cast<const uint4*>(row + k));
  uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (k + i < k_in) w[i >> 1] |= static_cast<uint32_t>(ld_global(row + k + i)) << (16 * (i & 1));
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// GROUPS: groups of eight tokens.  kReady: the activations are in 8 bits (of format FMT) already.
template <int GROUPS, bool kReady, int FMT>
__global__ void __launch_bounds__(32 * kFewMaxWarps)
linear_few_kernel(FewArgs A) {
  extern __shared__ float s_part[];          // [warp][token][16 outputs]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const int g = lane >> 2, t = lane & 3;
  const int n0 = static_cast<int>(blockIdx.x / tc::cluster_size()) * kFewRows;
  const int blocks = blocks_of(A.k_in);
  float acc[GROUPS][4] = {};
  pdl_wait();
  pdl_launch_dependents();
  // Everything a block needs is asked for before any of it is used.
  struct Block {
    uint4 w[2][2];                           // [half of the block][row g, row g + 8]
    uint4 x[GROUPS][2][kReady ? 1 : 2];
    uint32_t scale, scale_x[kReady ? GROUPS : 1];
  };
  auto load = [&](int kb) {
    Block q;
    const int k = kb * kBlock + 16 * t;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int n = n0 + g + 8 * u;
        q.w[h][u] = byte_piece(A.W + static_cast<size_t>(n) * A.ldw, k + 64 * h, A.k_in, n < A.n_out);
      }
    q.scale = ld_global(A.S + static_cast<size_t>(n0 / kBlock) * A.lds + kb);
#pragma unroll
    for (int j = 0; j < GROUPS; ++j) {
      const int token = 8 * j + g;
      const bool exists = token < A.tokens;
      if constexpr (kReady) {
        const uint8_t* row = static_cast<const uint8_t*>(A.X) + static_cast<size_t>(token) * A.ldx;
#pragma unroll
        for (int h = 0; h < 2; ++h) q.x[j][h][0] = byte_piece(row, k + 64 * h, A.k_in, exists);
        q.scale_x[j] = exists ? ld_global(A.XS + static_cast<size_t>(token) * A.ldxs + kb) : 127u;
      } else {
        const uint16_t* row = static_cast<const uint16_t*>(A.X) + static_cast<size_t>(token) * A.ldx;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int u = 0; u < 2; ++u) q.x[j][h][u] = token_piece(row, k + 64 * h + 8 * u, A.k_in, exists, A.wide);
      }
    }
    return q;
  };
  auto multiply = [&](const Block& q) {
#pragma unroll
    for (int j = 0; j < GROUPS; ++j) {
      float c[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      uint32_t scale_x;                      // as a byte
      uint4 v[2];                            // the token's values in 8 bits
      if constexpr (kReady) {
        scale_x = q.scale_x[j];
        v[0] = q.x[j][0][0];
        v[1] = q.x[j][1][0];
      } else {
        const uint4 (&x)[2][2] = q.x[j];
        uint32_t m = 0u;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int u = 0; u < 2; ++u) m = abs_max2(m, abs_max2(abs_max2(x[h][u].x, x[h][u].y), abs_max2(x[h][u].z, x[h][u].w)));
        m = abs_max2(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = abs_max2(m, __shfl_xor_sync(0xffffffffu, m, 2));
        float inv;
        scale_x = block_scale<FMT>(abs_max_of(m), inv);
#pragma unroll
        for (int h = 0; h < 2; ++h)
          v[h] = make_uint4(four_to_fp8<FMT>(x[h][0].x, x[h][0].y, inv, inv, inv, inv), four_to_fp8<FMT>(x[h][0].z, x[h][0].w, inv, inv, inv, inv),
                            four_to_fp8<FMT>(x[h][1].x, x[h][1].y, inv, inv, inv, inv), four_to_fp8<FMT>(x[h][1].z, x[h][1].w, inv, inv, inv, inv));
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        mma_fp8<FMT>(c, q.w[h][0].x, q.w[h][1].x, q.w[h][0].y, q.w[h][1].y, v[h].x, v[h].y);
        mma_fp8<FMT>(c, q.w[h][0].z, q.w[h][1].z, q.w[h][0].w, q.w[h][1].w, v[h].z, v[h].w);
      }
      // this lane's outputs are of tokens 2 t and 2 t + 1 of the group
      // (The product of two scales can lie outside float32's range where what it multiplies brings it back, or is zero: two factors of half
      // its exponent each.)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint32_t both = q.scale + __shfl_sync(0xffffffffu, scale_x, 8 * t + 4 * u), half = both >> 1;
        const float s0 = scale_value(half), s1 = scale_value(both - half);
        acc[j][u] = __fmaf_rn(c[u] * s0, s1, acc[j][u]);
        acc[j][2 + u] = __fmaf_rn(c[2 + u] * s0, s1, acc[j][2 + u]);
      }
    }
  };
  // the contraction's blocks are dealt to the warps of all CTAs of the cluster
  const int ranks = static_cast<int>(tc::cluster_size()), rank = static_cast<int>(tc::cluster_rank()), all = warps * ranks;
  for (int kb = warp * ranks + rank; kb < blocks; kb += all) {
    const Block p = load(kb);
    __syncwarp();                            // (the assembler would move loads down to save registers)
    multiply(p);
  }
#pragma unroll
  for (int j = 0; j < GROUPS; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) s_part[(warp * 8 * GROUPS + 8 * j + 2 * t + (e & 1)) * kFewRows + g + 8 * (e >> 1)] = acc[j][e];
  __syncthreads();
  constexpr int kOutputs = 8 * GROUPS * kFewRows;
  if (ranks > 1) {
    // each CTA adds up its warps, then takes its share of the outputs and adds up the CTAs
    for (int e = threadIdx.x; e < kOutputs; e += blockDim.x) {
      float y = 0.0f;
      for (int w = 0; w < warps; ++w) y += s_part[w * kOutputs + e];
      s_part[e] = y;                         // (only this thread reads or writes column e)
    }
    tc::cluster_sync();
  }
  for (int e = threadIdx.x + rank * static_cast<int>(blockDim.x); e < A.tokens * kFewRows; e += ranks * static_cast<int>(blockDim.x)) {
    const int n = n0 + (e & (kFewRows - 1)), token = e / kFewRows;
    if (n >= A.n_out) continue;
    float y = 0.0f;
    if (ranks > 1) {
      for (int r = 0; r < ranks; ++r) {
        float part;
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(part) : "r"(tc::map_to_cta(tc::smem_u32(s_part + e), r)) : "memory");
        y += part;
      }
    } else {
      for (int w = 0; w < warps; ++w) y += s_part[w * kOutputs + e];
    }
    if (A.bias != nullptr) y += bf16_bits_to_float(ld_global(A.bias + n));
    if (A.act == BSP_ACT_GELU) {
      float unused = 0.0f;
      tc::gelu_erf_pair(y, unused);
    }
    A.Y[static_cast<size_t>(token) * A.ldy + n] = __bfloat16_as_ushort(__float2bfloat16_rn(y));
  }
  if (ranks > 1) {                           // no CTA leaves while another may read its sums
    tc::cluster_arrive_relaxed();
    tc::cluster_wait();
  }
}

}  // namespace

namespace fp8 {

namespace {

template <bool kReady, int FMT>
int launch_few_of(FewArgs A, cudaStream_t s) {
  const int n_out = A.n_out, k_in = A.k_in, tokens = A.tokens;
  const int blocks = blocks_of(k_in), tiles = (n_out - 1) / kFewRows + 1;
  int ranks = 1;
  while (ranks < 4 && tiles * ranks * 2 <= kFewCtas && blocks / (ranks * 2) >= kFewLeastBlocks) ranks *= 2;
  const int each = (blocks - 1) / ranks + 1, warps = each < kFewMaxWarps ? each : kFewMaxWarps;
  const int groups = tokens <= 8 ? 1 : tokens <= 16 ? 2 : 4;
  constexpr int kMostGroups = (kReady ? kFewReady : kFewTokens) / 8;
  auto kernel = groups == 1   ? linear_few_kernel<1, kReady, FMT>
                : groups == 2 ? linear_few_kernel<2, kReady, FMT>
                              : linear_few_kernel<kMostGroups, kReady, FMT>;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(tiles) * ranks);
  cfg.blockDim = dim3(32 * warps);
  cfg.dynamicSmemBytes = sizeof(float) * warps * 8 * groups * kFewRows;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ranks;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = ranks > 1 ? 2 : 1;
  BSP_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, A));
  return BSP_OK;
}

}  // namespace

bool few_tokens_ok(const void* Wq, int ldw, int tokens) { return tokens <= kFewTokens && aligned_to(Wq, 16) && ldw % 16 == 0; }

int launch_few(const void* Wq, int ldw, const uint8_t* WS, int ldws, int n_out, int k_in, const void* X, int tokens, int ldx, const void* bias, int act,
               void* Y, int ldy, cudaStream_t s) {
  return launch_few_of<false, BSP_FP8_E4M3>(FewArgs{static_cast<const uint8_t*>(Wq), ldw, WS, ldws, n_out, k_in, X, tokens, ldx,
                                                    aligned_to(X, 16) && ldx % 8 == 0, nullptr, 0, static_cast<const uint16_t*>(bias), act,
                                                    static_cast<uint16_t*>(Y), ldy}, s);
}
int launch_few_ready(const Product& p, cudaStream_t s) {
  const FewArgs A{p.B.q, p.B.ld, p.B.s, static_cast<int>(p.B.s_row), p.B.rows, p.contraction, p.A.q, p.A.rows, p.A.ld, 1, p.A.s, static_cast<int>(p.A.s_row),
                  p.bias, p.act, p.Y, p.ldy};
  return p.A.fmt == BSP_FP8_E4M3 ? launch_few_of<true, BSP_FP8_E4M3>(A, s) : launch_few_of<true, BSP_FP8_E5M2>(A, s);
}

}  // namespace fp8
}  // namespace bsp
