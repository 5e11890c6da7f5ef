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
// operands in shared memory first.  Times: see few_tokens_ok.
#include "bsp_fp8_gemm.cuh"
#include "bsp_tc.cuh"

namespace bsp {
using namespace fp8;

namespace {

constexpr int kFewRows = 16;                 // outputs per CTA
constexpr int kFewMaxWarps = 16;

struct FewArgs {
  const uint8_t* W;
  int ldw;
  const uint8_t* S;
  int lds, n_out, k_in;
  const uint16_t* X;
  int tokens, ldx, wide;     // 16-byte loads of X
  const uint16_t* bias;
  int act;
  uint16_t* Y;
  int ldy;
};

__device__ __forceinline__ void mma_e4m3(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Sixteen 8-bit weights from column k on, zeros where the row has ended.
__device__ __forceinline__ uint4 weight_piece(const uint8_t* row, int k, int k_in, bool exists) {
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

// GROUPS: groups of eight tokens.
template <int GROUPS>
__global__ void __launch_bounds__(32 * kFewMaxWarps)
linear_few_kernel(FewArgs A) {
  extern __shared__ float s_part[];          // [warp][token][16 outputs]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const int g = lane >> 2, t = lane & 3;
  const int n0 = blockIdx.x * kFewRows;
  const int blocks = blocks_of(A.k_in);
  float acc[GROUPS][4] = {};
  pdl_wait();
  pdl_launch_dependents();
  for (int kb = warp; kb < blocks; kb += warps) {
    const int k = kb * kBlock + 16 * t;
    uint4 w[2][2];                           // [half of the block][row g, row g + 8]
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int n = n0 + g + 8 * u;
        w[h][u] = weight_piece(A.W + static_cast<size_t>(n) * A.ldw, k + 64 * h, A.k_in, n < A.n_out);
      }
    const float scale_w = scale_value(ld_global(A.S + static_cast<size_t>(n0 / kBlock) * A.lds + kb));
#pragma unroll
    for (int j = 0; j < GROUPS; ++j) {
      const int token = 8 * j + g;
      const uint16_t* row = A.X + static_cast<size_t>(token) * A.ldx;
      uint4 x[2][2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int u = 0; u < 2; ++u) x[h][u] = token_piece(row, k + 64 * h + 8 * u, A.k_in, token < A.tokens, A.wide);
      uint32_t m = 0u;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int u = 0; u < 2; ++u) m = abs_max2(m, abs_max2(abs_max2(x[h][u].x, x[h][u].y), abs_max2(x[h][u].z, x[h][u].w)));
      m = abs_max2(m, __shfl_xor_sync(0xffffffffu, m, 1));
      m = abs_max2(m, __shfl_xor_sync(0xffffffffu, m, 2));
      float inv;
      const float scale_x = scale_value(block_scale<BSP_FP8_E4M3>(abs_max_of(m), inv));
      float c[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t q0 = four_to_fp8<BSP_FP8_E4M3>(x[h][0].x, x[h][0].y, inv, inv, inv, inv);
        const uint32_t q1 = four_to_fp8<BSP_FP8_E4M3>(x[h][0].z, x[h][0].w, inv, inv, inv, inv);
        const uint32_t q2 = four_to_fp8<BSP_FP8_E4M3>(x[h][1].x, x[h][1].y, inv, inv, inv, inv);
        const uint32_t q3 = four_to_fp8<BSP_FP8_E4M3>(x[h][1].z, x[h][1].w, inv, inv, inv, inv);
        mma_e4m3(c, w[h][0].x, w[h][1].x, w[h][0].y, w[h][1].y, q0, q1);
        mma_e4m3(c, w[h][0].z, w[h][1].z, w[h][0].w, w[h][1].w, q2, q3);
      }
      // this lane's outputs are of tokens 2 t and 2 t + 1 of the group
      const float s0 = scale_w * __shfl_sync(0xffffffffu, scale_x, 8 * t), s1 = scale_w * __shfl_sync(0xffffffffu, scale_x, 8 * t + 4);
      acc[j][0] = __fmaf_rn(c[0], s0, acc[j][0]);
      acc[j][1] = __fmaf_rn(c[1], s1, acc[j][1]);
      acc[j][2] = __fmaf_rn(c[2], s0, acc[j][2]);
      acc[j][3] = __fmaf_rn(c[3], s1, acc[j][3]);
    }
  }
#pragma unroll
  for (int j = 0; j < GROUPS; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) s_part[(warp * 8 * GROUPS + 8 * j + 2 * t + (e & 1)) * kFewRows + g + 8 * (e >> 1)] = acc[j][e];
  __syncthreads();
  for (int e = threadIdx.x; e < A.tokens * kFewRows; e += blockDim.x) {
    const int n = n0 + (e & (kFewRows - 1)), token = e / kFewRows;
    if (n >= A.n_out) continue;
    float y = 0.0f;
    for (int w = 0; w < warps; ++w) y += s_part[w * 8 * GROUPS * kFewRows + e];
    if (A.bias != nullptr) y += bf16_bits_to_float(ld_global(A.bias + n));
    if (A.act == BSP_ACT_GELU) {
      float unused = 0.0f;
      tc::gelu_erf_pair(y, unused);
    }
    A.Y[static_cast<size_t>(token) * A.ldy + n] = __bfloat16_as_ushort(__float2bfloat16_rn(y));
  }
}

}  // namespace

namespace fp8 {

bool few_tokens_ok(const void* Wq, int ldw, int tokens) { return tokens <= kFewTokens && aligned_to(Wq, 16) && ldw % 16 == 0; }

int launch_few(const void* Wq, int ldw, const uint8_t* WS, int ldws, int n_out, int k_in, const void* X, int tokens, int ldx, const void* bias, int act,
               void* Y, int ldy, cudaStream_t s) {
  const FewArgs A{static_cast<const uint8_t*>(Wq), ldw, WS, ldws, n_out, k_in, static_cast<const uint16_t*>(X), tokens, ldx,
                  aligned_to(X, 16) && ldx % 8 == 0, static_cast<const uint16_t*>(bias), act, static_cast<uint16_t*>(Y), ldy};
  const int blocks = blocks_of(k_in), warps = blocks < kFewMaxWarps ? blocks : kFewMaxWarps;
  const int groups = tokens <= 8 ? 1 : tokens <= 16 ? 2 : 4;
  auto kernel = groups == 1 ? linear_few_kernel<1> : groups == 2 ? linear_few_kernel<2> : linear_few_kernel<4>;
  BSP_CUDA_TRY(launch_pdl(kernel, dim3((n_out - 1) / kFewRows + 1), dim3(32 * warps), sizeof(float) * warps * 8 * groups * kFewRows, s, A));
  return BSP_OK;
}

}  // namespace fp8
}  // namespace bsp
