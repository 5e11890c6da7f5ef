// The linear layer in 8-bit floating point: entry points, the choice of a kernel, and the plain kernel for operands that the tensor core's
// copies cannot fetch.
#include "bsp_fp8.cuh"
#include "bsp_fp8_gemm.cuh"

namespace bsp {
using namespace fp8;

namespace {

// ------------------------------------------------------------------------------------------ any alignment
// 64 x 64 outputs per CTA, 4 x 4 per thread, 32 of the contraction at a time from shared memory, values already multiplied by
// their scales (powers of two: exact).  For operands whose rows do not begin at multiples of 16 bytes.  Bound by CUDA-core multiply-adds and byte loads:
// 1003 tokens, 920 -> 2128 282 us, 11 with padded rows on tensor cores.
constexpr int kAnyTile = 64, kAnyDepth = 32;

struct AnyArgs {
  Product p;
};

__device__ __forceinline__ float operand_value(const Operand& O, int i, int k) {
  const uint8_t q = ld_global(O.q + (O.mn ? static_cast<size_t>(k) * O.ld + i : static_cast<size_t>(i) * O.ld + k));
  float lo, hi;
  if (O.fmt == BSP_FP8_E4M3) from_fp8x2<BSP_FP8_E4M3>(q, lo, hi);
  else from_fp8x2<BSP_FP8_E5M2>(q, lo, hi);
  return lo * scale_value(ld_global(O.s + static_cast<long long>(i >> O.s_shift) * O.s_row + static_cast<long long>(k / kBlock) * O.s_k));
}

__global__ void __launch_bounds__(256)
product_any_kernel(const __grid_constant__ AnyArgs args) {
  const Product& P = args.p;
  __shared__ float s_a[kAnyDepth][kAnyTile + 1], s_b[kAnyDepth][kAnyTile + 1];
  const int n_tiles = (P.B.rows + kAnyTile - 1) / kAnyTile;
  const int i0 = (blockIdx.x / n_tiles) * kAnyTile, j0 = (blockIdx.x % n_tiles) * kAnyTile;
  const int ti = threadIdx.x >> 4, tj = threadIdx.x & 15;
  float acc[4][4] = {};
  pdl_wait();
  pdl_launch_dependents();
  for (int k0 = 0; k0 < P.contraction; k0 += kAnyDepth) {
    __syncthreads();
    for (int e = threadIdx.x; e < kAnyDepth * kAnyTile; e += 256) {
      // neighbouring threads take neighbouring bytes
      const int ka = P.A.mn ? e / kAnyTile : e % kAnyDepth, ia = P.A.mn ? e % kAnyTile : e / kAnyDepth;
      s_a[ka][ia] = i0 + ia < P.A.rows && k0 + ka < P.contraction ? operand_value(P.A, i0 + ia, k0 + ka) : 0.0f;
      const int kb = P.B.mn ? e / kAnyTile : e % kAnyDepth, jb = P.B.mn ? e % kAnyTile : e / kAnyDepth;
      s_b[kb][jb] = j0 + jb < P.B.rows && k0 + kb < P.contraction ? operand_value(P.B, j0 + jb, k0 + kb) : 0.0f;
    }
    __syncthreads();
#pragma unroll 8
    for (int k = 0; k < kAnyDepth; ++k) {
      float a[4], b[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) { a[u] = s_a[k][ti + 16 * u]; b[u] = s_b[k][tj + 16 * u]; }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[u][v] = __fmaf_rn(a[u], b[v], acc[u][v]);
    }
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int i = i0 + ti + 16 * u, j = j0 + tj + 16 * v;
      if (i >= P.A.rows || j >= P.B.rows) continue;
      float y = acc[u][v] + (P.bias != nullptr ? bf16_bits_to_float(ld_global(P.bias + j)) : 0.0f);
      if (P.act == BSP_ACT_GELU) y = 0.5f * y * (1.0f + erff(y * 0.70710678118654752f));
      if (P.keep != nullptr && ld_global(P.keep + static_cast<size_t>(i / P.block) * P.B.rows + j) == 0) y = 0.0f;
      P.Y[static_cast<size_t>(i) * P.ldy + j] = __bfloat16_as_ushort(__float2bfloat16_rn(y));
    }
  }
}

int run_product(const Product& p, cudaStream_t s) {
  if (p.A.rows > kMostSize || p.B.rows > kMostSize || p.contraction > kMostSize) return BSP_ERR_UNSUPPORTED;
  if (tensor_core_ok(p)) return launch_tensor_core(p, s);
  const long long tiles = static_cast<long long>((p.A.rows + kAnyTile - 1) / kAnyTile) * ((p.B.rows + kAnyTile - 1) / kAnyTile);
  if (tiles > 0x7fffffffLL) return BSP_ERR_UNSUPPORTED;
  BSP_CUDA_TRY(launch_pdl(product_any_kernel, dim3(static_cast<unsigned>(tiles)), dim3(256), 0, s, AnyArgs{p}));
  return BSP_OK;
}

// ------------------------------------------------------------------------------------------ arguments
int check_weight(const void* Wq, int ldw, const uint8_t* WS, int ldws, int n_out, int k_in) {
  if (Wq == nullptr || WS == nullptr || n_out <= 0 || k_in <= 0) return BSP_ERR_ARG;
  return ldw < k_in || ldws < blocks_of(k_in) ? BSP_ERR_SHAPE : BSP_OK;
}
Operand weight_operand(const void* Wq, int ldw, const uint8_t* WS, int ldws, int n_out) {
  return Operand{static_cast<const uint8_t*>(Wq), n_out, ldw, 0, BSP_FP8_E4M3, WS, ldws, 1, 7};
}
// Whether the kernel for few tokens takes a product.  Its CTAs of 16 outputs each read all tokens, and bring them to 8 bits themselves if they are not
// yet (ready).  Up to 8 tokens it is the fastest everywhere, up to 16 unless the weight is large, up to 32 only where it also saves the quantiser's
// launch and the weight is small.  In one launch / quantised first, then on tensor cores (us): 16 tokens, 4096 x 1024 3.6 / 5.0, 2048 x 2048 4.3 / 4.9, 2048
// x 4096 8.5 / 6.1, 4096 x 4096 9.8 / 7.8; 32 tokens, 768 x 768 4.2 / 4.6, 1024 x 1024 4.1 / 4.5, 512 x 2048 4.8 / 4.7, 4096 x 1024 5.8 / 5.0, 1024 x 4096 6.4 /
// 5.9.  Ready, 24 tokens: 1024 x 1024 2.95 / 3.18, 512 x 2048 3.65 / 3.18, 4096 x 1024 3.96 / 3.76.
bool few_is_faster(int tokens, int n_out, int k_in, bool ready) {
  const long long weights = static_cast<long long>(n_out) * k_in;
  return tokens <= 8 || (tokens <= 16 ? weights < (8ll << 20) : !ready && weights <= (1ll << 20));
}
int row_pitch(int k_in) { return (k_in - 1) / 16 * 16 + 16; }

}  // namespace
}  // namespace bsp

extern "C" int bsp_linear_fp8_quantized(const void* Wq, int ldw, const uint8_t* WS, int ldws, int n_out, int k_in, const void* Xq, int ldx,
                                        const uint8_t* XS, int ldxs, int fmt, int tokens, const void* bias, int act, void* Y, int ldy, void* stream) {
  using namespace bsp;
  BSP_TRY(check_weight(Wq, ldw, WS, ldws, n_out, k_in));
  if (Xq == nullptr || XS == nullptr || Y == nullptr || tokens <= 0 || !known_format(fmt)) return BSP_ERR_ARG;
  if ((act != BSP_ACT_NONE && act != BSP_ACT_GELU) || !aligned_to(Y, 2) || !aligned_to(bias, 2)) return BSP_ERR_ARG;
  if (ldx < k_in || ldxs < blocks_of(k_in) || ldy < n_out) return BSP_ERR_SHAPE;
  const Product p{Operand{static_cast<const uint8_t*>(Xq), tokens, ldx, 0, fmt, XS, ldxs, 1, 0}, weight_operand(Wq, ldw, WS, ldws, n_out), k_in,
                  static_cast<uint16_t*>(Y), ldy, static_cast<const uint16_t*>(bias), act, nullptr, 1};
  if (n_out > kMostSize || k_in > kMostSize) return BSP_ERR_UNSUPPORTED;
  if (few_tokens_ok(Wq, ldw, tokens) && aligned_to(Xq, 16) && ldx % 16 == 0 && few_is_faster(tokens, n_out, k_in, true))
    return launch_few_ready(p, static_cast<cudaStream_t>(stream));
  return run_product(p, static_cast<cudaStream_t>(stream));
}

extern "C" int bsp_linear_fp8_ws_bytes(int tokens, int k_in, size_t* bytes) {
  using namespace bsp;
  if (tokens <= 0 || k_in <= 0 || bytes == nullptr) return BSP_ERR_ARG;
  if (tokens > kMostSize || k_in > kMostSize) return BSP_ERR_UNSUPPORTED;
  *bytes = round_up(static_cast<size_t>(tokens) * (row_pitch(k_in) + blocks_of(k_in)), 256);
  return BSP_OK;
}

extern "C" int bsp_linear_fp8(const void* Wq, int ldw, const uint8_t* WS, int ldws, int n_out, int k_in, const void* X, int tokens, int ldx,
                              const void* bias, int act, void* Y, int ldy, void* ws, size_t ws_bytes, void* stream) {
  using namespace bsp;
  BSP_TRY(check_weight(Wq, ldw, WS, ldws, n_out, k_in));
  if (X == nullptr || Y == nullptr || ws == nullptr || tokens <= 0) return BSP_ERR_ARG;
  if ((act != BSP_ACT_NONE && act != BSP_ACT_GELU) || !aligned_to(X, 2) || !aligned_to(Y, 2) || !aligned_to(bias, 2) || !aligned_to(ws, 16))
    return BSP_ERR_ARG;
  if (ldx < k_in || ldy < n_out) return BSP_ERR_SHAPE;
  size_t need = 0;
  BSP_TRY(bsp_linear_fp8_ws_bytes(tokens, k_in, &need));
  if (ws_bytes < need) return BSP_ERR_WORKSPACE;
  if (n_out > kMostSize) return BSP_ERR_UNSUPPORTED;
  if (few_tokens_ok(Wq, ldw, tokens) && few_is_faster(tokens, n_out, k_in, false))
    return launch_few(Wq, ldw, WS, ldws, n_out, k_in, X, tokens, ldx, bias, act, Y, ldy, static_cast<cudaStream_t>(stream));
  uint8_t* Q = static_cast<uint8_t*>(ws);
  uint8_t* S = Q + static_cast<size_t>(tokens) * row_pitch(k_in);
  BSP_TRY(bsp_fp8_quantize(X, tokens, k_in, ldx, BSP_FP8_E4M3, Q, row_pitch(k_in), S, blocks_of(k_in), nullptr, 0, nullptr, 0, nullptr, nullptr, 0,
                           stream));
  return bsp_linear_fp8_quantized(Wq, ldw, WS, ldws, n_out, k_in, Q, row_pitch(k_in), S, blocks_of(k_in), BSP_FP8_E4M3, tokens, bias, act, Y, ldy,
                                  stream);
}

extern "C" int bsp_linear_fp8_backward_input(const void* Wq, int ldw, const uint8_t* WS, int ldws, int n_out, int k_in, const void* dYq, int ldy,
                                             const uint8_t* dYS, int ldys, int fmt, int tokens, void* dX, int ldx, void* stream) {
  using namespace bsp;
  BSP_TRY(check_weight(Wq, ldw, WS, ldws, n_out, k_in));
  if (dYq == nullptr || dYS == nullptr || dX == nullptr || tokens <= 0 || !known_format(fmt) || !aligned_to(dX, 2)) return BSP_ERR_ARG;
  if (ldy < n_out || ldys < blocks_of(n_out) || ldx < k_in) return BSP_ERR_SHAPE;
  // the weight as the operand whose rows are its columns
  const Operand w{static_cast<const uint8_t*>(Wq), k_in, ldw, 1, BSP_FP8_E4M3, WS, 1, ldws, 7};
  const Product p{Operand{static_cast<const uint8_t*>(dYq), tokens, ldy, 0, fmt, dYS, ldys, 1, 0}, w, n_out, static_cast<uint16_t*>(dX), ldx, nullptr,
                  BSP_ACT_NONE, nullptr, 1};
  return run_product(p, static_cast<cudaStream_t>(stream));
}

extern "C" int bsp_linear_fp8_backward_weight(const void* dYq, int ldy, const uint8_t* dYS, int ldys, int fmt_dy, const void* Xq, int ldx,
                                              const uint8_t* XS, int ldxs, int fmt_x, int tokens, int n_out, int k_in, int block, const uint8_t* keep,
                                              void* dW, int lddw, void* stream) {
  using namespace bsp;
  if (dYq == nullptr || dYS == nullptr || Xq == nullptr || XS == nullptr || dW == nullptr || !aligned_to(dW, 2)) return BSP_ERR_ARG;
  if (tokens <= 0 || n_out <= 0 || k_in <= 0 || block <= 0 || !known_format(fmt_dy) || !known_format(fmt_x)) return BSP_ERR_ARG;
  if (n_out % block) return BSP_ERR_SHAPE;
  if (ldy < n_out || ldys < n_out || ldx < k_in || ldxs < k_in || lddw < k_in) return BSP_ERR_SHAPE;
  const Product p{Operand{static_cast<const uint8_t*>(dYq), n_out, ldy, 1, fmt_dy, dYS, 1, ldys, 0},
                  Operand{static_cast<const uint8_t*>(Xq), k_in, ldx, 1, fmt_x, XS, 1, ldxs, 0}, tokens, static_cast<uint16_t*>(dW), lddw, nullptr,
                  BSP_ACT_NONE, keep, block};
  return run_product(p, static_cast<cudaStream_t>(stream));
}
