// bsp_fp8_quantize, bsp_fp8_quantize_weight: bf16 matrices to 8 bits with a scale for each block of 128.
//
// A CTA holds a tile of 128 x 128 in registers (256 threads, 4 rows x 16 columns each, all loads in flight) and writes from
// there whichever forms are asked for: along the rows (a scale for each 128 columns of a row: the operand of a product that
// sums over the columns), along the columns (a scale for each 128 rows of a column: the operand of a product that sums over the
// rows), or one scale for the tile (weights: the same 8-bit values then serve both products).  A training step needs the first
// two of the same matrix, and for the output gradient its column sums (the bias gradient) too: one pass over the matrix.
// HBM-bound: 2 bytes read and 1 or 2 written per value.
#include <algorithm>

#include "bsp_fp8.cuh"

namespace bsp {
using namespace fp8;

namespace {

constexpr int kQuantThreads = 256;

struct QuantArgs {
  const uint16_t* X;
  int rows, cols, ldx;
  uint8_t* q_row;
  int ld_row;
  uint8_t* s_row;
  int lds_row;
  uint8_t* q_col;
  int ld_col;
  uint8_t* s_col;
  int lds_col;
  float* partial;            // column sums of each block of 128 rows, [row blocks, cols], or null
  int wide_in, wide_out;     // 16-byte loads; stores of 16 (2), 8 (1) or single bytes (0)
};

// kRows: along the rows only.  kBoth: along the columns, column sums, and along the rows where asked for.  kTile: one scale for the tile.
enum class QuantKind { kRows, kBoth, kTile };

// Sixteen bytes, of which n exist.
__device__ __forceinline__ void store_sixteen(uint8_t* dst, const uint32_t (&q)[4], int n, int wide) {
  if (wide == 2 && n == 16) {
    *reinterpret_cast<uint4*>(dst) = make_uint4(q[0], q[1], q[2], q[3]);
  } else if (wide >= 1 && n >= 8 && (n & 7) == 0) {
    *reinterpret_cast<uint2*>(dst) = make_uint2(q[0], q[1]);
    if (n == 16) *reinterpret_cast<uint2*>(dst + 8) = make_uint2(q[2], q[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i < n) dst[i] = static_cast<uint8_t>(q[i >> 2] >> (8 * (i & 3)));
  }
}

template <int FMT, QuantKind KIND>
__global__ void __launch_bounds__(kQuantThreads)
quantize_kernel(QuantArgs A) {
  __shared__ uint32_t s_max[8][64];          // [warp][pair of columns]
  __shared__ __align__(16) float s_inv[128];
  __shared__ float s_sum[8][128];
  const int warp = threadIdx.x >> 5, l = threadIdx.x & 7, slot = threadIdx.x >> 3;   // eight threads to a row
  const int r0 = blockIdx.y * kBlock, c0 = blockIdx.x * kBlock, c = c0 + 16 * l;
  const int n = max(0, min(16, A.cols - c));   // of this thread's columns, those that exist
  pdl_wait();
  pdl_launch_dependents();
  uint32_t x[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {              // rows slot, slot + 32, ...
    const int r = r0 + slot + 32 * i;
    const uint16_t* src = A.X + static_cast<size_t>(r) * A.ldx + c;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint4 v = make_uint4(0u, 0u, 0u, 0u);
      if (r < A.rows) {
        if (A.wide_in && n >= 8 * h + 8) {
          v = ld_global(reinterpret_cast<const uint4*>(src + 8 * h));
        } else if (n > 8 * h) {
          uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (8 * h + j < n) w[j >> 1] |= static_cast<uint32_t>(ld_global(src + 8 * h + j)) << (16 * (j & 1));
          v = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
      x[i][4 * h] = v.x; x[i][4 * h + 1] = v.y; x[i][4 * h + 2] = v.z; x[i][4 * h + 3] = v.w;
    }
  }
  if (KIND == QuantKind::kTile) {
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) m = abs_max2(m, x[i][j]);
    m = __reduce_max_sync(0xffffffffu, abs_max_of(m));
    if ((threadIdx.x & 31) == 0) s_max[warp][0] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) m = max(m, s_max[w][0]);
    float inv;
    const uint32_t byte = block_scale<FMT>(m, inv);
    if (threadIdx.x == 0) A.s_row[static_cast<size_t>(blockIdx.y) * A.lds_row + blockIdx.x] = static_cast<uint8_t>(byte);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = r0 + slot + 32 * i;
      if (r >= A.rows) continue;
      uint32_t q[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) q[j] = four_to_fp8<FMT>(x[i][2 * j], x[i][2 * j + 1], inv, inv, inv, inv);
      store_sixteen(A.q_row + static_cast<size_t>(r) * A.ld_row + c, q, n, A.wide_out);
    }
    return;
  }
  if (KIND == QuantKind::kRows || A.q_row != nullptr) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = r0 + slot + 32 * i;
      uint32_t m = abs_max2(x[i][0], x[i][1]);
#pragma unroll
      for (int j = 2; j < 8; ++j) m = abs_max2(m, x[i][j]);
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) m = abs_max2(m, __shfl_xor_sync(0xffffffffu, m, o));
      float inv;
      const uint32_t byte = block_scale<FMT>(abs_max_of(m), inv);
      if (r >= A.rows) continue;
      if (l == 0) A.s_row[static_cast<size_t>(r) * A.lds_row + blockIdx.x] = static_cast<uint8_t>(byte);
      uint32_t q[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) q[j] = four_to_fp8<FMT>(x[i][2 * j], x[i][2 * j + 1], inv, inv, inv, inv);
      store_sixteen(A.q_row + static_cast<size_t>(r) * A.ld_row + c, q, n, A.wide_out);
    }
  }
  if (KIND == QuantKind::kRows) return;
  if (A.q_col != nullptr) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t m = abs_max2(abs_max2(x[0][j], x[1][j]), abs_max2(x[2][j], x[3][j]));
      m = abs_max2(m, __shfl_xor_sync(0xffffffffu, m, 8));
      m = abs_max2(m, __shfl_xor_sync(0xffffffffu, m, 16));
      if ((threadIdx.x & 24) == 0) s_max[warp][8 * l + j] = m;
    }
  }
  if (A.partial != nullptr) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float lo = 0.0f, hi = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lo += __uint_as_float(x[i][j] << 16);
        hi += __uint_as_float(x[i][j] & 0xffff0000u);
      }
#pragma unroll
      for (int o = 8; o < 32; o <<= 1) {
        lo += __shfl_xor_sync(0xffffffffu, lo, o);
        hi += __shfl_xor_sync(0xffffffffu, hi, o);
      }
      if ((threadIdx.x & 24) == 0) {
        s_sum[warp][16 * l + 2 * j] = lo;
        s_sum[warp][16 * l + 2 * j + 1] = hi;
      }
    }
  }
  __syncthreads();
  if (threadIdx.x < 64) {                    // a pair of columns each
    if (A.q_col != nullptr) {
      uint32_t m = 0u;
#pragma unroll
      for (int w = 0; w < 8; ++w) m = abs_max2(m, s_max[w][threadIdx.x]);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int at = 2 * threadIdx.x + u;
        float inv;
        const uint32_t byte = block_scale<FMT>((u ? m >> 16 : m) & 0x7fffu, inv);
        s_inv[at] = inv;
        if (c0 + at < A.cols) A.s_col[static_cast<size_t>(blockIdx.y) * A.lds_col + c0 + at] = static_cast<uint8_t>(byte);
      }
    }
  } else if (A.partial != nullptr && threadIdx.x >= 128 && c0 + static_cast<int>(threadIdx.x) - 128 < A.cols) {
    float t = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; ++w) t += s_sum[w][threadIdx.x - 128];
    A.partial[static_cast<size_t>(blockIdx.y) * A.cols + c0 + threadIdx.x - 128] = t;
  }
  if (A.q_col == nullptr) return;
  __syncthreads();
  float4 inv[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) inv[j] = reinterpret_cast<const float4*>(s_inv)[4 * l + j];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = r0 + slot + 32 * i;
    if (r >= A.rows) continue;
    uint32_t q[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = four_to_fp8<FMT>(x[i][2 * j], x[i][2 * j + 1], inv[j].x, inv[j].y, inv[j].z, inv[j].w);
    store_sixteen(A.q_col + static_cast<size_t>(r) * A.ld_col + c, q, n, A.wide_out);
  }
}

// The blocks' column sums, added in their order.
__global__ void __launch_bounds__(128)
column_sums_kernel(const float* partial, int blocks, int cols, float* out) {
  const int c = blockIdx.x * 128 + threadIdx.x;
  pdl_wait();
  pdl_launch_dependents();
  if (c >= cols) return;
  float t = 0.0f;
#pragma unroll 8
  for (int b = 0; b < blocks; ++b) t += ld_global(partial + static_cast<size_t>(b) * cols + c);
  out[c] = t;
}

int wide_stores(const void* q, int ld) { return aligned_to(q, 16) && ld % 16 == 0 ? 2 : aligned_to(q, 8) && ld % 8 == 0 ? 1 : 0; }
bool grid_fits(int rows) { return blocks_of(rows) <= 65535; }

}  // namespace
}  // namespace bsp

extern "C" int bsp_fp8_quantize(const void* X, int rows, int cols, int ldx, int fmt, void* Q, int ldq, uint8_t* S, int lds, void* Qc,
                                int ldqc, uint8_t* Sc, int ldsc, float* col_sums, void* ws, size_t ws_bytes, void* stream) {
  using namespace bsp;
  if (X == nullptr || rows <= 0 || cols <= 0 || !known_format(fmt) || !aligned_to(X, 2)) return BSP_ERR_ARG;
  if ((Q == nullptr) != (S == nullptr) || (Qc == nullptr) != (Sc == nullptr)) return BSP_ERR_ARG;
  if (Q == nullptr && Qc == nullptr && col_sums == nullptr) return BSP_ERR_ARG;
  if (ldx < cols || (Q != nullptr && (ldq < cols || lds < blocks_of(cols))) || (Qc != nullptr && (ldqc < cols || ldsc < cols))) return BSP_ERR_SHAPE;
  if (!grid_fits(rows)) return BSP_ERR_UNSUPPORTED;
  if (col_sums != nullptr) {
    if (ws == nullptr || !aligned_to(ws, 4) || !aligned_to(col_sums, 4)) return BSP_ERR_ARG;
    if (ws_bytes < sizeof(float) * static_cast<size_t>(blocks_of(rows)) * cols) return BSP_ERR_WORKSPACE;
  }
  QuantArgs A;
  A.X = static_cast<const uint16_t*>(X);
  A.rows = rows; A.cols = cols; A.ldx = ldx;
  A.q_row = static_cast<uint8_t*>(Q); A.ld_row = ldq; A.s_row = S; A.lds_row = lds;
  A.q_col = static_cast<uint8_t*>(Qc); A.ld_col = ldqc; A.s_col = Sc; A.lds_col = ldsc;
  A.partial = col_sums != nullptr ? static_cast<float*>(ws) : nullptr;
  A.wide_in = aligned_to(X, 16) && ldx % 8 == 0;
  A.wide_out = std::min(wide_stores(Q, ldq), wide_stores(Qc, ldqc));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const dim3 grid(blocks_of(cols), blocks_of(rows));
  const bool rows_only = Qc == nullptr && col_sums == nullptr;
  auto kernel = fmt == BSP_FP8_E4M3 ? (rows_only ? quantize_kernel<BSP_FP8_E4M3, QuantKind::kRows> : quantize_kernel<BSP_FP8_E4M3, QuantKind::kBoth>)
                                    : (rows_only ? quantize_kernel<BSP_FP8_E5M2, QuantKind::kRows> : quantize_kernel<BSP_FP8_E5M2, QuantKind::kBoth>);
  BSP_CUDA_TRY(launch_pdl(kernel, grid, dim3(kQuantThreads), 0, s, A));
  if (col_sums != nullptr)
    BSP_CUDA_TRY(launch_pdl(column_sums_kernel, dim3(blocks_of(cols)), dim3(128), 0, s, A.partial, static_cast<int>(grid.y), cols, col_sums));
  return BSP_OK;
}

extern "C" int bsp_fp8_quantize_weight(const void* W, int n_out, int k_in, int ldw, void* Q, int ldq, uint8_t* S, int lds, void* stream) {
  using namespace bsp;
  if (W == nullptr || Q == nullptr || S == nullptr || n_out <= 0 || k_in <= 0 || !aligned_to(W, 2)) return BSP_ERR_ARG;
  if (ldw < k_in || ldq < k_in || lds < blocks_of(k_in)) return BSP_ERR_SHAPE;
  if (!grid_fits(n_out)) return BSP_ERR_UNSUPPORTED;
  QuantArgs A = {};
  A.X = static_cast<const uint16_t*>(W);
  A.rows = n_out; A.cols = k_in; A.ldx = ldw;
  A.q_row = static_cast<uint8_t*>(Q); A.ld_row = ldq; A.s_row = S; A.lds_row = lds;
  A.wide_in = aligned_to(W, 16) && ldw % 8 == 0;
  A.wide_out = wide_stores(Q, ldq);
  BSP_CUDA_TRY(launch_pdl(quantize_kernel<BSP_FP8_E4M3, QuantKind::kTile>, dim3(blocks_of(k_in), blocks_of(n_out)), dim3(kQuantThreads), 0,
                          static_cast<cudaStream_t>(stream), A));
  return BSP_OK;
}
