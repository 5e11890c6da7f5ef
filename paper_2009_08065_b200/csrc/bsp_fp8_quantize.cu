// bsp_fp8_quantize, bsp_fp8_quantize_weight: bf16 matrices to 8 bits with a scale for each block of 128.
//
// A CTA holds a tile of 128 x 128 in registers (256 threads, 8 rows x 8 columns each, all loads in flight) and writes from
// there whichever forms are asked for: along the rows (a scale for each 128 columns of a row: the operand of a product that
// sums over the columns), along the columns (a scale for each 128 rows of a column: the operand of a product that sums over the
// rows), or one scale for the tile (weights: the same 8-bit values then serve both products).  A training step needs the first
// two of the same matrix, and for the output gradient its column sums (the bias gradient) too: one pass over the matrix.
// HBM-bound: 2 bytes read and 1 or 2 written per value.
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
  int wide;                  // 16-byte loads and 8-byte stores are possible
};

enum class QuantKind { kVectors, kTiles };

// Eight values times `inv` as 8 bits.
template <int FMT>
__device__ __forceinline__ uint2 eight_to_fp8(const uint4& x, const float (&inv)[8]) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    h[i] = to_fp8x2<FMT>(__uint_as_float(w[i] << 16) * inv[2 * i], __uint_as_float(w[i] & 0xffff0000u) * inv[2 * i + 1]);
  return make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
}
__device__ __forceinline__ void store_eight(uint8_t* dst, uint2 v, int n, int wide) {
  if (wide && n == 8) {
    *reinterpret_cast<uint2*>(dst) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) dst[i] = static_cast<uint8_t>((i < 4 ? v.x : v.y) >> (8 * (i & 3)));
  }
}
__device__ __forceinline__ uint32_t abs_max8(const uint4& x) {
  return max_u16x2(max_u16x2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), max_u16x2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu));
}
// (a block with an infinity or a NaN is NaN throughout, under scale 1)
constexpr uint32_t kNotFinite = 0x7f80u;

template <int FMT, QuantKind KIND>
__global__ void __launch_bounds__(kQuantThreads)
quantize_kernel(QuantArgs A) {
  constexpr int kTop = top_of(FMT);
  __shared__ uint32_t s_max[8][64];          // [warp][pair of columns]
  __shared__ float s_sum[8][128];
  const int warp = threadIdx.x >> 5, half = threadIdx.x >> 4, l = threadIdx.x & 15;
  const int r0 = blockIdx.y * kBlock, c0 = blockIdx.x * kBlock, c = c0 + 8 * l;
  const int n = min(8, A.cols - c);          // of this thread's columns, those that exist (may be negative)
  pdl_wait();
  pdl_launch_dependents();
  uint4 x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {              // rows half, half + 16, ...
    const int r = r0 + half + 16 * i;
    x[i] = make_uint4(0u, 0u, 0u, 0u);
    if (r < A.rows && n > 0) {
      const uint16_t* src = A.X + static_cast<size_t>(r) * A.ldx + c;
      if (A.wide && n == 8) {
        x[i] = ld_global(reinterpret_cast<const uint4*>(src));
      } else {
        uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < n) w[j >> 1] |= static_cast<uint32_t>(ld_global(src + j)) << (16 * (j & 1));
        x[i] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
  if (KIND == QuantKind::kTiles) {
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max_u16x2(m, abs_max8(x[i]));
    m = __reduce_max_sync(0xffffffffu, max(m & 0xffffu, m >> 16));
    if ((threadIdx.x & 31) == 0) s_max[warp][0] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) m = max(m, s_max[w][0]);
    const bool bad = m >= kNotFinite;
    const int byte = bad ? 127 : scale_byte(m << 16, kTop);
    float inv[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) inv[j] = scale_inverse(byte);
    if (threadIdx.x == 0) A.s_row[static_cast<size_t>(blockIdx.y) * A.lds_row + blockIdx.x] = static_cast<uint8_t>(byte);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = r0 + half + 16 * i;
      if (r < A.rows && n > 0)
        store_eight(A.q_row + static_cast<size_t>(r) * A.ld_row + c, bad ? make_uint2(kNan * 0x01010101u, kNan * 0x01010101u) : eight_to_fp8<FMT>(x[i], inv),
                    n, A.wide);
    }
    return;
  }
  if (A.q_row != nullptr) {
    const uint32_t lanes = 0xffffu << (threadIdx.x & 16);      // the sixteen threads of a row
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = r0 + half + 16 * i;
      uint32_t m = abs_max8(x[i]);
      m = __reduce_max_sync(lanes, max(m & 0xffffu, m >> 16));
      const bool bad = m >= kNotFinite;
      const int byte = bad ? 127 : scale_byte(m << 16, kTop);
      float inv[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) inv[j] = scale_inverse(byte);
      if (r < A.rows) {
        if (l == 0) A.s_row[static_cast<size_t>(r) * A.lds_row + blockIdx.x] = static_cast<uint8_t>(byte);
        if (n > 0)
          store_eight(A.q_row + static_cast<size_t>(r) * A.ld_row + c, bad ? make_uint2(kNan * 0x01010101u, kNan * 0x01010101u) : eight_to_fp8<FMT>(x[i], inv),
                      n, A.wide);
      }
    }
  }
  if (A.q_col != nullptr) {
    uint32_t m[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) m[j] = max_u16x2(m[j], w[j] & 0x7fff7fffu);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m[j] = max_u16x2(m[j], __shfl_xor_sync(0xffffffffu, m[j], 16));
      if ((threadIdx.x & 16) == 0) s_max[warp][4 * l + j] = m[j];
    }
  }
  if (A.partial != nullptr) {
    float sum[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        sum[2 * j] += __uint_as_float(w[j] << 16);
        sum[2 * j + 1] += __uint_as_float(w[j] & 0xffff0000u);
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 16);
      if ((threadIdx.x & 16) == 0) s_sum[warp][8 * l + j] = sum[j];
    }
  }
  if (A.q_col == nullptr && A.partial == nullptr) return;
  __syncthreads();
  if (A.partial != nullptr && threadIdx.x < 128 && c0 + static_cast<int>(threadIdx.x) < A.cols) {
    float t = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; ++w) t += s_sum[w][threadIdx.x];
    A.partial[static_cast<size_t>(blockIdx.y) * A.cols + c0 + threadIdx.x] = t;
  }
  if (A.q_col != nullptr) {
    float inv[8];
    uint32_t bad = 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t m = 0u;
#pragma unroll
      for (int w = 0; w < 8; ++w) m = max_u16x2(m, s_max[w][4 * l + j]);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint32_t mm = u ? m >> 16 : m & 0xffffu;
        const bool b = mm >= kNotFinite;
        const int byte = b ? 127 : scale_byte(mm << 16, kTop);
        if (b) bad |= 1u << (2 * j + u);
        inv[2 * j + u] = scale_inverse(byte);
        if (half == 0 && 2 * j + u < n) A.s_col[static_cast<size_t>(blockIdx.y) * A.lds_col + c + 2 * j + u] = static_cast<uint8_t>(byte);
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = r0 + half + 16 * i;
      if (r < A.rows && n > 0) {
        uint2 q = eight_to_fp8<FMT>(x[i], inv);
        if (bad != 0u) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if ((bad >> j) & 1u) (j < 4 ? q.x : q.y) = ((j < 4 ? q.x : q.y) & ~(0xffu << (8 * (j & 3)))) | (kNan << (8 * (j & 3)));
        }
        store_eight(A.q_col + static_cast<size_t>(r) * A.ld_col + c, q, n, A.wide);
      }
    }
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
  A.wide = aligned_to(X, 16) && ldx % 8 == 0 && (Q == nullptr || (aligned_to(Q, 8) && ldq % 8 == 0)) &&
           (Qc == nullptr || (aligned_to(Qc, 8) && ldqc % 8 == 0));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const dim3 grid(blocks_of(cols), blocks_of(rows));
  if (fmt == BSP_FP8_E4M3) BSP_CUDA_TRY(launch_pdl(quantize_kernel<BSP_FP8_E4M3, QuantKind::kVectors>, grid, dim3(kQuantThreads), 0, s, A));
  else BSP_CUDA_TRY(launch_pdl(quantize_kernel<BSP_FP8_E5M2, QuantKind::kVectors>, grid, dim3(kQuantThreads), 0, s, A));
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
  A.wide = aligned_to(W, 16) && ldw % 8 == 0 && aligned_to(Q, 8) && ldq % 8 == 0;
  BSP_CUDA_TRY(launch_pdl(quantize_kernel<BSP_FP8_E4M3, QuantKind::kTiles>, dim3(blocks_of(k_in), blocks_of(n_out)), dim3(kQuantThreads), 0,
                          static_cast<cudaStream_t>(stream), A));
  return BSP_OK;
}
