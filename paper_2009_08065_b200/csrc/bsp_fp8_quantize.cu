// bsp_fp8_quantize, bsp_fp8_quantize_weight: bf16 matrices to 8 bits with a scale for each block of 128.
//
// A CTA holds a tile of 128 x 128 in registers (256 threads, 4 rows x 16 columns each, all loads in flight; along the rows alone, beyond 64 of them, 64 x 128
// and 128 threads) and writes from there whichever forms are asked for: along the rows (a scale for each 128 columns of a row: the operand of a product that
// sums over the columns), along the columns (a scale for each 128 rows of a column: the operand of a product that sums over the
// rows), or one scale for the tile (weights: the same 8-bit values then serve both products).  A training step needs the first
// two of the same matrix, and for the output gradient its column sums (the bias gradient) too: one pass over the matrix.
// 2 bytes read and 1 or 2 written per value: along the rows HBM binds, along both directions half of the time goes at barriers (see there).
#include <algorithm>

#include "bsp_fp8.cuh"
#include "bsp_tc.cuh"

namespace bsp {
using namespace fp8;

namespace {

constexpr int kQuantThreads = 256;
constexpr int kMostCluster = 8;              // CTAs

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
  float* sums;               // or, where the row blocks are one cluster, the column sums
  int wide_in, wide_out;     // 16-byte loads; stores of 16 (2), 8 (1) or single bytes (0)
};

// A pair of bf16 values as float32, and times a pair of multipliers.
__device__ __forceinline__ unsigned long long values_of(uint32_t x) { return tc::pack_f32x2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)); }
// Two pairs of values times their multipliers, as 8 bits.
template <int FMT>
__device__ __forceinline__ uint32_t four_times(unsigned long long v0, unsigned long long v1, unsigned long long m0, unsigned long long m1) {
  float x[4];
  unsigned long long p0, p1;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(p0) : "l"(v0), "l"(m0));
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(p1) : "l"(v1), "l"(m1));
  tc::unpack_f32x2(p0, x[0], x[1]);
  tc::unpack_f32x2(p1, x[2], x[3]);
  return to_fp8x4<FMT>(x[0], x[1], x[2], x[3]);
}
__device__ __noinline__ void store_some(uint8_t* dst, uint4 q, int n) {
  unsigned long long v = q.x | (static_cast<unsigned long long>(q.y) << 32);
#pragma unroll 1
  for (int i = 0; i < n; ++i, v >>= 8) {
    if (i == 8) v = q.z | (static_cast<unsigned long long>(q.w) << 32);
    dst[i] = static_cast<uint8_t>(v);
  }
}
// Sixteen bytes, of which n exist.
template <bool kWhole = false>
__device__ __forceinline__ void store_sixteen(uint8_t* dst, const uint32_t (&q)[4], int n, int wide) {
  if (kWhole || (wide == 2 && n == 16)) {
    *reinterpret_cast<uint4*>(dst) = make_uint4(q[0], q[1], q[2], q[3]);
  } else if (wide >= 1 && n >= 8 && (n & 7) == 0) {
    *reinterpret_cast<uint2*>(dst) = make_uint2(q[0], q[1]);
    if (n == 16) *reinterpret_cast<uint2*>(dst + 8) = make_uint2(q[2], q[3]);
  } else if (n > 0) {
    store_some(dst, make_uint4(q[0], q[1], q[2], q[3]), n);
  }
}

// Up to eight values one by one.  (A loop, and so below: unrolled into every place that may need it, this was most of the kernel's code,
// and in a short launch every instruction is fetched for the first time.)
__device__ __noinline__ uint4 load_some(const uint16_t* src, int n) {
  unsigned long long lo = 0ull, hi = 0ull;
#pragma unroll 1
  for (int j = 0; j < n; ++j) {
    const unsigned long long v = ld_global(src + j);
    if (j < 4) lo |= v << (16 * j);
    else hi |= v << (16 * (j - 4));
  }
  return make_uint4(static_cast<uint32_t>(lo), static_cast<uint32_t>(lo >> 32), static_cast<uint32_t>(hi), static_cast<uint32_t>(hi >> 32));
}
// A thread's rows x 16 columns of the tile, as pairs.
template <bool kWhole, int STEP, int ROWS>
__device__ __forceinline__ void load_tile(const QuantArgs& A, int r0, int c, int n, uint32_t (&x)[ROWS][8]) {
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {           // evenly spread from this thread's first one on
    const int r = r0 + STEP * i;
    const uint16_t* src = A.X + static_cast<size_t>(r) * A.ldx + c;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint4 v = make_uint4(0u, 0u, 0u, 0u);
      if (kWhole || r < A.rows) {
        if (kWhole || (A.wide_in && n >= 8 * h + 8)) {
          v = ld_global(reinterpret_cast<const uint4*>(src + 8 * h));
        } else if (n > 8 * h) {
          v = load_some(src + 8 * h, min(8, n - 8 * h));
        }
      }
      x[i][4 * h] = v.x; x[i][4 * h + 1] = v.y; x[i][4 * h + 2] = v.z; x[i][4 * h + 3] = v.w;
    }
  }
}
// Largest magnitude of a row of the tile, by its eight threads.
__device__ __forceinline__ uint32_t row_max(const uint32_t (&x)[8]) {
  uint32_t m = abs_max2(x[0], x[1]);
#pragma unroll
  for (int j = 2; j < 8; ++j) m = abs_max2(m, x[j]);
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) m = abs_max2(m, __shfl_xor_sync(0xffffffffu, m, o));
  return abs_max_of(m);
}

// Along the rows, or (kTile) with one scale for the tile of 128 x 128.  Along the rows a CTA is 128 threads with 64 rows: 8192 registers, which
// an SM has left beside a CTA of the products (bsp_gemm_fp8.cu).  With 256 threads neither could take its seat while the other ran: 1003 tokens, 4096 x 1024
// 12.4 us for the whole layer, this way 11.4.  Up to 64 rows 256 threads share what there is (64 tokens, 1024 x 4096 6.3 and 6.8 us).
constexpr int kSmallThreads = 128;
template <int FMT, bool kTile, int THREADS>
__global__ void __launch_bounds__(THREADS)
quantize_kernel(QuantArgs A) {
  constexpr int kRows = THREADS / 2, kStep = kRows / 4;
  static_assert(!kTile || kRows == kBlock, "a tile to a CTA");
  __shared__ uint32_t s_max[8];
  const int warp = threadIdx.x >> 5, l = threadIdx.x & 7, slot = threadIdx.x >> 3;   // eight threads to a row
  const int col_blocks = blocks_of(A.cols), tile_r = static_cast<int>(blockIdx.x) / col_blocks, tile_c = static_cast<int>(blockIdx.x) - tile_r * col_blocks;
  const int r0 = tile_r * kRows + slot, c = tile_c * kBlock + 16 * l;
  const int n = max(0, min(16, A.cols - c));   // of this thread's columns, those that exist
  pdl_wait();
  pdl_launch_dependents();
  uint32_t x[4][8];
  load_tile<false, kStep>(A, r0, c, n, x);
  uint32_t tile = 0u;
  if (kTile) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) tile = abs_max2(tile, x[i][j]);
    tile = __reduce_max_sync(0xffffffffu, abs_max_of(tile));
    if ((threadIdx.x & 31) == 0) s_max[warp] = tile;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) tile = max(tile, s_max[w]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = r0 + kStep * i;
    float inv;
    const uint32_t byte = block_scale<FMT>(kTile ? tile : row_max(x[i]), inv);
    if (r >= A.rows) continue;
    if (kTile ? threadIdx.x == 0 && i == 0 : l == 0)
      A.s_row[static_cast<size_t>(kTile ? tile_r : r) * A.lds_row + tile_c] = static_cast<uint8_t>(byte);
    uint32_t q[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = four_to_fp8<FMT>(x[i][2 * j], x[i][2 * j + 1], inv, inv, inv, inv);
    store_sixteen(A.q_row + static_cast<size_t>(r) * A.ld_row + c, q, n, A.wide_out);
  }
}

// Along the columns, and column sums and along the rows where they are asked for.  Bound by issue beside HBM (14 instructions a value,
// 18 with column sums, and half of the time waiting for the other warps' maxima): every pair is unpacked once for both forms and multiplied
// as a pair, and whole tiles have a body without conditions.  4096 x 4096 14.7 us (10.3 of HBM; 15.7 with one body for all tiles), with column sums
// 17.3; 512 threads with two rows each, or the rows' form ahead of the barrier, were no faster.
constexpr int kBothRows = kBlock * 8 / kQuantThreads, kBothWarps = kQuantThreads / 32;
struct BothShared {
  uint32_t max[kBothWarps][64];              // [warp][pair of columns]
  float sum[kBothWarps][128];
  float inv[128];
};
// kWhole: the tile is whole, and its rows begin at multiples of 16 bytes everywhere.
template <int FMT, bool kWhole>
__device__ __forceinline__ void quantize_both(const QuantArgs& A, BothShared& s) {
  constexpr int kRows = kBothRows, kWarps = kBothWarps, kStep = kBlock / kRows;
  const int warp = threadIdx.x >> 5, l = threadIdx.x & 7, slot = threadIdx.x >> 3;
  const int r0 = blockIdx.y * kBlock + slot, c0 = blockIdx.x * kBlock, c = c0 + 16 * l;
  const int n = max(0, min(16, A.cols - c));
  uint32_t x[kRows][8];
  load_tile<kWhole, kStep>(A, r0, c, n, x);
  if (A.q_col != nullptr) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t m = x[0][j];
#pragma unroll
      for (int i = 1; i < kRows; ++i) m = abs_max2(m, x[i][j]);
      m = abs_max2(m, __shfl_xor_sync(0xffffffffu, m, 8));
      m = abs_max2(m, __shfl_xor_sync(0xffffffffu, m, 16));
      if ((threadIdx.x & 24) == 0) s.max[warp][8 * l + j] = m;
    }
  }
  if (A.partial != nullptr || A.sums != nullptr) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float lo = 0.0f, hi = 0.0f;
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        lo += __uint_as_float(x[i][j] << 16);
        hi += __uint_as_float(x[i][j] & 0xffff0000u);
      }
#pragma unroll
      for (int o = 8; o < 32; o <<= 1) {
        lo += __shfl_xor_sync(0xffffffffu, lo, o);
        hi += __shfl_xor_sync(0xffffffffu, hi, o);
      }
      if ((threadIdx.x & 24) == 0) *reinterpret_cast<float2*>(&s.sum[warp][16 * l + 2 * j]) = make_float2(lo, hi);
    }
  }
  __syncthreads();
  if (threadIdx.x < 64) {                    // a pair of columns each
    if (A.q_col != nullptr) {
      uint32_t m = 0u;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) m = abs_max2(m, s.max[w][threadIdx.x]);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int at = 2 * threadIdx.x + u;
        float inv;
        const uint32_t byte = block_scale<FMT>((u ? m >> 16 : m) & 0x7fffu, inv);
        s.inv[at] = inv;
        if (kWhole || c0 + at < A.cols) A.s_col[static_cast<size_t>(blockIdx.y) * A.lds_col + c0 + at] = static_cast<uint8_t>(byte);
      }
    }
  } else if ((A.partial != nullptr || A.sums != nullptr) && threadIdx.x >= 128) {
    const int at = threadIdx.x - 128;
    float t = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) t += s.sum[w][at];
    if (A.sums != nullptr) s.sum[0][at] = t;                         // (nobody else uses this column's sums)
    else if (c0 + at < A.cols) A.partial[static_cast<size_t>(blockIdx.y) * A.cols + c0 + at] = t;
  }
  uint32_t top[kRows];
  if (A.q_row != nullptr) {
#pragma unroll
    for (int i = 0; i < kRows; ++i) top[i] = row_max(x[i]);
  }
  __syncthreads();
  if (A.sums != nullptr) tc::cluster_arrive();                       // this CTA's sums are there
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int r = r0 + kStep * i;
    if (!kWhole && r >= A.rows) continue;
    float inv = 0.0f;
    if (A.q_row != nullptr) {
      const uint32_t byte = block_scale<FMT>(top[i], inv);
      if (l == 0) A.s_row[static_cast<size_t>(r) * A.lds_row + blockIdx.x] = static_cast<uint8_t>(byte);
    }
    const unsigned long long along = tc::pack_f32x2(inv, inv);
    uint32_t q[4], p[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned long long v0 = values_of(x[i][2 * j]), v1 = values_of(x[i][2 * j + 1]);
      q[j] = four_times<FMT>(v0, v1, along, along);
      const float4 down = A.q_col != nullptr ? reinterpret_cast<const float4*>(s.inv)[4 * l + j] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      p[j] = four_times<FMT>(v0, v1, tc::pack_f32x2(down.x, down.y), tc::pack_f32x2(down.z, down.w));
    }
    if (A.q_row != nullptr) store_sixteen<kWhole>(A.q_row + static_cast<size_t>(r) * A.ld_row + c, q, n, A.wide_out);
    if (A.q_col != nullptr) store_sixteen<kWhole>(A.q_col + static_cast<size_t>(r) * A.ld_col + c, p, n, A.wide_out);
  }
  if (A.sums != nullptr) {
    // each CTA adds up some of the columns, the row blocks in their order
    tc::cluster_wait();
    const uint32_t ranks = tc::cluster_size();
    if (threadIdx.x < 128 && threadIdx.x % ranks == tc::cluster_rank() && c0 + static_cast<int>(threadIdx.x) < A.cols) {
      float t = 0.0f;
      for (uint32_t k = 0; k < ranks; ++k) {
        float part;
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(part) : "r"(tc::map_to_cta(tc::smem_u32(&s.sum[0][threadIdx.x]), k)) : "memory");
        t += part;
      }
      A.sums[c0 + threadIdx.x] = t;
    }
    tc::cluster_arrive_relaxed();            // no CTA leaves while another may read its sums
    tc::cluster_wait();
  }
}
template <int FMT>
__global__ void __launch_bounds__(kQuantThreads, 4)
quantize_both_kernel(QuantArgs A) {
  __shared__ __align__(16) BothShared s;
  pdl_wait();
  pdl_launch_dependents();
  const bool whole = A.wide_in && A.wide_out == 2 && static_cast<int>(blockIdx.y + 1) * kBlock <= A.rows && static_cast<int>(blockIdx.x + 1) * kBlock <= A.cols;
  if (whole) quantize_both<FMT, true>(A, s);
  else quantize_both<FMT, false>(A, s);
}

// The blocks' column sums: four runs of blocks side by side, and the runs in their order.
__global__ void __launch_bounds__(512)
column_sums_kernel(const float* partial, int blocks, int cols, float* out) {
  __shared__ float s_sum[4][128];
  const int c = blockIdx.x * 128 + (threadIdx.x & 127), run = threadIdx.x >> 7;
  const int each = (blocks + 3) / 4, begin = run * each, end = min(blocks, begin + each);
  pdl_wait();
  pdl_launch_dependents();
  float t = 0.0f;
  if (c < cols) {
#pragma unroll 8
    for (int b = begin; b < end; ++b) t += ld_global(partial + static_cast<size_t>(b) * cols + c);
  }
  s_sum[run][threadIdx.x & 127] = t;
  __syncthreads();
  if (run == 0 && c < cols) out[c] = s_sum[0][threadIdx.x] + s_sum[1][threadIdx.x] + s_sum[2][threadIdx.x] + s_sum[3][threadIdx.x];
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
  if (!grid_fits(rows) || cols > kMostSize) return BSP_ERR_UNSUPPORTED;
  if (col_sums != nullptr) {
    if (ws == nullptr || !aligned_to(ws, 4) || !aligned_to(col_sums, 4)) return BSP_ERR_ARG;
    if (ws_bytes < sizeof(float) * static_cast<size_t>(blocks_of(rows)) * cols) return BSP_ERR_WORKSPACE;
  }
  QuantArgs A;
  A.X = static_cast<const uint16_t*>(X);
  A.rows = rows; A.cols = cols; A.ldx = ldx;
  A.q_row = static_cast<uint8_t*>(Q); A.ld_row = ldq; A.s_row = S; A.lds_row = lds;
  A.q_col = static_cast<uint8_t*>(Qc); A.ld_col = ldqc; A.s_col = Sc; A.lds_col = ldsc;
  // Up to 1024 rows the row blocks of 128 columns are a cluster, which adds up their sums itself: one launch less (407 x 1920 5.0 -> 4.5 us, 700 x 1024 5.1 -> 4.7).
  const bool in_cluster = col_sums != nullptr && blocks_of(rows) <= kMostCluster;
  A.partial = col_sums != nullptr && !in_cluster ? static_cast<float*>(ws) : nullptr;
  A.sums = in_cluster ? col_sums : nullptr;
  A.wide_in = aligned_to(X, 16) && ldx % 8 == 0;
  A.wide_out = std::min(wide_stores(Q, ldq), wide_stores(Qc, ldqc));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const dim3 grid(blocks_of(cols), blocks_of(rows));
  const bool rows_only = Qc == nullptr && col_sums == nullptr;
  if (rows_only) {
    const int threads = rows <= kSmallThreads / 2 ? kQuantThreads : kSmallThreads;
    const long long tiles = ((rows - 1ll) / (threads / 2) + 1) * grid.x;
    if (tiles > 0x7fffffffll) return BSP_ERR_UNSUPPORTED;
    auto rows_kernel = fmt == BSP_FP8_E4M3
                           ? (threads == kSmallThreads ? quantize_kernel<BSP_FP8_E4M3, false, kSmallThreads> : quantize_kernel<BSP_FP8_E4M3, false, kQuantThreads>)
                           : (threads == kSmallThreads ? quantize_kernel<BSP_FP8_E5M2, false, kSmallThreads> : quantize_kernel<BSP_FP8_E5M2, false, kQuantThreads>);
    BSP_CUDA_TRY(launch_pdl(rows_kernel, dim3(static_cast<unsigned>(tiles)), dim3(threads), 0, s, A));
    return BSP_OK;
  }
  auto kernel = fmt == BSP_FP8_E4M3 ? quantize_both_kernel<BSP_FP8_E4M3> : quantize_both_kernel<BSP_FP8_E5M2>;
  if (in_cluster) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kQuantThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 1;
    attr[1].val.clusterDim.y = grid.y;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    BSP_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, A));
    return BSP_OK;
  }
  BSP_CUDA_TRY(launch_pdl(kernel, grid, dim3(kQuantThreads), 0, s, A));
  if (col_sums != nullptr)
    BSP_CUDA_TRY(launch_pdl(column_sums_kernel, dim3(blocks_of(cols)), dim3(512), 0, s, A.partial, static_cast<int>(grid.y), cols, col_sums));
  return BSP_OK;
}

extern "C" int bsp_fp8_quantize_weight(const void* W, int n_out, int k_in, int ldw, void* Q, int ldq, uint8_t* S, int lds, void* stream) {
  using namespace bsp;
  if (W == nullptr || Q == nullptr || S == nullptr || n_out <= 0 || k_in <= 0 || !aligned_to(W, 2)) return BSP_ERR_ARG;
  if (ldw < k_in || ldq < k_in || lds < blocks_of(k_in)) return BSP_ERR_SHAPE;
  if (!grid_fits(n_out) || k_in > kMostSize) return BSP_ERR_UNSUPPORTED;
  QuantArgs A = {};
  A.X = static_cast<const uint16_t*>(W);
  A.rows = n_out; A.cols = k_in; A.ldx = ldw;
  A.q_row = static_cast<uint8_t*>(Q); A.ld_row = ldq; A.s_row = S; A.lds_row = lds;
  A.wide_in = aligned_to(W, 16) && ldw % 8 == 0;
  A.wide_out = wide_stores(Q, ldq);
  const long long tiles = static_cast<long long>(blocks_of(k_in)) * blocks_of(n_out);
  if (tiles > 0x7fffffffll) return BSP_ERR_UNSUPPORTED;
  BSP_CUDA_TRY(launch_pdl(quantize_kernel<BSP_FP8_E4M3, true, kQuantThreads>, dim3(static_cast<unsigned>(tiles)), dim3(kQuantThreads), 0,
                          static_cast<cudaStream_t>(stream), A));
  return BSP_OK;
}
