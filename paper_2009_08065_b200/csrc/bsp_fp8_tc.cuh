// What the tensor-core kernels of 8-bit operands share: scales on their way to tensor memory, descriptors, tensor maps.
#pragma once

#include "bsp_fp8.cuh"
#include "bsp_fp8_gemm.cuh"
#include "bsp_tc.cuh"

namespace bsp {
namespace fp8 {

using namespace tc;

constexpr int kScaleTile = 512;                    // bytes: 128 rows x 4 blocks
// A load without a branch around it, zero where it does not take place: the loads of a group of scales have to be in flight together
// (one after the other, 0.4 us each, they had bound the whole kernel: 8192 x 4096 x 4096 130 us, and its weight gradient 241).
__device__ __forceinline__ uint32_t load_word_if(const void* p, bool there) {
  uint32_t v;
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %2, 0;\n\tmov.b32 %0, 0;\n\t@p ld.global.b32 %0, [%1];\n\t}" : "=r"(v) : "l"(p), "r"(there ? 1u : 0u));
  return v;
}
// How an operand's scales lie: those of a row next to each other (row form of activations), those of a block next to each other (column
// form), or one for each 128 rows (weights, either way round).
enum class ScaleForm { kRows, kColumns, kTiles };

// Scales of up to eight blocks (from `block0` on, n of them) of the 128 rows from `row0` on: load() asks for them, all together, and
// store() writes those of four blocks to a tile of 512 bytes as the tensor core wants it, row r at 16 (r % 32) + 4 (r / 32).
// Arrays begin anywhere: bytes at an address that is no multiple of four come from two words (aligned words that hold a byte
// of the array are read whole).  Scales that do not exist may be anything: no instruction, or no output that exists, uses them.
template <ScaleForm FORM>
struct Scales {
  uint32_t x[FORM == ScaleForm::kRows ? 12 : FORM == ScaleForm::kColumns ? 16 : 1];

  static __device__ __forceinline__ uint32_t offset(const uint8_t* p) { return static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p) & 3u); }

  __device__ __forceinline__ void load(const Operand& O, int row0, int block0, int n, int lane) {
    if (FORM == ScaleForm::kTiles) {
      // at most two different scales for a block: one byte per lane
      const int first = row0 >> O.s_shift, last = (O.rows - 1) >> O.s_shift;
      x[0] = ld_global(O.s + min(first + ((lane >> 3) & 1), last) * O.s_row + (block0 + min(lane & 7, n - 1)) * O.s_k);
    } else if (FORM == ScaleForm::kRows) {               // lane l: rows l, l + 32, l + 64, l + 96
      const bool wide = ((reinterpret_cast<uintptr_t>(O.s) | static_cast<uintptr_t>(O.s_row) | static_cast<uintptr_t>(block0)) & 7u) == 0;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int r = row0 + lane + 32 * q;
        const uint8_t* p = O.s + r * O.s_row + block0;
        if (wide) {
          asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %3, 0;\n\tmov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\t@p ld.global.v2.b32 {%0, %1}, [%2];\n\t}"
                       : "=r"(x[3 * q]), "=r"(x[3 * q + 1]) : "l"(p), "r"(r < O.rows ? 1u : 0u));
          x[3 * q + 2] = 0u;
        } else {
          const int bytes = r < O.rows ? n + static_cast<int>(offset(p)) : 0;           // from the first word's beginning on
#pragma unroll
          for (int i = 0; i < 3; ++i) x[3 * q + i] = load_word_if(p - offset(p) + 4 * i, 4 * i < bytes);
        }
      }
    } else {                                             // lane l: rows 4 l to 4 l + 3
      const int r = row0 + 4 * lane;
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        const uint8_t* p = O.s + (block0 + b) * O.s_k + r;
        const int bytes = b < n && r < O.rows ? O.rows - r + static_cast<int>(offset(p)) : 0;
        x[2 * b] = load_word_if(p - offset(p), bytes > 0);
        x[2 * b + 1] = load_word_if(p - offset(p) + 4, offset(p) != 0u && bytes > 4);
      }
    }
  }
  // Blocks block0 + 4 g to block0 + 4 g + 3 (load's block0).
  __device__ __forceinline__ void store(const Operand& O, int row0, int block0, int g, uint32_t dst, int lane) const {
    if (FORM == ScaleForm::kTiles) {
      uint32_t w[2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
        w[i] = __shfl_sync(0xffffffffu, x[0], 8 * i + 4 * g) | (__shfl_sync(0xffffffffu, x[0], 8 * i + 4 * g + 1) << 8) |
               (__shfl_sync(0xffffffffu, x[0], 8 * i + 4 * g + 2) << 16) | (__shfl_sync(0xffffffffu, x[0], 8 * i + 4 * g + 3) << 24);
      auto word = [&](int q) { return (row0 + lane + 32 * q) >> O.s_shift == row0 >> O.s_shift ? w[0] : w[1]; };
      st_shared_v4(dst + 16u * lane, word(0), word(1), word(2), word(3));
    } else if (FORM == ScaleForm::kRows) {
      uint32_t w[4];
#pragma unroll
      for (int q = 0; q < 4; ++q)
        w[q] = __funnelshift_r(x[3 * q + g], x[3 * q + g + 1], 8u * offset(O.s + (row0 + lane + 32 * q) * O.s_row + block0));
      st_shared_v4(dst + 16u * lane, w[0], w[1], w[2], w[3]);
    } else {
      uint32_t v[4];
#pragma unroll
      for (int b = 0; b < 4; ++b)
        v[b] = __funnelshift_r(x[2 * (4 * g + b)], x[2 * (4 * g + b) + 1], 8u * offset(O.s + (block0 + 4 * g + b) * O.s_k + row0 + 4 * lane));
      const uint32_t t0 = __byte_perm(v[0], v[1], 0x5140), t1 = __byte_perm(v[2], v[3], 0x5140);
      const uint32_t t2 = __byte_perm(v[0], v[1], 0x7362), t3 = __byte_perm(v[2], v[3], 0x7362);
      const uint32_t at = dst + 16u * ((4 * lane) & 31) + 4u * (lane >> 3);
      asm volatile("st.shared.b32 [%0], %1;" ::"r"(at), "r"(__byte_perm(t0, t1, 0x5410)));
      asm volatile("st.shared.b32 [%0], %1;" ::"r"(at + 16u), "r"(__byte_perm(t0, t1, 0x7632)));
      asm volatile("st.shared.b32 [%0], %1;" ::"r"(at + 32u), "r"(__byte_perm(t2, t3, 0x5410)));
      asm volatile("st.shared.b32 [%0], %1;" ::"r"(at + 48u), "r"(__byte_perm(t2, t3, 0x7632)));
    }
  }
};
// Forms of the two operands by the product: linear and input (activations, weight), weight (both along the tokens).
template <bool kAMn>
using ScalesA = Scales<kAMn ? ScaleForm::kColumns : ScaleForm::kRows>;
template <bool kAMn>
using ScalesB = Scales<kAMn ? ScaleForm::kColumns : ScaleForm::kTiles>;

// 512 bytes of scales (32 rows of 16 bytes: no swizzle, groups of eight rows 128 bytes apart) to four columns of tensor memory,
// for all four quarters of its lanes.
__device__ __forceinline__ uint64_t scale_desc(uint32_t smem_addr) {
  return static_cast<uint64_t>((smem_addr & 0x3ffff) >> 4) | (static_cast<uint64_t>(1) << 16) | (static_cast<uint64_t>(128 >> 4) << 32) |
         (static_cast<uint64_t>(1) << 46);
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

// Mask flags of eight outputs, a byte each.
template <class PARAMS>
__device__ __forceinline__ uint2 output_flags(const PARAMS& P, int r, int n) {
  if (r >= P.A.rows || n >= P.B.rows) return make_uint2(0u, 0u);
  const uint8_t* f = P.keep + static_cast<size_t>(r / P.block) * P.B.rows + n;
  if (P.keep_wide) return ld_global(reinterpret_cast<const uint2*>(f));            // (then the output's width is a multiple of 8)
  uint2 k = make_uint2(0u, 0u);
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (n + e < P.B.rows) (e < 4 ? k.x : k.y) |= static_cast<uint32_t>(ld_global(f + e)) << (8 * (e & 3));
  return k;
}

// Rows of a copy of up to `most` rows: no more than the matrix has, in whole groups of eight.  (What no copy writes are rows of outputs that do not
// exist.)  Rows of a box behind the last one are not free: 4096 x 4096 with 31 tokens took 9.7 to 12.5 us with boxes of 128 rows.
inline int box_rows(int rows, int most) { return rows >= most ? most : (rows + 7) / 8 * 8; }
// 8-bit matrix [outer, inner], boxes of 128 x box_outer, 128-byte swizzle; what lies outside reads as zero.
inline bool make_map8(CUtensorMap* map, const void* base, uint64_t inner, uint64_t outer, uint64_t ld, uint32_t box_outer) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {inner, outer};
  const cuuint64_t strides[1] = {ld};
  const cuuint32_t box[2] = {kBlock, box_outer};
  const cuuint32_t elem[2] = {1, 1};
  auto encode = [&] {
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  };
  if (encode()) return true;
  int device = 0;            // (a thread without a current context: see make_map)
  return cudaGetDevice(&device) == cudaSuccess && cudaSetDevice(device) == cudaSuccess && encode();
}

// bsp_gemm_fp8_split.cu: tiles of 128 x 64, the contraction of each shared by a cluster of c CTAs (1, 2, 4 or 8).
int choose_split(const Product& p, const TcDevice& dev, double* us);
int launch_split(const Product& p, int c, TcDevice* dev, cudaStream_t s);

}  // namespace fp8
}  // namespace bsp
