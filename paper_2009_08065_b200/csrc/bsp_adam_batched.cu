// bsp_masked_adam_step_batched: Algorithm 2's retraining step (Adam, then W = W * Mask) on many tensors in one launch, the
// moments in 32 or in 8 bits.
//
// 8-bit moments: m in e4m3, v in e5m2, a power-of-two scale for each 128 neighbouring weights of a row (bsp_fp8.cuh).  The new
// moments are rounded stochastically: with beta2 = 0.999 a step changes v by a thousandth, far less than half a step of two or
// three mantissa bits, and a moment rounded to the nearest value would never move again; with probabilities by distance it is
// right on average.  The random bits are a hash of seed, step, tensor and position, so a step can be repeated bit for bit.  A
// positive v stays positive (the smallest value instead of zero): m / (sqrt(0) + eps) would be a step of any size.  W is
// updated from the moments before they are rounded.
//
// HBM-bound.  Bytes per weight with a bf16 gradient: 8 bits 2 + 8 + 4 + 2 = 16, 32 bits 2 + 8 + 16 + 2 = 28.  Sixteen threads
// share a block of 128 weights, eight neighbouring ones each: 16-byte accesses, and the block's largest moments are a
// reduction over half a warp.
#include <math.h>

#include "bsp_fp8.cuh"

namespace bsp {
using namespace fp8;

namespace {

constexpr int kAdamThreads = 256;
constexpr int kAdamGroups = kAdamThreads / 16;     // blocks of 128 weights per CTA
constexpr int kAdamMaxJobs = 96;                   // per launch; the table travels as a kernel parameter

struct AdamJob {
  float* W;
  const void* G;
  void *M, *V;
  uint8_t *ms, *vs;
  const uint8_t* keep;
  uint16_t* Wb;
  int rows, cols, ldw, ldg, ldm, ldb;
  int block, orient;
  float lr, decay;
  uint32_t tensor;           // its number in the call's array, for the random bits
  uint8_t bits8, grad16, wide, keep_wide;
};
struct AdamTable {
  AdamJob job[kAdamMaxJobs];
  int first[kAdamMaxJobs + 1];                     // CTA at which a job begins
  int n_jobs;
  float beta1, beta2, eps;
  float inv_c1, inv_c2, log_beta1, log_beta2;      // 1 / (1 - beta^step); natural logarithms for a step that the device holds
  uint32_t seed;
  int step;
  const int* step_dev;
  const float* grad_scale;
};

// The random bits of a weight: multiplications by odd constants (the fractions of 2^(1/2) and 3^(1/2)) between shifts that
// bring the upper half down.
__device__ __forceinline__ uint32_t mix(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x6A09E667u;
  x = (x ^ (x >> 15)) * 0xBB67AE85u;
  return x ^ (x >> 16);
}
// y (finite, not negative, in the format's range) to one of its two neighbours in the format, given 16 random bits: they are
// added at the upper end of what is then cut off.  Below the smallest normal value steps are as wide as just above it, so that
// value is added first and taken off again.
template <int FMT>
__device__ __forceinline__ float round_randomly(float y, uint32_t random16) {
  constexpr int kDrop = FMT == BSP_FP8_E4M3 ? 20 : 21;
  constexpr float kLow = FMT == BSP_FP8_E4M3 ? 0x1p-6f : 0x1p-14f;
  const float add = y < kLow ? kLow : 0.0f;
  const uint32_t z = __float_as_uint(__fadd_rn(y, add)) + (random16 << (kDrop - 16));
  return __uint_as_float(z & ~((1u << kDrop) - 1u)) - add;
}

__device__ __forceinline__ void load8(const float* p, float (&f)[8]) {
  const float4 a = ld_global(reinterpret_cast<const float4*>(p)), b = ld_global(reinterpret_cast<const float4*>(p) + 1);
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ void store8(float* p, const float (&f)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
template <int FMT>
__device__ __forceinline__ void decode8(uint2 q, float scale, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    from_fp8x2<FMT>((i < 2 ? q.x : q.y) >> (16 * (i & 1)), f[2 * i], f[2 * i + 1]);
    f[2 * i] *= scale;
    f[2 * i + 1] *= scale;
  }
}

__global__ void __launch_bounds__(kAdamThreads)
adam_batched_kernel(const __grid_constant__ AdamTable T) {
  // the job of this CTA
  int lo = 0, hi = T.n_jobs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (T.first[mid] <= static_cast<int>(blockIdx.x)) lo = mid;
    else hi = mid - 1;
  }
  const AdamJob& J = T.job[lo];
  const uint32_t l = threadIdx.x & 15u;
  const uint32_t kb = static_cast<uint32_t>(blocks_of(J.cols));
  const unsigned long long group = static_cast<unsigned long long>(blockIdx.x - T.first[lo]) * kAdamGroups + (threadIdx.x >> 4);
  const uint32_t r = group < 0xffffffffull ? static_cast<uint32_t>(group) / kb : static_cast<uint32_t>(group / kb);
  const uint32_t b = static_cast<uint32_t>(group - static_cast<unsigned long long>(r) * kb);
  const int c = static_cast<int>(b * kBlock + 8u * l);
  const int n = r < static_cast<uint32_t>(J.rows) ? min(8, J.cols - c) : 0;
  const bool wide = J.wide != 0 && n == 8;
  pdl_wait();
  pdl_launch_dependents();

  const size_t iw = static_cast<size_t>(r) * J.ldw + c, ig = static_cast<size_t>(r) * J.ldg + c, im = static_cast<size_t>(r) * J.ldm + c;
  const size_t is = static_cast<size_t>(r) * kb + b;
  float w[8], g[8], m[8], v[8];
  uint32_t keep = 0xffu;                           // one bit per weight
  uint32_t byte_m = 127u, byte_v = 127u;
  uint2 q_m = make_uint2(0u, 0u), q_v = make_uint2(0u, 0u);
  if (J.bits8 && n > 0) {
    byte_m = ld_global(J.ms + is);
    byte_v = ld_global(J.vs + is);
  }
  if (wide) {
    load8(J.W + iw, w);
    if (J.grad16) {
      const uint4 h = ld_global(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(J.G) + ig));
      const uint32_t hw[4] = {h.x, h.y, h.z, h.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) { g[2 * i] = __uint_as_float(hw[i] << 16); g[2 * i + 1] = __uint_as_float(hw[i] & 0xffff0000u); }
    } else {
      load8(static_cast<const float*>(J.G) + ig, g);
    }
    if (J.bits8) {
      q_m = ld_global(reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(J.M) + im));
      q_v = ld_global(reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(J.V) + im));
    } else {
      load8(static_cast<const float*>(J.M) + im, m);
      load8(static_cast<const float*>(J.V) + im, v);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[i] = g[i] = m[i] = v[i] = 0.0f;
      if (i < n) {
        w[i] = ld_global(J.W + iw + i);
        g[i] = J.grad16 ? bf16_bits_to_float(ld_global(static_cast<const uint16_t*>(J.G) + ig + i)) : ld_global(static_cast<const float*>(J.G) + ig + i);
        if (J.bits8) {
          const uint32_t a = ld_global(static_cast<const uint8_t*>(J.M) + im + i), e = ld_global(static_cast<const uint8_t*>(J.V) + im + i);
          (i < 4 ? q_m.x : q_m.y) |= a << (8 * (i & 3));
          (i < 4 ? q_v.x : q_v.y) |= e << (8 * (i & 3));
        } else {
          m[i] = ld_global(static_cast<const float*>(J.M) + im + i);
          v[i] = ld_global(static_cast<const float*>(J.V) + im + i);
        }
      }
    }
  }
  if (J.keep != nullptr && n > 0) {
    if (J.orient == BSP_ORIENT_C) {
      const uint8_t* f = J.keep + static_cast<size_t>(r / static_cast<uint32_t>(J.block)) * J.cols + c;
      if (J.keep_wide && n == 8) {
        const uint2 k = ld_global(reinterpret_cast<const uint2*>(f));
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if ((((i < 4 ? k.x : k.y) >> (8 * (i & 3))) & 0xffu) == 0u) keep &= ~(1u << i);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < n && ld_global(f + i) == 0) keep &= ~(1u << i);
      }
    } else {
      const uint8_t* f = J.keep + static_cast<size_t>(r) * (J.cols / J.block);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < n && ld_global(f + (c + i) / J.block) == 0) keep &= ~(1u << i);
    }
  }
  const float gs = T.grad_scale != nullptr ? ld_global(T.grad_scale) : 1.0f;
  int step = T.step;
  float i1 = T.inv_c1, i2 = T.inv_c2;
  if (T.step_dev != nullptr) {
    step = ld_global(T.step_dev);
    i1 = 1.0f / -expm1f(static_cast<float>(step) * T.log_beta1);
    i2 = 1.0f / -expm1f(static_cast<float>(step) * T.log_beta2);
  }
  if (J.bits8) {
    decode8<BSP_FP8_E4M3>(q_m, scale_value(byte_m), m);
    decode8<BSP_FP8_E5M2>(q_v, scale_value(byte_v), v);
  }
  // The moments' roundings are spelled out: one behind product and sum.  8-bit values follow the last bit.
  const float c1 = 1.0f - T.beta1, c2 = 1.0f - T.beta2;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (T.grad_scale != nullptr) g[i] = __fmul_rn(g[i], gs);
    m[i] = __fmaf_rn(T.beta1, m[i], __fmul_rn(c1, g[i]));
    v[i] = __fmaf_rn(T.beta2, v[i], __fmul_rn(__fmul_rn(c2, g[i]), g[i]));
    const float mhat = m[i] * i1, vhat = v[i] * i2;
    const float upd = __fdiv_rn(mhat, __fsqrt_rn(vhat) + T.eps) + J.decay * w[i];
    w[i] = (keep >> i) & 1u ? __fmaf_rn(-J.lr, upd, w[i]) : 0.0f;
  }
  if (J.bits8) {
    uint32_t top_m = 0u, top_v = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      top_m = max(top_m, __float_as_uint(m[i]) & 0x7fffffffu);
      top_v = max(top_v, __float_as_uint(v[i]) & 0x7fffffffu);
    }
    const uint32_t lanes = 0xffffu << (threadIdx.x & 16u);
    top_m = __reduce_max_sync(lanes, top_m);
    top_v = __reduce_max_sync(lanes, top_v);
    const bool bad_m = top_m >= 0x7f800000u, bad_v = top_v >= 0x7f800000u;   // then the block is NaN throughout, under scale 1
    const int new_m = bad_m ? 127 : scale_byte(top_m, top_of(BSP_FP8_E4M3)), new_v = bad_v ? 127 : scale_byte(top_v, top_of(BSP_FP8_E5M2));
    const float inv_m = scale_inverse(new_m), inv_v = scale_inverse(new_v);
    const uint32_t at = r * static_cast<uint32_t>(J.cols) + static_cast<uint32_t>(c);
    const uint32_t key = mix(T.seed + 0x9E3779B9u * static_cast<uint32_t>(step) + 0xBB67AE85u * J.tensor);
    q_m = q_v = make_uint2(kNan * 0x01010101u, kNan * 0x01010101u);
    float rm[8], rv[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t h = mix(at + static_cast<uint32_t>(i) + key);
      rm[i] = copysignf(round_randomly<BSP_FP8_E4M3>(fabsf(m[i]) * inv_m, h & 0xffffu), m[i]);
      const float y = v[i] * inv_v;
      rv[i] = fmaxf(round_randomly<BSP_FP8_E5M2>(y, h >> 16), v[i] > 0.0f ? 0x1p-16f : 0.0f);
    }
    if (!bad_m) q_m = make_uint2(to_fp8x2<BSP_FP8_E4M3>(rm[0], rm[1]) | (to_fp8x2<BSP_FP8_E4M3>(rm[2], rm[3]) << 16),
                                 to_fp8x2<BSP_FP8_E4M3>(rm[4], rm[5]) | (to_fp8x2<BSP_FP8_E4M3>(rm[6], rm[7]) << 16));
    if (!bad_v) q_v = make_uint2(to_fp8x2<BSP_FP8_E5M2>(rv[0], rv[1]) | (to_fp8x2<BSP_FP8_E5M2>(rv[2], rv[3]) << 16),
                                 to_fp8x2<BSP_FP8_E5M2>(rv[4], rv[5]) | (to_fp8x2<BSP_FP8_E5M2>(rv[6], rv[7]) << 16));
    if (l == 0 && n > 0) {
      J.ms[is] = static_cast<uint8_t>(new_m);
      J.vs[is] = static_cast<uint8_t>(new_v);
    }
  }
  uint32_t half[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(half[i]) : "f"(w[2 * i + 1]), "f"(w[2 * i]));
  uint16_t* wb = J.Wb != nullptr ? J.Wb + static_cast<size_t>(r) * J.ldb + c : nullptr;
  if (wide) {
    store8(J.W + iw, w);
    if (J.bits8) {
      *reinterpret_cast<uint2*>(static_cast<uint8_t*>(J.M) + im) = q_m;
      *reinterpret_cast<uint2*>(static_cast<uint8_t*>(J.V) + im) = q_v;
    } else {
      store8(static_cast<float*>(J.M) + im, m);
      store8(static_cast<float*>(J.V) + im, v);
    }
    if (wb != nullptr) *reinterpret_cast<uint4*>(wb) = make_uint4(half[0], half[1], half[2], half[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i < n) {
        J.W[iw + i] = w[i];
        if (J.bits8) {
          static_cast<uint8_t*>(J.M)[im + i] = static_cast<uint8_t>((i < 4 ? q_m.x : q_m.y) >> (8 * (i & 3)));
          static_cast<uint8_t*>(J.V)[im + i] = static_cast<uint8_t>((i < 4 ? q_v.x : q_v.y) >> (8 * (i & 3)));
        } else {
          static_cast<float*>(J.M)[im + i] = m[i];
          static_cast<float*>(J.V)[im + i] = v[i];
        }
        if (wb != nullptr) wb[i] = static_cast<uint16_t>(half[i >> 1] >> (16 * (i & 1)));
      }
    }
  }
}

// Checks one job and fills its entry; *ctas receives what it needs.
int make_job(const bsp_adam_job& a, uint32_t tensor, AdamJob* j, long long* ctas) {
  if (a.W == nullptr || a.grad == nullptr || a.m == nullptr || a.v == nullptr || a.rows <= 0 || a.cols <= 0) return BSP_ERR_ARG;
  if (a.state_bits != 8 && a.state_bits != 32) return BSP_ERR_ARG;
  if (a.grad_type != BSP_GRAD_F32 && a.grad_type != BSP_GRAD_BF16) return BSP_ERR_ARG;
  if (a.state_bits == 8 && (a.m_scale == nullptr || a.v_scale == nullptr)) return BSP_ERR_ARG;
  if (!(a.lr == a.lr) || !(a.weight_decay == a.weight_decay)) return BSP_ERR_ARG;
  if (a.ldw < a.cols || a.ldg < a.cols || a.ldm < a.cols || (a.W_bf16 != nullptr && a.ldb < a.cols)) return BSP_ERR_SHAPE;
  if (a.keep != nullptr) {
    if (a.block <= 0 || (a.orient != BSP_ORIENT_C && a.orient != BSP_ORIENT_R)) return BSP_ERR_ARG;
    int nb, ng;
    if (!geometry(a.rows, a.cols, a.block, a.orient, &nb, &ng)) return BSP_ERR_SHAPE;
  }
  const bool bits8 = a.state_bits == 8, grad16 = a.grad_type == BSP_GRAD_BF16;
  const size_t state_align = bits8 ? 1 : 4;
  if (!aligned_to(a.W, 4) || !aligned_to(a.grad, grad16 ? 2 : 4) || !aligned_to(a.m, state_align) || !aligned_to(a.v, state_align) ||
      (a.W_bf16 != nullptr && !aligned_to(a.W_bf16, 2)))
    return BSP_ERR_ARG;
  j->W = a.W; j->G = a.grad; j->M = a.m; j->V = a.v; j->ms = a.m_scale; j->vs = a.v_scale;
  j->keep = a.keep; j->Wb = static_cast<uint16_t*>(a.W_bf16);
  j->rows = a.rows; j->cols = a.cols; j->ldw = a.ldw; j->ldg = a.ldg; j->ldm = a.ldm; j->ldb = a.ldb;
  j->block = a.keep != nullptr ? a.block : 1; j->orient = a.orient;
  j->lr = a.lr; j->decay = a.weight_decay;
  j->tensor = tensor;
  j->bits8 = bits8; j->grad16 = grad16;
  j->wide = aligned_to(a.W, 16) && a.ldw % 4 == 0 && aligned_to(a.grad, 16) && a.ldg % (grad16 ? 8 : 4) == 0 && aligned_to(a.m, bits8 ? 8 : 16) &&
            aligned_to(a.v, bits8 ? 8 : 16) && a.ldm % (bits8 ? 8 : 4) == 0 && (a.W_bf16 == nullptr || (aligned_to(a.W_bf16, 16) && a.ldb % 8 == 0));
  j->keep_wide = aligned_to(a.keep, 8) && a.cols % 8 == 0;
  const long long groups = static_cast<long long>(a.rows) * blocks_of(a.cols);
  *ctas = (groups + kAdamGroups - 1) / kAdamGroups;
  return *ctas > 0x3fffffffLL ? BSP_ERR_UNSUPPORTED : BSP_OK;
}

}  // namespace
}  // namespace bsp

extern "C" int bsp_masked_adam_step_batched(const bsp_adam_job* jobs, int n_jobs, float beta1, float beta2, float eps, int step, uint32_t seed,
                                            const float* grad_scale, const int* step_dev, void* stream) {
  using namespace bsp;
  if (jobs == nullptr || n_jobs <= 0) return BSP_ERR_ARG;
  if (!(beta1 >= 0.0f && beta1 < 1.0f) || !(beta2 >= 0.0f && beta2 < 1.0f) || !(eps >= 0.0f)) return BSP_ERR_ARG;
  if (step_dev == nullptr && step < 1) return BSP_ERR_ARG;
  if (!aligned_to(grad_scale, 4) || !aligned_to(step_dev, 4)) return BSP_ERR_ARG;
  AdamTable T;
  for (int i = 0; i < n_jobs; ++i) {                  // all jobs are checked before the first launch
    long long ctas;
    BSP_TRY(make_job(jobs[i], static_cast<uint32_t>(i), &T.job[0], &ctas));
  }
  T.beta1 = beta1; T.beta2 = beta2; T.eps = eps;
  T.inv_c1 = T.inv_c2 = 0.0f;
  if (step_dev == nullptr) {                          // bias corrections in double on the host, rounded once
    T.inv_c1 = static_cast<float>(1.0 / (1.0 - pow(static_cast<double>(beta1), step)));
    T.inv_c2 = static_cast<float>(1.0 / (1.0 - pow(static_cast<double>(beta2), step)));
  }
  T.log_beta1 = static_cast<float>(log(static_cast<double>(beta1)));
  T.log_beta2 = static_cast<float>(log(static_cast<double>(beta2)));
  T.seed = seed; T.step = step; T.step_dev = step_dev; T.grad_scale = grad_scale;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  for (int i = 0; i < n_jobs;) {
    long long total = 0;
    T.n_jobs = 0;
    while (i < n_jobs && T.n_jobs < kAdamMaxJobs) {
      long long ctas;
      BSP_TRY(make_job(jobs[i], static_cast<uint32_t>(i), &T.job[T.n_jobs], &ctas));
      if (T.n_jobs > 0 && total + ctas > 0x7fffffffLL) break;
      T.first[T.n_jobs++] = static_cast<int>(total);
      total += ctas;
      ++i;
    }
    T.first[T.n_jobs] = static_cast<int>(total);
    BSP_CUDA_TRY(launch_pdl(adam_batched_kernel, dim3(static_cast<unsigned>(total)), dim3(kAdamThreads), 0, s, T));
  }
  return BSP_OK;
}
