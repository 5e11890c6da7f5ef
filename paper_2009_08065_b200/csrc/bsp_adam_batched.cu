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
#include <float.h>
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
  uint8_t grad16, wide, keep_wide;
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
__device__ __forceinline__ void load8(const float* p, float (&f)[8]) {
  const float4 a = ld_global(reinterpret_cast<const float4*>(p)), b = ld_global(reinterpret_cast<const float4*>(p) + 1);
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ void store8(float* p, const float (&f)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
// Two neighbouring values as a register pair, for the packed float32 operations (each half rounds as the single operation does).
struct Pair {
  unsigned long long v;
};
__device__ __forceinline__ Pair pair_of(float lo, float hi) {
  Pair p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p.v) : "f"(lo), "f"(hi));
  return p;
}
__device__ __forceinline__ Pair pair_of(float x) { return pair_of(x, x); }
__device__ __forceinline__ void split(Pair p, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p.v)); }
__device__ __forceinline__ Pair mul(Pair a, Pair b) {
  Pair d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
  return d;
}
__device__ __forceinline__ Pair add(Pair a, Pair b) {
  Pair d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
  return d;
}
__device__ __forceinline__ Pair fma(Pair a, Pair b, Pair c) {
  Pair d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return d;
}

// Two magnitudes (not negative, in the format's range) to one of their two neighbours in the format: random bits are added at
// the upper end of what is then cut off (r: 16 of them, already at their place).  Below the smallest normal value steps are as
// wide as just above it, so that value is added first and taken off again.
template <int FMT>
__device__ __forceinline__ Pair round_pair(float y0, float y1, uint32_t r0, uint32_t r1) {
  constexpr uint32_t kKeep = ~((1u << (FMT == BSP_FP8_E4M3 ? 20 : 21)) - 1u);
  constexpr float kLow = FMT == BSP_FP8_E4M3 ? 0x1p-6f : 0x1p-14f;
  const float a0 = y0 < kLow ? kLow : 0.0f, a1 = y1 < kLow ? kLow : 0.0f;
  const Pair low = pair_of(a0, a1);
  float z0, z1;
  split(add(pair_of(y0, y1), low), z0, z1);
  const Pair cut = pair_of(__uint_as_float((__float_as_uint(z0) + r0) & kKeep), __uint_as_float((__float_as_uint(z1) + r1) & kKeep));
  return fma(low, pair_of(-1.0f), cut);
}

// Eight neighbouring weights: what the kernels for both kinds of moments share.
struct Place {
  int c, n;                  // first column, how many of the eight exist
  uint32_t r, b;             // row, block of 128
  size_t iw, ig, im, is;
  bool wide;
};
__device__ __forceinline__ const AdamJob& find_job(const AdamTable& T, Place& p) {
  int lo = 0, hi = T.n_jobs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (T.first[mid] <= static_cast<int>(blockIdx.x)) lo = mid;
    else hi = mid - 1;
  }
  const AdamJob& J = T.job[lo];
  const uint32_t kb = static_cast<uint32_t>(blocks_of(J.cols));
  const unsigned long long group = static_cast<unsigned long long>(blockIdx.x - T.first[lo]) * kAdamGroups + (threadIdx.x >> 4);
  p.r = group < 0xffffffffull ? static_cast<uint32_t>(group) / kb : static_cast<uint32_t>(group / kb);
  p.b = static_cast<uint32_t>(group - static_cast<unsigned long long>(p.r) * kb);
  p.c = static_cast<int>(p.b * kBlock + 8u * (threadIdx.x & 15u));
  p.n = p.r < static_cast<uint32_t>(J.rows) ? max(0, min(8, J.cols - p.c)) : 0;
  p.wide = J.wide != 0 && p.n == 8;
  p.iw = static_cast<size_t>(p.r) * J.ldw + p.c;
  p.ig = static_cast<size_t>(p.r) * J.ldg + p.c;
  p.im = static_cast<size_t>(p.r) * J.ldm + p.c;
  p.is = static_cast<size_t>(p.r) * kb + p.b;
  return J;
}
__device__ __forceinline__ void load_weights(const AdamJob& J, const Place& p, float (&w)[8], float (&g)[8]) {
  if (p.wide) {
    load8(J.W + p.iw, w);
    if (J.grad16) {
      const uint4 h = ld_global(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(J.G) + p.ig));
      const uint32_t hw[4] = {h.x, h.y, h.z, h.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) { g[2 * i] = __uint_as_float(hw[i] << 16); g[2 * i + 1] = __uint_as_float(hw[i] & 0xffff0000u); }
    } else {
      load8(static_cast<const float*>(J.G) + p.ig, g);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[i] = g[i] = 0.0f;
      if (i < p.n) {
        w[i] = ld_global(J.W + p.iw + i);
        g[i] = J.grad16 ? bf16_bits_to_float(ld_global(static_cast<const uint16_t*>(J.G) + p.ig + i)) : ld_global(static_cast<const float*>(J.G) + p.ig + i);
      }
    }
  }
}
// A byte for each weight, zero where it is pruned.
__device__ __forceinline__ uint2 load_flags(const AdamJob& J, const Place& p) {
  uint2 k = make_uint2(0xffffffffu, 0xffffffffu);
  if (J.keep == nullptr || p.n == 0) return k;
  if (J.orient == BSP_ORIENT_C) {
    const uint8_t* f = J.keep + static_cast<size_t>(p.r / static_cast<uint32_t>(J.block)) * J.cols + p.c;
    if (J.keep_wide && p.n == 8) return ld_global(reinterpret_cast<const uint2*>(f));
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < p.n && ld_global(f + i) == 0) (i < 4 ? k.x : k.y) &= ~(0xffu << (8 * (i & 3)));
  } else {
    const uint8_t* f = J.keep + static_cast<size_t>(p.r) * (J.cols / J.block);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < p.n && ld_global(f + (p.c + i) / J.block) == 0) (i < 4 ? k.x : k.y) &= ~(0xffu << (8 * (i & 3)));
  }
  return k;
}
__device__ __forceinline__ bool kept(uint2 k, int i) { return ((i < 4 ? k.x : k.y) & (0xffu << (8 * (i & 3)))) != 0u; }
__device__ __forceinline__ void store_weights(const AdamJob& J, const Place& p, const float (&w)[8]) {
  uint32_t half[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(half[i]) : "f"(w[2 * i + 1]), "f"(w[2 * i]));
  uint16_t* wb = J.Wb != nullptr ? J.Wb + static_cast<size_t>(p.r) * J.ldb + p.c : nullptr;
  if (p.wide) {
    store8(J.W + p.iw, w);
    if (wb != nullptr) *reinterpret_cast<uint4*>(wb) = make_uint4(half[0], half[1], half[2], half[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i < p.n) {
        J.W[p.iw + i] = w[i];
        if (wb != nullptr) wb[i] = static_cast<uint16_t>(half[i >> 1] >> (16 * (i & 1)));
      }
    }
  }
}
// Step number and bias corrections.
__device__ __forceinline__ int corrections(const AdamTable& T, float& i1, float& i2) {
  i1 = T.inv_c1;
  i2 = T.inv_c2;
  if (T.step_dev == nullptr) return T.step;
  const int step = ld_global(T.step_dev);
  i1 = 1.0f / -expm1f(static_cast<float>(step) * T.log_beta1);
  i2 = 1.0f / -expm1f(static_cast<float>(step) * T.log_beta2);
  return step;
}

// 32-bit moments: the operations of bsp_masked_adam_step, in its order.
__global__ void __launch_bounds__(kAdamThreads)
adam_batched_kernel(const __grid_constant__ AdamTable T) {
  Place p;
  const AdamJob& J = find_job(T, p);
  pdl_wait();
  pdl_launch_dependents();
  float w[8], g[8], m[8], v[8];
  load_weights(J, p, w, g);
  float *M = static_cast<float*>(J.M) + p.im, *V = static_cast<float*>(J.V) + p.im;
  if (p.wide) {
    load8(M, m);
    load8(V, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      m[i] = i < p.n ? ld_global(M + i) : 0.0f;
      v[i] = i < p.n ? ld_global(V + i) : 0.0f;
    }
  }
  const uint2 keep = load_flags(J, p);
  float i1, i2;
  corrections(T, i1, i2);
  const float gs = T.grad_scale != nullptr ? ld_global(T.grad_scale) : 1.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float gi = __fmul_rn(g[i], gs);
    m[i] = __fmaf_rn(T.beta1, m[i], __fmul_rn(1.0f - T.beta1, gi));
    v[i] = __fmaf_rn(T.beta2, v[i], __fmul_rn(__fmul_rn(1.0f - T.beta2, gi), gi));
    const float upd = __fdiv_rn(m[i] * i1, __fsqrt_rn(v[i] * i2) + T.eps) + J.decay * w[i];
    w[i] = kept(keep, i) ? __fmaf_rn(-J.lr, upd, w[i]) : 0.0f;
  }
  if (p.wide) {
    store8(M, m);
    store8(V, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i < p.n) {
        M[i] = m[i];
        V[i] = v[i];
      }
    }
  }
  store_weights(J, p, w);
}

// 8-bit moments.  What bounds this one is instruction issue as much as HBM (16 bytes per weight leave 90 issue slots for a
// warp's 32 weights), hence packed float32 operations, and the hardware's approximate square root and reciprocal (each within about a place) for
// the update of W; the moments, which the 8-bit values follow to the last bit, are rounded as defined.
__global__ void __launch_bounds__(kAdamThreads)
adam_batched8_kernel(const __grid_constant__ AdamTable T) {
  Place p;
  const AdamJob& J = find_job(T, p);
  pdl_wait();
  pdl_launch_dependents();
  float w[8], g[8];
  load_weights(J, p, w, g);
  uint32_t byte_m = 127u, byte_v = 127u;
  uint2 q_m = make_uint2(0u, 0u), q_v = make_uint2(0u, 0u);
  uint8_t *M = static_cast<uint8_t*>(J.M) + p.im, *V = static_cast<uint8_t*>(J.V) + p.im;
  if (p.n > 0) {
    byte_m = ld_global(J.ms + p.is);
    byte_v = ld_global(J.vs + p.is);
  }
  if (p.wide) {
    q_m = ld_global(reinterpret_cast<const uint2*>(M));
    q_v = ld_global(reinterpret_cast<const uint2*>(V));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i < p.n) {
        (i < 4 ? q_m.x : q_m.y) |= static_cast<uint32_t>(ld_global(M + i)) << (8 * (i & 3));
        (i < 4 ? q_v.x : q_v.y) |= static_cast<uint32_t>(ld_global(V + i)) << (8 * (i & 3));
      }
    }
  }
  const uint2 keep = load_flags(J, p);
  float i1, i2;
  const int step = corrections(T, i1, i2);
  const Pair gs = pair_of(T.grad_scale != nullptr ? ld_global(T.grad_scale) : 1.0f);
  const Pair b1 = pair_of(T.beta1), b2 = pair_of(T.beta2), c1 = pair_of(1.0f - T.beta1), c2 = pair_of(1.0f - T.beta2);
  const Pair p1 = pair_of(i1), p2 = pair_of(i2), eps = pair_of(T.eps), lr = pair_of(-J.lr), decay = pair_of(J.decay);
  const Pair scale_m = pair_of(scale_value(byte_m)), scale_v = pair_of(scale_value(byte_v));
  float m[8], v[8];
  uint32_t top_m = 0u, top_v = 0u;
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    float lo, hi;
    const Pair gi = mul(pair_of(g[i], g[i + 1]), gs);
    from_fp8x2<BSP_FP8_E4M3>((i < 4 ? q_m.x : q_m.y) >> (8 * (i & 2)), lo, hi);
    const Pair mi = fma(b1, mul(pair_of(lo, hi), scale_m), mul(c1, gi));
    from_fp8x2<BSP_FP8_E5M2>((i < 4 ? q_v.x : q_v.y) >> (8 * (i & 2)), lo, hi);
    const Pair vi = fma(b2, mul(pair_of(lo, hi), scale_v), mul(mul(c2, gi), gi));
    split(mi, m[i], m[i + 1]);
    split(vi, v[i], v[i + 1]);
    top_m = max(top_m, max(__float_as_uint(m[i]) & 0x7fffffffu, __float_as_uint(m[i + 1]) & 0x7fffffffu));
    top_v = max(top_v, max(__float_as_uint(v[i]) & 0x7fffffffu, __float_as_uint(v[i + 1]) & 0x7fffffffu));
    split(mul(vi, p2), lo, hi);
    asm("sqrt.approx.f32 %0, %0;" : "+f"(lo));
    asm("sqrt.approx.f32 %0, %0;" : "+f"(hi));
    split(add(pair_of(lo, hi), eps), lo, hi);
    const Pair wi = pair_of(w[i], w[i + 1]);
    const Pair upd = fma(mul(mi, p1), pair_of(reciprocal(lo), reciprocal(hi)), mul(decay, wi));
    split(fma(lr, upd, wi), lo, hi);
    w[i] = kept(keep, i) ? lo : 0.0f;
    w[i + 1] = kept(keep, i + 1) ? hi : 0.0f;
  }
  store_weights(J, p, w);
  const uint32_t lanes = 0xffffu << (threadIdx.x & 16u);
  top_m = __reduce_max_sync(lanes, top_m);
  top_v = __reduce_max_sync(lanes, top_v);
  // a block with an infinity or a NaN becomes NaN throughout (the multiplier makes every value one), under scale 1
  const bool bad_m = top_m >= 0x7f800000u, bad_v = top_v >= 0x7f800000u;
  const int new_m = bad_m ? 127 : scale_byte(top_m, top_of(BSP_FP8_E4M3)), new_v = bad_v ? 127 : scale_byte(top_v, top_of(BSP_FP8_E5M2));
  const Pair inv_m = pair_of(scale_inverse(new_m)), inv_v = pair_of(scale_inverse(new_v));
  const uint32_t key = mix(T.seed + 0x9E3779B9u * static_cast<uint32_t>(step) + 0xBB67AE85u * J.tensor);
  const uint32_t at = p.r * static_cast<uint32_t>(J.cols) + static_cast<uint32_t>(p.c) + key;
  uint32_t out_m[4], out_v[4];
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const uint32_t h0 = mix(at + static_cast<uint32_t>(i)), h1 = mix(at + static_cast<uint32_t>(i + 1));
    float lo, hi;
    split(mul(pair_of(fabsf(m[i]), fabsf(m[i + 1])), inv_m), lo, hi);
    split(round_pair<BSP_FP8_E4M3>(lo, hi, (h0 << 4) & 0xffff0u, (h1 << 4) & 0xffff0u), lo, hi);
    out_m[i >> 1] = to_fp8x2<BSP_FP8_E4M3>(copysignf(lo, m[i]), copysignf(hi, m[i + 1]));
    // (a positive value below the smallest one becomes that, which random bits leave as it is)
    split(mul(pair_of(v[i], v[i + 1]), inv_v), lo, hi);
    lo = v[i] > 0.0f ? fmaxf(lo, 0x1p-16f) : 0.0f;
    hi = v[i + 1] > 0.0f ? fmaxf(hi, 0x1p-16f) : 0.0f;
    split(round_pair<BSP_FP8_E5M2>(lo, hi, (h0 >> 11) & 0x1fffe0u, (h1 >> 11) & 0x1fffe0u), lo, hi);
    out_v[i >> 1] = to_fp8x2<BSP_FP8_E5M2>(lo, hi);
  }
  q_m = make_uint2(out_m[0] | (out_m[1] << 16), out_m[2] | (out_m[3] << 16));
  q_v = make_uint2(out_v[0] | (out_v[1] << 16), out_v[2] | (out_v[3] << 16));
  if (bad_m) q_m = make_uint2(kNan * 0x01010101u, kNan * 0x01010101u);
  if (bad_v) q_v = make_uint2(kNan * 0x01010101u, kNan * 0x01010101u);
  if ((threadIdx.x & 15u) == 0 && p.n > 0) {
    J.ms[p.is] = static_cast<uint8_t>(new_m);
    J.vs[p.is] = static_cast<uint8_t>(new_v);
  }
  if (p.wide) {
    *reinterpret_cast<uint2*>(M) = q_m;
    *reinterpret_cast<uint2*>(V) = q_v;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i < p.n) {
        M[i] = static_cast<uint8_t>((i < 4 ? q_m.x : q_m.y) >> (8 * (i & 3)));
        V[i] = static_cast<uint8_t>((i < 4 ? q_v.x : q_v.y) >> (8 * (i & 3)));
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
  j->grad16 = grad16;
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
  // one kernel for each kind of moments, and launches of up to kAdamMaxJobs tensors of that kind
  for (const int bits : {8, 32}) {
    if (bits == 8 && T.eps > 0.0f && T.eps < FLT_MIN) T.eps = FLT_MIN;     // (a denormal one has no reciprocal there)
    for (int i = 0; i < n_jobs;) {
      long long total = 0;
      T.n_jobs = 0;
      for (; i < n_jobs && T.n_jobs < kAdamMaxJobs; ++i) {
        if (jobs[i].state_bits != bits) continue;
        long long ctas;
        BSP_TRY(make_job(jobs[i], static_cast<uint32_t>(i), &T.job[T.n_jobs], &ctas));
        if (T.n_jobs > 0 && total + ctas > 0x7fffffffLL) break;
        T.first[T.n_jobs++] = static_cast<int>(total);
        total += ctas;
      }
      if (T.n_jobs == 0) break;
      T.first[T.n_jobs] = static_cast<int>(total);
      BSP_CUDA_TRY(launch_pdl(bits == 8 ? adam_batched8_kernel : adam_batched_kernel, dim3(static_cast<unsigned>(total)), dim3(kAdamThreads), 0, s, T));
    }
    T.eps = eps;
  }
  return BSP_OK;
}
