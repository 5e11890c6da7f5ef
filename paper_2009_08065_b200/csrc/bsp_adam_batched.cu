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
// Bytes per weight with a bf16 gradient: 8 bits 2 + 8 + 4 + 2 = 16, 32 bits 2 + 8 + 16 + 2 = 28.  32 bits are bound by HBM, eight neighbouring
// weights a thread in 16-byte accesses; 8 bits by HBM and issue together (adam_stream8_kernel: 1.25 to 1.35 times the bytes' time by GPU).  There sixteen threads share a block
// of 128 weights, eight each, and the block's largest moments are a reduction over half a warp.
#include <float.h>
#include <math.h>

#include "bsp_fp8.cuh"
#include "bsp_tc.cuh"

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
  uint32_t block_magic;      // row / block = the upper half of row * block_magic
  uint8_t grad16, wide, keep_wide;
  uint32_t kb_magic;         // block of 128 / blocks in a row, the same way
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
  int* status;                                     // where a wait that ran out is recorded
  int g_size;                                      // bytes of the widest gradient
};

// The random bits of a weight: multiplications by odd constants (the fractions of 2^(1/2) and 3^(1/2)) between shifts that
// bring the upper half down.
__device__ __forceinline__ uint32_t mix_open(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x6A09E667u;
  return (x ^ (x >> 15)) * 0xBB67AE85u;
}
__device__ __forceinline__ uint32_t mix(uint32_t x) {
  x = mix_open(x);
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

__device__ __forceinline__ float one_if_less(float a, float b) {
  float r;
  asm("set.lt.f32.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// Two magnitudes (not negative, in the format's range) to one of their two neighbours in the format: random bits are added at the
// upper end of what is then cut off (r: 16 of them).  Below the smallest normal value steps are as wide as just above it, so that
// value is added first and taken off again.  (The integer pipe, at half the rate of the others, is what this kernel fills:
// hence a comparison that gives 1 or 0 as float32, and a multiply-add for the random bits.  The two values go one by one here: packed
// operations between single ones cost more moves than they save, 302 M weights 947 us and 937.)
template <int FMT>
__device__ __forceinline__ Pair round_pair(Pair y, uint32_t r0, uint32_t r1) {
  constexpr int kDrop = FMT == BSP_FP8_E4M3 ? 20 : 21;
  constexpr uint32_t kKeep = ~((1u << kDrop) - 1u);
  constexpr float kLow = FMT == BSP_FP8_E4M3 ? 0x1p-6f : 0x1p-14f;
  float y0, y1;
  split(y, y0, y1);
  const float b0 = one_if_less(y0, kLow), b1 = one_if_less(y1, kLow);
  uint32_t u0, u1;
  asm("mad.lo.u32 %0, %1, %2, %3;" : "=r"(u0) : "r"(r0), "n"(1 << (kDrop - 16)), "r"(__float_as_uint(__fmaf_rn(b0, kLow, y0))));
  asm("mad.lo.u32 %0, %1, %2, %3;" : "=r"(u1) : "r"(r1), "n"(1 << (kDrop - 16)), "r"(__float_as_uint(__fmaf_rn(b1, kLow, y1))));
  return pair_of(__fmaf_rn(b0, -kLow, __uint_as_float(u0 & kKeep)), __fmaf_rn(b1, -kLow, __uint_as_float(u1 & kKeep)));
}
// Denormal values count as zero.
__device__ __forceinline__ float square_root(float x) {
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// The largest magnitude of three, NaN if there is one.
__device__ __forceinline__ float abs_max3(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)), "f"(fabsf(c)));
  return r;
}

// The job of this CTA.
__device__ __forceinline__ int find_job(const AdamTable& T) {
  int lo = 0, hi = T.n_jobs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (T.first[mid] <= static_cast<int>(blockIdx.x)) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}
// Up to eight neighbouring weights of a row: row, first column, how many of the eight exist.
struct Place {
  uint32_t r;
  int c, n;
  bool wide;
};
__device__ __forceinline__ Place place_at(const AdamJob& J, uint32_t r, int c) {
  Place p;
  p.r = r;
  p.c = c;
  p.n = r < static_cast<uint32_t>(J.rows) ? max(0, min(8, J.cols - c)) : 0;
  p.wide = J.wide != 0 && p.n == 8;
  return p;
}
__device__ __forceinline__ uint32_t divided(unsigned long long n, uint32_t d) {
  return n < 0xffffffffull ? static_cast<uint32_t>(n) / d : static_cast<uint32_t>(n / d);
}
// Sixteen threads to a block of 128 (8-bit moments; kb: blocks in a row), of which b is this thread's.
__device__ __forceinline__ Place place_of(const AdamJob& J, uint32_t kb, unsigned long long group, uint32_t& b) {
  const uint32_t r = divided(group, kb);
  b = static_cast<uint32_t>(group - static_cast<unsigned long long>(r) * kb);
  return place_at(J, r, static_cast<int>(b * kBlock + 8u * (threadIdx.x & 15u)));
}
// The rows' pieces of eight one after the other (32-bit moments, which have no blocks: whole blocks of 16 threads left the threads behind
// a row's end idle: 4.9 M weights in rows of 184 and 736 37.4 -> 26.1 us).
__device__ __forceinline__ Place piece_of(const AdamJob& J, unsigned long long piece) {
  const uint32_t each = (static_cast<uint32_t>(J.cols) + 7u) / 8u, r = divided(piece, each);
  return place_at(J, r, static_cast<int>(8u * static_cast<uint32_t>(piece - static_cast<unsigned long long>(r) * each)));
}
__device__ __forceinline__ size_t at(const Place& p, int ld) { return static_cast<size_t>(p.r) * ld + p.c; }
__device__ __forceinline__ void load_weights(const AdamJob& J, const Place& p, float (&w)[8], float (&g)[8]) {
  if (p.wide) {
    load8(J.W + at(p, J.ldw), w);
    if (J.grad16) {
      const uint4 h = ld_global(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(J.G) + at(p, J.ldg)));
      const uint32_t hw[4] = {h.x, h.y, h.z, h.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) { g[2 * i] = __uint_as_float(hw[i] << 16); g[2 * i + 1] = __uint_as_float(hw[i] & 0xffff0000u); }
    } else {
      load8(static_cast<const float*>(J.G) + at(p, J.ldg), g);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[i] = g[i] = 0.0f;
      if (i < p.n) {
        w[i] = ld_global(J.W + at(p, J.ldw) + i);
        g[i] = J.grad16 ? bf16_bits_to_float(ld_global(static_cast<const uint16_t*>(J.G) + at(p, J.ldg) + i)) : ld_global(static_cast<const float*>(J.G) + at(p, J.ldg) + i);
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
__device__ __forceinline__ uint4 eight_bf16(const float (&w)[8]) {
  uint32_t half[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(half[i]) : "f"(w[2 * i + 1]), "f"(w[2 * i]));
  return make_uint4(half[0], half[1], half[2], half[3]);
}
__device__ __forceinline__ void store_weights(const AdamJob& J, const Place& p, const float (&w)[8]) {
  const uint4 packed = eight_bf16(w);
  const uint32_t half[4] = {packed.x, packed.y, packed.z, packed.w};
  uint16_t* wb = J.Wb != nullptr ? J.Wb + at(p, J.ldb) : nullptr;
  if (p.wide) {
    store8(J.W + at(p, J.ldw), w);
    if (wb != nullptr) *reinterpret_cast<uint4*>(wb) = packed;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i < p.n) {
        J.W[at(p, J.ldw) + i] = w[i];
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
  const int job = find_job(T);
  const AdamJob& J = T.job[job];
  const Place p = piece_of(J, static_cast<unsigned long long>(blockIdx.x - T.first[job]) * kAdamThreads + threadIdx.x);
  pdl_wait();
  pdl_launch_dependents();
  float w[8], g[8], m[8], v[8];
  load_weights(J, p, w, g);
  float *M = static_cast<float*>(J.M) + at(p, J.ldm), *V = static_cast<float*>(J.V) + at(p, J.ldm);
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

// 8-bit moments.  HBM allows 90 issue slots (45 of the integer pipe) for a warp's 32 weights, and the kernel takes 84 (35), of which the random
// bits are 11: it runs 1.25 times as long as its bytes would (without the hash 889 us in place of 947).  Hence packed float32 operations, and
// the hardware's approximate square root and reciprocal (each within about a place) for the update of W (the moments, which the 8-bit
// values follow to the last bit, are rounded as defined).
// Eight weights as they lie in memory.
struct Raw {
  uint4 w[2], g[2];            // g: float32, or bf16 in the first half
  uint2 m, v, keep;            // keep: a byte for each weight, zero where it is pruned
  uint32_t byte_m, byte_v;
};
struct Stepped {
  float w[8];
  uint2 m, v;
  int byte_m, byte_v;
  bool bad;                    // the block has a moment that is not finite (the same for its sixteen threads)
};
// What is the same for all weights of a job.
struct Rates {
  Pair gs, b1, b2, c1, c2, decay;      // decay: -lr weight_decay
  float rate, eps, i2;                 // rate: -lr / (1 - beta1^step)
  uint32_t key;
};
// One step of eight weights; `position` is the first one's place in its tensor.  Sixteen neighbouring threads meet in it.
template <bool kGrad16, bool kMask>
__device__ __forceinline__ Stepped step_eight(const Raw& x, uint32_t position, const Rates& R) {
  Stepped out;
  const Pair scale_m = pair_of(scale_value(x.byte_m)), scale_v = pair_of(scale_value(x.byte_v));
  const uint32_t wb[8] = {x.w[0].x, x.w[0].y, x.w[0].z, x.w[0].w, x.w[1].x, x.w[1].y, x.w[1].z, x.w[1].w};
  const uint32_t gb[8] = {x.g[0].x, x.g[0].y, x.g[0].z, x.g[0].w, x.g[1].x, x.g[1].y, x.g[1].z, x.g[1].w};
  Pair m[4], v[4];
  float most_m = 0.0f, most_v = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float lo, hi;
    const Pair gi = mul(kGrad16 ? pair_of(__uint_as_float(gb[i] << 16), __uint_as_float(gb[i] & 0xffff0000u))
                                : pair_of(__uint_as_float(gb[2 * i]), __uint_as_float(gb[2 * i + 1])), R.gs);
    from_fp8x2<BSP_FP8_E4M3>((i < 2 ? x.m.x : x.m.y) >> (16 * (i & 1)), lo, hi);
    m[i] = fma(R.b1, mul(pair_of(lo, hi), scale_m), mul(R.c1, gi));
    split(m[i], lo, hi);
    most_m = abs_max3(most_m, lo, hi);
    from_fp8x2<BSP_FP8_E5M2>((i < 2 ? x.v.x : x.v.y) >> (16 * (i & 1)), lo, hi);
    v[i] = fma(R.b2, mul(pair_of(lo, hi), scale_v), mul(mul(R.c2, gi), gi));
    split(v[i], lo, hi);
    most_v = abs_max3(most_v, lo, hi);
  }
  const uint32_t lanes = 0xffffu << (threadIdx.x & 16u);
  const uint32_t top_m = __reduce_max_sync(lanes, __float_as_uint(most_m)), top_v = __reduce_max_sync(lanes, __float_as_uint(most_v));
  // The square root takes denormal values for zero, so in a block that has room for that v goes through it 2^24 times larger,
  // and eps and the rate are 2^12 times larger too.
  const bool room = top_v < 0x5f800000u;               // 2^64
  const float larger = room ? 0x1p12f : 1.0f;
  const Pair p2 = pair_of(R.i2 * (larger * larger)), eps = pair_of(R.eps * larger), rate = pair_of(R.rate * larger);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float lo, hi;
    split(mul(v[i], p2), lo, hi);
    split(add(pair_of(square_root(lo), square_root(hi)), eps), lo, hi);
    const Pair wi = pair_of(__uint_as_float(wb[2 * i]), __uint_as_float(wb[2 * i + 1]));
    split(fma(R.decay, wi, fma(mul(m[i], rate), pair_of(reciprocal(lo), reciprocal(hi)), wi)), lo, hi);
    out.w[2 * i] = !kMask || kept(x.keep, 2 * i) ? lo : 0.0f;
    out.w[2 * i + 1] = !kMask || kept(x.keep, 2 * i + 1) ? hi : 0.0f;
  }
  // a block with an infinity or a NaN becomes NaN throughout, under scale 1
  const bool bad_m = top_m >= 0x7f800000u, bad_v = top_v >= 0x7f800000u;
  out.byte_m = bad_m ? 127 : scale_byte(top_m, top_of(BSP_FP8_E4M3));
  out.byte_v = bad_v ? 127 : scale_byte(top_v, top_of(BSP_FP8_E5M2));
  const Pair inv_m = pair_of(scale_inverse(out.byte_m)), inv_v = pair_of(scale_inverse(out.byte_v));
  uint32_t out_m[2], out_v[2];
  float qm[8], qv[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t m_bits[2], v_bits[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t h = mix_open(position + static_cast<uint32_t>(2 * i + e) + R.key);
      v_bits[e] = h >> 16;                             // the upper and the lower half of h ^ (h >> 16)
      m_bits[e] = (h ^ v_bits[e]) & 0xffffu;
    }
    float lo, hi, a, b;
    split(m[i], a, b);
    split(round_pair<BSP_FP8_E4M3>(mul(pair_of(fabsf(a), fabsf(b)), inv_m), m_bits[0], m_bits[1]), lo, hi);
    qm[2 * i] = copysignf(lo, a);
    qm[2 * i + 1] = copysignf(hi, b);
    if (i & 1) out_m[i >> 1] = to_fp8x4<BSP_FP8_E4M3>(qm[2 * i - 2], qm[2 * i - 1], qm[2 * i], qm[2 * i + 1]);
    // A positive value below the smallest one becomes that, which random bits leave as it is.
    split(v[i], lo, hi);
    split(mul(pair_of(one_if_less(0.0f, lo), one_if_less(0.0f, hi)), pair_of(0x1p-16f)), a, b);
    split(mul(v[i], inv_v), lo, hi);
    split(round_pair<BSP_FP8_E5M2>(pair_of(fmaxf(lo, a), fmaxf(hi, b)), v_bits[0], v_bits[1]), lo, hi);
    qv[2 * i] = lo;
    qv[2 * i + 1] = hi;
    if (i & 1) out_v[i >> 1] = to_fp8x4<BSP_FP8_E5M2>(qv[2 * i - 2], qv[2 * i - 1], qv[2 * i], qv[2 * i + 1]);
  }
  out.m = make_uint2(out_m[0], out_m[1]);
  out.v = make_uint2(out_v[0], out_v[1]);
  if (bad_m) out.m = make_uint2(kNan * 0x01010101u, kNan * 0x01010101u);
  if (bad_v) out.v = make_uint2(kNan * 0x01010101u, kNan * 0x01010101u);
  out.bad = bad_m || bad_v;
  return out;
}
// What is not finite at a pruned place stays out of its block's kept weights: its moments begin again at zero.  Blocks that need it take
// their step a second time, out of line and from what memory still holds: 302 M weights 1012 us, 996 without the question; with the values kept
// in registers for it 1062.
template <bool kGrad16>
__device__ __forceinline__ void begin_again(Raw& x, const Rates& R) {
  uint32_t g[8] = {x.g[0].x, x.g[0].y, x.g[0].z, x.g[0].w, x.g[1].x, x.g[1].y, x.g[1].z, x.g[1].w};
  uint32_t m[2] = {x.m.x, x.m.y}, v[2] = {x.v.x, x.v.y};
  float gs, b1, c1, b2, c2, unused;
  split(R.gs, gs, unused);
  split(R.b1, b1, unused);
  split(R.c1, c1, unused);
  split(R.b2, b2, unused);
  split(R.c2, c2, unused);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float hi, om, ov;
    const float gi = __fmul_rn(kGrad16 ? __uint_as_float((i & 1) ? g[i >> 1] & 0xffff0000u : g[i >> 1] << 16) : __uint_as_float(g[i]), gs);
    from_fp8x2<BSP_FP8_E4M3>((m[i >> 2] >> (8 * (i & 3))) & 0xffu, om, hi);
    from_fp8x2<BSP_FP8_E5M2>((v[i >> 2] >> (8 * (i & 3))) & 0xffu, ov, hi);
    om = __fmaf_rn(b1, om * scale_value(x.byte_m), __fmul_rn(c1, gi));
    ov = __fmaf_rn(b2, ov * scale_value(x.byte_v), __fmul_rn(__fmul_rn(c2, gi), gi));
    if (kept(x.keep, i) || (fabsf(om) <= FLT_MAX && fabsf(ov) <= FLT_MAX)) continue;
    if (kGrad16) g[i >> 1] &= (i & 1) ? 0xffffu : 0xffff0000u;
    else g[i] = 0u;
    m[i >> 2] &= ~(0xffu << (8 * (i & 3)));
    v[i >> 2] &= ~(0xffu << (8 * (i & 3)));
  }
  x.g[0] = make_uint4(g[0], g[1], g[2], g[3]);
  x.g[1] = make_uint4(g[4], g[5], g[6], g[7]);
  x.m = make_uint2(m[0], m[1]);
  x.v = make_uint2(v[0], v[1]);
}

// What is the same for all jobs of a launch, read once.
struct Common {
  int step;
  float i1, i2, gs;
};
__device__ __forceinline__ Common common(const AdamTable& T) {
  Common C;
  C.step = corrections(T, C.i1, C.i2);
  C.gs = T.grad_scale != nullptr ? ld_global(T.grad_scale) : 1.0f;
  return C;
}
__device__ __forceinline__ void rates(const AdamTable& T, const Common& C, const AdamJob& J, Rates& R) {
  R.key = mix(T.seed + 0x9E3779B9u * static_cast<uint32_t>(C.step) + 0xBB67AE85u * J.tensor);
  R.gs = pair_of(C.gs);
  R.b1 = pair_of(T.beta1); R.b2 = pair_of(T.beta2); R.c1 = pair_of(1.0f - T.beta1); R.c2 = pair_of(1.0f - T.beta2);
  R.i2 = C.i2; R.rate = -J.lr * C.i1; R.eps = T.eps; R.decay = pair_of(-J.lr * J.decay);
}

// Tensors without gaps whose rows are whole pieces of eight, masked along columns or not at all.  Sixteen blocks of 128 lie next to each
// other in memory then, and reach shared memory by bulk copies, two such chunks ahead: 100 KB on their way per SM.  Loads to registers, also one
// turn ahead, came to half of that at 24 warps per SM, and the kernel waited for them: 302 M weights 1088 us however little was computed, this
// way 937 (5.2 TB/s).  A fourth stage takes its room from L1, where the flags of a block's rows are found again (5 % slower); four and five CTAs per
// SM, with fewer registers, were no faster.  CTAs that run at once work on neighbouring chunks.
constexpr int kChunk = kAdamGroups * kBlock;       // weights
constexpr int kStreamCtas = 3;                     // of an SM
constexpr int kStreamStages = 3;
constexpr int kStreamW = kChunk * 4, kStreamQ = kChunk + 32, kStreamS = 32;      // bytes (8-bit values begin anywhere: copied from a multiple of 16 on)
constexpr int kStreamHead = 16 * kStreamStages + 80;               // mbarriers, a flag
// A stage: W, m, v, the scales of both, and the gradients of the widest type among the launch's tensors.
__host__ __device__ constexpr int stream_stage(int g_size) { return kStreamW + 2 * kStreamQ + 2 * kStreamS + kChunk * g_size; }
static_assert(kStreamHead % 16 == 0 && stream_stage(2) % 16 == 0, "alignment of bulk copies");

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}
// The bytes [p, p + n) in whole pieces of 16; they begin (p % 16) bytes behind dst.
__device__ __forceinline__ uint32_t pieces16(const uint8_t* p, uint32_t n) { return (n + static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p) & 15u) + 15u) & ~15u; }
__device__ __forceinline__ const uint8_t* floor16(const uint8_t* p) { return p - (reinterpret_cast<uintptr_t>(p) & 15u); }
// First weight of a block of 128 in its tensor, and its row.
__device__ __forceinline__ size_t block_begin(const AdamJob& J, uint32_t kb, uint32_t group, uint32_t& r, uint32_t& c) {
  r = J.kb_magic != 0u ? __umulhi(group, J.kb_magic) : group;
  c = (group - r * kb) * kBlock;
  return static_cast<size_t>(r) * static_cast<uint32_t>(J.cols) + c;
}
// Asks for a chunk of a job, by a whole warp: lanes 0 to 5 one copy each.
constexpr int kCopies = 6;
__device__ __forceinline__ void ask_for(const AdamJob& J, uint32_t chunk, uint32_t stage, uint32_t bar) {
  const uint32_t kb = static_cast<uint32_t>(blocks_of(J.cols)), groups = static_cast<uint32_t>(J.rows) * kb;
  const uint32_t first = chunk * kAdamGroups, behind = min(first + kAdamGroups, groups);
  uint32_t r, c;
  const size_t e = block_begin(J, kb, first, r, c);
  const size_t end = behind == groups ? static_cast<size_t>(J.rows) * static_cast<uint32_t>(J.cols) : block_begin(J, kb, behind, r, c);
  const uint32_t lane = threadIdx.x & 31u;
  const bool scales = lane == 3u || lane == 4u;
  const uint32_t size = lane == 0u ? 4u : lane == 5u ? (J.grad16 ? 2u : 4u) : 1u;
  const void* from = lane == 0u ? J.W : lane == 1u ? J.M : lane == 2u ? J.V : lane == 3u ? J.ms : lane == 4u ? J.vs : J.G;
  const uint32_t to = lane == 0u ? 0u : lane == 1u ? kStreamW : lane == 2u ? kStreamW + kStreamQ : lane == 3u ? kStreamW + 2 * kStreamQ
                      : lane == 4u ? kStreamW + 2 * kStreamQ + kStreamS : kStreamW + 2 * kStreamQ + 2 * kStreamS;
  const uint8_t* src = static_cast<const uint8_t*>(from) + (scales ? static_cast<size_t>(first) : e * size);
  const uint32_t bytes = pieces16(src, scales ? behind - first : static_cast<uint32_t>(end - e) * size);
  if (lane < kCopies) {
    tc::mbar_arrive_expect_tx(bar, bytes);
    bulk_load(stage + to, floor16(src), bytes, bar);
  }
  __syncwarp();
}

// A thread's eight weights of a chunk: block of 128, row and column of the first, and their flags, asked for a turn ahead.
struct Turn {
  uint32_t group, r, c;
  uint2 keep;
};
// kRagged: rows end inside a block of 128.  (Where they don't, a block's sixteen threads all have weights or none have, and those that have none
// may work on what shared memory holds.)
template <bool kGrad16, bool kRagged>
struct Piece {
  size_t e, e0;                // the first of the eight weights, and of the chunk
  bool exists;
  __device__ __forceinline__ Piece(const AdamJob& J, const Turn& t, uint32_t chunk) {
    e = static_cast<size_t>(t.r) * static_cast<uint32_t>(J.cols) + t.c;
    exists = t.r < static_cast<uint32_t>(J.rows) && (!kRagged || t.c < static_cast<uint32_t>(J.cols));
    if (kRagged) {
      uint32_t r, c;
      e0 = block_begin(J, static_cast<uint32_t>(blocks_of(J.cols)), chunk * kAdamGroups, r, c);
    } else {
      e0 = e - 8u * threadIdx.x;
    }
  }
  // What the stage holds of it.
  __device__ __forceinline__ Raw load(const AdamJob& J, const Turn& t, uint32_t stage) const {
    const uint32_t i = !kRagged ? 8u * threadIdx.x : exists ? static_cast<uint32_t>(e - e0) : 0u;      // place in the chunk
    auto two = [](uint32_t a) {
      uint2 v;
      asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
      return v;
    };
    Raw x;
    x.w[0] = tc::ld_shared_v4(stage + 4u * i);
    x.w[1] = tc::ld_shared_v4(stage + 4u * i + 16u);
    stage += kStreamW;
    x.m = two(stage + i + (static_cast<uint32_t>(reinterpret_cast<uintptr_t>(J.M) + e0) & 15u));
    x.v = two(stage + kStreamQ + i + (static_cast<uint32_t>(reinterpret_cast<uintptr_t>(J.V) + e0) & 15u));
    stage += 2 * kStreamQ;
    auto byte = [](uint32_t a) {
      uint32_t v;
      asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a));
      return v;
    };
    const uint32_t block = threadIdx.x >> 4;             // of the chunk
    x.byte_m = byte(stage + block + (static_cast<uint32_t>(reinterpret_cast<uintptr_t>(J.ms) + t.group - block) & 15u));
    x.byte_v = byte(stage + kStreamS + block + (static_cast<uint32_t>(reinterpret_cast<uintptr_t>(J.vs) + t.group - block) & 15u));
    stage += 2 * kStreamS;
    x.g[0] = tc::ld_shared_v4(stage + (kGrad16 ? 2u : 4u) * i);
    if (!kGrad16) x.g[1] = tc::ld_shared_v4(stage + 4u * i + 16u);
    if (kRagged && !exists) {
      x.g[0] = x.g[1] = make_uint4(0u, 0u, 0u, 0u);
      x.m = x.v = make_uint2(0u, 0u);
    }
    x.keep = t.keep;
    return x;
  }
  __device__ __forceinline__ void store(const AdamJob& J, const Turn& t, const Stepped& z) const {
    if (!exists) return;
    store8(J.W + e, z.w);
    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(J.M) + e) = z.m;
    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(J.V) + e) = z.v;
    if (J.Wb != nullptr) *reinterpret_cast<uint4*>(J.Wb + e) = eight_bf16(z.w);
    if ((threadIdx.x & 15u) == 0u) {
      J.ms[t.group] = static_cast<uint8_t>(z.byte_m);
      J.vs[t.group] = static_cast<uint8_t>(z.byte_v);
    }
  }
};
// (a whole warp: a block that did not need it gets the same results again, over those that are stored)
template <bool kGrad16, bool kRagged>
__device__ __noinline__ void chunk_again(const AdamJob& J, Turn t, uint32_t chunk, uint32_t stage, Rates R) {
  const Piece<kGrad16, kRagged> p(J, t, chunk);
  Raw x = p.load(J, t, stage);
  begin_again<kGrad16>(x, R);
  p.store(J, t, step_eight<kGrad16, true>(x, static_cast<uint32_t>(p.e), R));
}
template <bool kGrad16, bool kMask, bool kRagged>
__device__ __forceinline__ void chunk_step(const AdamJob& J, const Turn& t, uint32_t chunk, uint32_t stage, const Rates& R) {
  const Piece<kGrad16, kRagged> p(J, t, chunk);
  const Stepped z = step_eight<kGrad16, kMask>(p.load(J, t, stage), static_cast<uint32_t>(p.e), R);
  p.store(J, t, z);
  if (kMask && __any_sync(0xffffffffu, z.bad)) chunk_again<kGrad16, kRagged>(J, t, chunk, stage, R);
}
template <bool kRagged>
__device__ __forceinline__ void chunk_step(const AdamJob& J, const Turn& t, uint32_t chunk, uint32_t stage, const Rates& R) {
  if (J.grad16) {
    if (J.keep != nullptr) chunk_step<true, true, kRagged>(J, t, chunk, stage, R);
    else chunk_step<true, false, kRagged>(J, t, chunk, stage, R);
  } else {
    if (J.keep != nullptr) chunk_step<false, true, kRagged>(J, t, chunk, stage, R);
    else chunk_step<false, false, kRagged>(J, t, chunk, stage, R);
  }
}

__global__ void __launch_bounds__(kAdamThreads, kStreamCtas)
adam_stream8_kernel(const __grid_constant__ AdamTable T) {
  extern __shared__ __align__(128) uint8_t smem[];
  const uint32_t full = tc::smem_u32(smem), empty = full + 8u * kStreamStages, base = full + kStreamHead;
  volatile uint32_t* timed_out = reinterpret_cast<volatile uint32_t*>(smem + 16 * kStreamStages);
  constexpr int stages = kStreamStages;
  const int stage_bytes = stream_stage(T.g_size);
  if (threadIdx.x == 0) {
    *timed_out = 0u;
    for (int s = 0; s < stages; ++s) {
      tc::mbar_init(full + 8u * s, kCopies);
      tc::mbar_init(empty + 8u * s, kAdamThreads / 32);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tc::fence_async_smem();
  }
  __syncthreads();
  const int chunks = T.first[T.n_jobs];
  // The job of a chunk, by a whole warp whose lanes hold where the jobs begin.  (By a walk through the table, each step of it a read of
  // constant memory: 192 tensors of 4.9 M weights in rows of 184 and 736 35.1 us, this way 31.2.)
  static_assert(kAdamMaxJobs == 96, "three jobs to a lane");
  int begin[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const int job = 32 * i + static_cast<int>(threadIdx.x & 31u);
    begin[i] = job < T.n_jobs ? T.first[job] : 0x7fffffff;
  }
  auto job_of = [&](int chunk) {
    return __popc(__ballot_sync(0xffffffffu, begin[0] <= chunk)) + __popc(__ballot_sync(0xffffffffu, begin[1] <= chunk)) +
           __popc(__ballot_sync(0xffffffffu, begin[2] <= chunk)) - 1;
  };
  pdl_wait();
  pdl_launch_dependents();
  int asked_job = 0;
  auto ask = [&](int chunk, int stage) {
    if (chunk >= T.first[asked_job + 1]) asked_job = job_of(chunk);
    ask_for(T.job[asked_job], static_cast<uint32_t>(chunk - T.first[asked_job]), base + stage * stage_bytes, full + 8u * stage);
  };
  const int grid = static_cast<int>(gridDim.x);
  if (threadIdx.x < 32) {
    for (int s = 0; s < stages && static_cast<int>(blockIdx.x) + s * grid < chunks; ++s) ask(blockIdx.x + s * grid, s);
  }
  const Common same = common(T);
  int job = -1, stage = 0;
  uint32_t turn = 0u;
  uint32_t phase = 0u, last = 0u;                    // last: parity of the stage before
  Rates R;
  bool ok = true;
  int next_job = 0;
  Turn next;
  auto look_up = [&](int chunk) {
    if (chunk >= T.first[next_job + 1]) next_job = job_of(chunk);
    const AdamJob& J = T.job[next_job];
    next.group = static_cast<uint32_t>(chunk - T.first[next_job]) * kAdamGroups + (threadIdx.x >> 4);
    block_begin(J, static_cast<uint32_t>(blocks_of(J.cols)), next.group, next.r, next.c);
    next.c += 8u * (threadIdx.x & 15u);
    if (J.keep != nullptr && next.r < static_cast<uint32_t>(J.rows) && next.c < static_cast<uint32_t>(J.cols))
      next.keep = ld_global(reinterpret_cast<const uint2*>(J.keep + static_cast<size_t>(J.block_magic != 0u ? __umulhi(next.r, J.block_magic) : next.r) * J.cols + next.c));
  };
  next.keep = make_uint2(0u, 0u);
  look_up(blockIdx.x);
  for (int chunk = blockIdx.x; chunk < chunks; chunk += grid) {
    const Turn now = next;
    if (next_job != job) {
      job = next_job;
      rates(T, same, T.job[job], R);
    }
    const AdamJob& J = T.job[job];
    // (one answer for the warp: its lanes meet again in what follows, so none may leave alone)
    if (!tc::mbar_wait_warp(full + 8u * stage, phase, T.status)) { ok = false; break; }
    if (chunk + grid < chunks) look_up(chunk + grid);
    const uint32_t at_stage = base + stage * stage_bytes, number = static_cast<uint32_t>(chunk - T.first[job]);
    if (J.cols % kBlock != 0) chunk_step<true>(J, now, number, at_stage, R);
    else chunk_step<false>(J, now, number, at_stage, R);
    __syncwarp();
    if ((threadIdx.x & 31u) == 0) tc::mbar_arrive(empty + 8u * stage);
    // The stage of the turn before, which the slowest warp has left by now or soon will have, is filled again, by each warp in turn: the warp
    // that asks falls behind the others.
    const int refill = chunk + (stages - 1) * grid;
    if (threadIdx.x >> 5 == (turn & 7u) && turn > 0 && refill < chunks) {
      const int before = stage == 0 ? stages - 1 : stage - 1;
      if (!tc::mbar_wait_warp(empty + 8u * before, last, T.status)) { ok = false; break; }
      ask(refill, before);
    }
    ++turn;
    last = phase;
    if (++stage == stages) { stage = 0; phase ^= 1u; }
  }
  if (!ok) tc::record_timeout(T.status, timed_out);
  __syncthreads();
  tc::quiet_period(timed_out);                       // (copies in flight still land in this CTA's shared memory)
}

// A thread's eight weights of any tensor, as float32 gradients (is: the place of their block's scales).
__device__ __forceinline__ Raw load_any(const AdamJob& J, const Place& p, size_t is) {
  const uint8_t *M = static_cast<const uint8_t*>(J.M) + at(p, J.ldm), *V = static_cast<const uint8_t*>(J.V) + at(p, J.ldm);
  float w[8], g[8];
  load_weights(J, p, w, g);
  uint32_t q[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (i < p.n) {
      q[i >> 2] |= static_cast<uint32_t>(ld_global(M + i)) << (8 * (i & 3));
      q[2 + (i >> 2)] |= static_cast<uint32_t>(ld_global(V + i)) << (8 * (i & 3));
    }
  }
  auto four = [](const float* f) { return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])); };
  Raw x;
  x.w[0] = four(w); x.w[1] = four(w + 4); x.g[0] = four(g); x.g[1] = four(g + 4);
  x.m = make_uint2(q[0], q[1]);
  x.v = make_uint2(q[2], q[3]);
  x.keep = load_flags(J, p);
  x.byte_m = p.n > 0 ? ld_global(J.ms + is) : 127u;
  x.byte_v = p.n > 0 ? ld_global(J.vs + is) : 127u;
  return x;
}
__device__ __noinline__ Stepped any_again(const AdamJob& J, Place p, size_t is, uint32_t position, Rates R) {
  Raw x = load_any(J, p, is);
  begin_again<false>(x, R);
  return step_eight<false, true>(x, position, R);
}

// Any other tensor.
__global__ void __launch_bounds__(kAdamThreads)
adam_batched8_kernel(const __grid_constant__ AdamTable T) {
  const int job = find_job(T);
  const AdamJob& J = T.job[job];
  const uint32_t kb = static_cast<uint32_t>(blocks_of(J.cols));
  uint32_t b;
  const Place p = place_of(J, kb, static_cast<unsigned long long>(blockIdx.x - T.first[job]) * kAdamGroups + (threadIdx.x >> 4), b);
  uint8_t *M = static_cast<uint8_t*>(J.M) + at(p, J.ldm), *V = static_cast<uint8_t*>(J.V) + at(p, J.ldm);
  const size_t is = static_cast<size_t>(p.r) * kb + b;
  pdl_wait();
  pdl_launch_dependents();
  Rates R;
  rates(T, common(T), J, R);
  const uint32_t position = p.r * static_cast<uint32_t>(J.cols) + static_cast<uint32_t>(p.c);
  Stepped z = step_eight<false, true>(load_any(J, p, is), position, R);
  if (z.bad) z = any_again(J, p, is, position, R);
  store_weights(J, p, z.w);
  if ((threadIdx.x & 15u) == 0 && p.n > 0) {
    J.ms[is] = static_cast<uint8_t>(z.byte_m);
    J.vs[is] = static_cast<uint8_t>(z.byte_v);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (i < p.n) {
      M[i] = static_cast<uint8_t>((i < 4 ? z.m.x : z.m.y) >> (8 * (i & 3)));
      V[i] = static_cast<uint8_t>((i < 4 ? z.v.x : z.v.y) >> (8 * (i & 3)));
    }
  }
}

// Whether a tensor of 8-bit moments goes through adam_stream8_kernel (its numbers of blocks and rows have to divide by multiplication).
bool streams(const bsp_adam_job& a, const AdamJob& j) {
  const unsigned long long kb = blocks_of(a.cols), most = 1ull << 32;
  return a.state_bits == 8 && j.wide && a.cols % 8 == 0 && a.ldw == a.cols && a.ldg == a.cols && a.ldm == a.cols && (a.W_bf16 == nullptr || a.ldb == a.cols) &&
         (static_cast<unsigned long long>(a.rows) * kb + kAdamGroups) * kb < most &&
         (a.keep == nullptr || (a.orient == BSP_ORIENT_C && j.keep_wide && (static_cast<unsigned long long>(a.rows) + kAdamGroups) * a.block < most));
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
  // ceil(2^32 / d): exact for numbers below 2^32 / d; 0 for d = 1
  auto magic = [](long long d) { return d > 1 ? static_cast<uint32_t>((0x100000000ll + d - 1) / d) : 0u; };
  j->block_magic = magic(j->block);
  j->kb_magic = magic(blocks_of(a.cols));
  const long long rows = a.rows, pieces = rows * ((a.cols - 1) / 8 + 1), groups = rows * blocks_of(a.cols);
  *ctas = bits8 ? (groups + kAdamGroups - 1) / kAdamGroups : (pieces + kAdamThreads - 1) / kAdamThreads;
  return *ctas > 0x3fffffffLL || a.rows > kMostSize || a.cols > kMostSize ? BSP_ERR_UNSUPPORTED : BSP_OK;
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
  // One kernel for each kind of tensor, and launches of up to kAdamMaxJobs tensors of that kind.  All jobs are checked before the first
  // launch, and the first kAdamMaxJobs of them looked over only then.
  enum { kStream8, kAny8, kBits32, kKinds };
  struct Made {
    AdamJob job;
    int kind;
    long long ctas;
  };
  auto make = [&](int i, Made* made) {
    BSP_TRY(make_job(jobs[i], static_cast<uint32_t>(i), &made->job, &made->ctas));
    made->kind = jobs[i].state_bits == 32 ? kBits32 : streams(jobs[i], made->job) ? kStream8 : kAny8;
    return static_cast<int>(BSP_OK);
  };
  AdamTable T;
  Made known[kAdamMaxJobs], other;
  int of_kind[kKinds] = {0, 0, 0};
  for (int i = 0; i < n_jobs; ++i) {
    Made* made = i < kAdamMaxJobs ? &known[i] : &other;
    BSP_TRY(make(i, made));
    ++of_kind[made->kind];
  }
  TcDevice* dev = tc_device();
  if (dev == nullptr) return BSP_ERR_CUDA;
  T.status = dev->status;
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
  for (const int kind : {kStream8, kAny8, kBits32}) {
    if (kind != kBits32 && T.eps > 0.0f && T.eps < FLT_MIN) T.eps = FLT_MIN;     // (a denormal one has no reciprocal there)
    for (int i = 0; of_kind[kind] > 0 && i < n_jobs;) {
      long long total = 0;
      T.n_jobs = 0;
      T.g_size = 2;
      for (; i < n_jobs && T.n_jobs < kAdamMaxJobs; ++i) {
        if (i >= kAdamMaxJobs) BSP_TRY(make(i, &other));
        const Made& made = i < kAdamMaxJobs ? known[i] : other;
        if (made.kind != kind) continue;
        if (T.n_jobs > 0 && total + made.ctas > 0x3fffffffLL) break;
        if (!made.job.grad16) T.g_size = 4;
        T.job[T.n_jobs] = made.job;
        T.first[T.n_jobs++] = static_cast<int>(total);
        total += made.ctas;
      }
      of_kind[kind] -= T.n_jobs;
      T.first[T.n_jobs] = static_cast<int>(total);
      // (the table by its address: 11 KB)
      void* args[1] = {&T};
      cudaLaunchConfig_t cfg = {};
      cfg.blockDim = dim3(kAdamThreads);
      cfg.stream = s;
      cudaLaunchAttribute attr[1];
      attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
      attr[0].val.programmaticStreamSerializationAllowed = 1;
      cfg.attrs = attr;
      cfg.numAttrs = 1;
      const void* kernel = reinterpret_cast<const void*>(kind == kAny8 ? adam_batched8_kernel : adam_batched_kernel);
      long long grid = total;
      if (kind == kStream8) {
        static OncePerDevice once;
        BSP_TRY(allow_dynamic_smem(once, adam_stream8_kernel, kStreamHead + kStreamStages * stream_stage(4)));
        cfg.dynamicSmemBytes = kStreamHead + kStreamStages * stream_stage(T.g_size);
        kernel = reinterpret_cast<const void*>(adam_stream8_kernel);
        const long long seats = static_cast<long long>(kStreamCtas) * dev->sms;
        if (seats < grid) grid = seats;
      }
      cfg.gridDim = dim3(static_cast<unsigned>(grid));
      BSP_CUDA_TRY(cudaLaunchKernelExC(&cfg, kernel, args));
    }
    T.eps = eps;
  }
  return BSP_OK;
}
