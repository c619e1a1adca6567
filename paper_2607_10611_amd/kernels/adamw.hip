// AdamW over a list of tensors and the global gradient norm, for AMD Instinct
// MI355X (gfx950): kernels and the entry points declared in include/madd.h.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>
#include <string.h>

#include <cmath>

#include "e8m0.h"
#include "elem.h"
#include "exact.h"
#include "launch.h"
#include "madd.h"

namespace madd_detail {

constexpr int kAdamThreads = 256;
constexpr int kAdamOwn = 8;  // consecutive elements of a thread: one Philox block
constexpr int kAdamChunk = kAdamThreads * kAdamOwn;

struct AdamScalars {
  float b1, omb1, b2, omb2;  // beta1, 1 - beta1, beta2, 1 - beta2
  float decay;               // 1 - lr weight_decay
  float lr;                  // lr / (1 - beta1^t)
  float ir2;                 // 1 / sqrt(1 - beta2^t)
  float eps;
  uint32_t key0, key1, t;
};

struct AdamTensor {
  void* w;
  const void* g;
  void* m;
  void* v;
  uint8_t* scales;
  uint16_t* copy;
  int64_t n;
  int64_t group0;  // global index of element 0, over 8
  int32_t chunk0;  // first workgroup of this tensor within the launch
  int32_t pad;
};

// The tensors of one launch travel in its kernel arguments: no table in device
// memory to allocate, fill, cache or order between streams.
constexpr int kAdamList = 52;
struct AdamList {
  AdamScalars s;
  int32_t count, pad;
  AdamTensor t[kAdamList];
};
static_assert(sizeof(AdamList) <= 4000, "kernel arguments");

template <typename List>
__device__ __forceinline__ int find_tensor(const List& l, int32_t chunk) {
  int lo = 0, hi = l.count - 1;
  while (lo < hi) {  // uniform
    const int mid = (lo + hi + 1) >> 1;
    if (l.t[mid].chunk0 <= chunk) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

#define GLOBAL __attribute__((address_space(1)))
template <typename T>
__device__ __forceinline__ T load_nt(const void* p) {
  return __builtin_nontemporal_load((const GLOBAL T*)p);
}
template <typename T>
__device__ __forceinline__ void store_nt(void* p, T x) {
  __builtin_nontemporal_store(x, (GLOBAL T*)p);
}
typedef u4 u4_half __attribute__((aligned(2)));
typedef u2 u2_byte __attribute__((aligned(1)));

// Eight consecutive values of fp32 or bf16 storage, `have` of which exist (zeros
// past them), as they lie in memory.  They are converted apart from the branch
// that loads them: a conversion inside it would wait for this load before the
// next one is issued.
template <int F>
struct Raw8;
template <>
struct Raw8<WF_FP32> {
  f4 a, b;
  __device__ __forceinline__ void values(float (&x)[8]) const {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[k] = a[k];
      x[4 + k] = b[k];
    }
  }
};
template <>
struct Raw8<WF_BF16> {
  u4 a;
  __device__ __forceinline__ void values(float (&x)[8]) const {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      x[k] = __uint_as_float((k & 1) ? (a[k >> 1] & 0xFFFF0000u) : (a[k >> 1] << 16));
  }
};
template <int F>
__device__ __forceinline__ Raw8<F> load8(const void* p, int64_t i, int have) {
  Raw8<F> r;
  if (have >= 8) {
    if constexpr (F == WF_FP32) {
      r.a = load_nt<f4_any>((const float*)p + i);
      r.b = load_nt<f4_any>((const float*)p + i + 4);
    } else {
      r.a = load_nt<u4_half>((const uint16_t*)p + i);
    }
  } else if constexpr (F == WF_FP32) {
    r = {f4{0.0f, 0.0f, 0.0f, 0.0f}, f4{0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
    for (int k = 0; k < 7; ++k)
      if (k < have) (k < 4 ? r.a : r.b)[k & 3] = ((const float*)p)[i + k];
  } else {
    r.a = u4{0u, 0u, 0u, 0u};
#pragma unroll
    for (int k = 0; k < 7; ++k)
      if (k < have) r.a[k >> 1] |= (uint32_t)((const uint16_t*)p)[i + k] << (16 * (k & 1));
  }
  return r;
}
__device__ __forceinline__ void store8(float* p, int64_t i, int have, const float (&x)[8]) {
  if (have >= 8) {
    store_nt<f4_any>(p + i, f4{x[0], x[1], x[2], x[3]});
    store_nt<f4_any>(p + i + 4, f4{x[4], x[5], x[6], x[7]});
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < have) p[i + k] = x[k];
  }
}
__device__ __forceinline__ void store8(uint16_t* p, int64_t i, int have, u4 c) {
  if (have >= 8) {
    store_nt<u4_half>(p + i, c);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < have) p[i + k] = (uint16_t)(c[k >> 1] >> (16 * (k & 1)));
  }
}
__device__ __forceinline__ u2 load8_codes(const uint8_t* p, int64_t i, int have) {
  if (have >= 8) return load_nt<u2_byte>(p + i);
  u2 c = {0u, 0u};
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (k < have) c[k >> 2] |= (uint32_t)p[i + k] << (8 * (k & 3));
  return c;
}
__device__ __forceinline__ void store8(uint8_t* p, int64_t i, int have, u2 c) {
  if (have >= 8) {
    store_nt<u2_byte>(p + i, c);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < have) p[i + k] = (uint8_t)(c[k >> 2] >> (8 * (k & 3)));
  }
}

// Values of eight E4M3 codes times their block's scale (exact).
__device__ __forceinline__ void decode8(u2 c, uint32_t code, float (&x)[8]) {
  const float s = dec_e8m0(code);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const f2v a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[h], false);
    const f2v b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[h], true);
    x[4 * h] = a.x * s;
    x[4 * h + 1] = a.y * s;
    x[4 * h + 2] = b.x * s;
    x[4 * h + 3] = b.y * s;
  }
}

// Bits of the largest magnitude of the block that 16 lanes hold: of finite
// values the maximum of floats, whose operands' signs cost nothing; NaN needs
// the order of the bits.
__device__ __forceinline__ uint32_t block_amax(const float (&x)[8], bool finite) {
  uint32_t amax = 0u;
  if (__builtin_expect(finite, 1)) {
    float f = __builtin_fabsf(x[0]);
#pragma unroll
    for (int k = 1; k < 8; ++k) f = __builtin_fmaxf(f, __builtin_fabsf(x[k]));
    amax = __float_as_uint(f);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t b = __float_as_uint(x[k]) & 0x7FFFFFFFu;
      amax = b > amax ? b : amax;
    }
  }
  return row_max(amax);
}

// Eight values to codes of a block with this scale (so none is above 448),
// rounded stochastically by the draws of a Philox block.  ROOT: values are not
// negative, one above zero is not rounded to zero, and the bytes of each draw
// are exchanged.
template <bool ROOT>
__device__ __forceinline__ u2 encode8(const float (&x)[8], u4 draw, uint32_t code) {
  const float inv = pow2_inverse(code);
  u2 c;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t q = 0u;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t word = draw[2 * h + k / 2];
      // the draw in the high half, zeros below: bytes 0 1, or 1 0, of its half
      const uint32_t bytes = (k % 2 ? (ROOT ? 0x0203u : 0x0302u) : (ROOT ? 0x0001u : 0x0100u)) << 16;
      const uint32_t r = __builtin_amdgcn_perm(0u, word, bytes | 0x0C0Cu);
      float y = x[4 * h + k] * inv;
      // y below 2^-9 becomes 2^-9, but for zero (a root above it is at least 2^-75,
      // and the inverse of a scale that it may have with one of 2^64 2^-56)
      if (ROOT) y = __builtin_amdgcn_fmed3f(y, 0x1p-9f, y * 0x1p127f);
      q = k == 0   ? (uint32_t)__builtin_amdgcn_cvt_sr_fp8_f32(y, (int)r, (int)q, 0)
          : k == 1 ? (uint32_t)__builtin_amdgcn_cvt_sr_fp8_f32(y, (int)r, (int)q, 1)
          : k == 2 ? (uint32_t)__builtin_amdgcn_cvt_sr_fp8_f32(y, (int)r, (int)q, 2)
                   : (uint32_t)__builtin_amdgcn_cvt_sr_fp8_f32(y, (int)r, (int)q, 3);
    }
    c[h] = q;
  }
  return code == 255u ? u2{0u, 0u} : c;
}

// The update of eight elements: m and v in place, r = sqrt(v), the new weights;
// false if an m or v may be infinite or a NaN.
//
// In the common range by the square root and division of exact.h, about half
// the instructions of the general ones, with the intermediates moved into
// their ranges by powers of two that leave again in products that are there
// anyway (m by 2^64, v by 2^80; r comes out 2^40 times, the quotient 2^64 times
// larger).  Each operation stays one rounding of the same real number but
// for a v below 2^-126 (a denormal): its root, below 2^-63, may be half
// again too large.  `usable` sees to it that such a root, with its factor, is less
// than half a unit in the last place of eps, so that the sum with eps is eps for
// either root; where the root would be stored (every root of the block is small) it
// is taken again.  Anything else outside takes the general operations: w, m or v
// from 2^26 on, infinities, NaN, hyper-parameters beyond `usable`.
template <bool S8>
__device__ __forceinline__ bool adamw8(const float (&w)[8], const float (&g)[8], float (&m)[8],
                                       float (&v)[8], float (&r)[8], float (&wn)[8], float c,
                                       const AdamScalars& s) {
  using namespace madd_exact;
  const float alr = fabsf(s.lr);
  // (1.5 2^-63 ir2 <= 0.75 2^-25 eps, half a unit of eps or less: ir2 <= 2^37 eps)
  const bool usable = s.eps >= 0x1p-38f && s.eps < 0x1p20f && s.ir2 < 0x1p20f &&
                      s.ir2 * 0x1p-37f <= s.eps &&
                      (alr == 0.0f || (alr >= 0x1p-60f && alr < 0x1p20f));
  float hi = 0.0f;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float a = g[k] * c;
    m[k] = s.b1 * m[k] + s.omb1 * a;
    v[k] = s.b2 * v[k] + s.omb2 * (a * a);
    const float mv = __builtin_elementwise_maximum(__builtin_fabsf(m[k]), v[k]);
    hi = __builtin_elementwise_maximum(mv, hi);
    hi = __builtin_elementwise_maximum(__builtin_fabsf(w[k]), hi);
  }
  const bool common = hi < 0x1p26f;
  if (__builtin_expect(usable && common, 1)) {
    const float ir2 = s.ir2 * kTwoM40, lr = s.lr * kTwoM64;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float root = sqrt_in_range(v[k] * 0x1p80f);
      const float q = div_in_range(m[k] * kTwo64, root * ir2 + s.eps);
      wn[k] = w[k] * s.decay - lr * q;
      if (S8) r[k] = root * kTwoM40;
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      r[k] = sqrtf(v[k]);
      wn[k] = w[k] * s.decay - s.lr * (m[k] / (r[k] * s.ir2 + s.eps));
      wn[k] = canon_nan(wn[k]);
    }
  }
  return common;
}

// One pass over a list of tensors, one launch for kAdamList of them; a thread has
// eight elements, sixteen lanes a block of the 8-bit states.
//   a = c g,  m' = b1 m + (1 - b1) a,  v' = b2 v + (1 - b2) a^2
//   w' = w (1 - lr decay) - lr / (1 - b1^t) m' / (sqrt(v') / sqrt(1 - b2^t) + eps)
// each operation rounded to fp32; bf16 weights and 8-bit states (m' and sqrt(v'), half
// of v's exponent range in E4M3's) are rounded last, the states stochastically, as
// what is below half a code would otherwise never add up.
// fp32 states are bound by memory: 1.2e8 fp32 weights with bf16 gradients and
// copies take 673 us, 5.2 TB/s.
// 8-bit ones by memory and by operations at once: 1.1e9 bf16 elements 2.17 ms, 5.1
// TB/s, with about as long in the vector units; eight waves a SIMD hide the one
// behind the other best (four 2.78 ms, three 3.45).
template <int WF, int GF, bool S8, bool SR, bool COPY>
__global__ __launch_bounds__(kAdamThreads) void adamw_kernel(AdamList l, const float* gscale) {
  const float c = gscale ? *gscale : 1.0f;
  if (c != c) return;  // a non-finite gradient norm: the step leaves everything as it is
  const AdamScalars& s = l.s;
  const AdamTensor& t = l.t[find_tensor(l, (int32_t)blockIdx.x)];
  const int64_t i = (int64_t)((int32_t)blockIdx.x - t.chunk0) * kAdamChunk + threadIdx.x * kAdamOwn;
  const int64_t left = t.n - i;
  const int have = left >= kAdamOwn ? kAdamOwn : (left > 0 ? (int)left : 0);

  float w[8], g[8], m[8], v[8];
  const Raw8<WF> wr = load8<WF>(t.w, i, have);
  constexpr int kGrad = GF == GF_FP32 ? WF_FP32 : WF_BF16;
  const Raw8<kGrad> gr = load8<kGrad>(t.g, i, have);
  uint32_t sm = 127u, sr = 127u;
  if constexpr (S8) {
    const u2 mr = load8_codes((const uint8_t*)t.m, i, have);
    const u2 vr = load8_codes((const uint8_t*)t.v, i, have);
    if (have > 0) {
      sm = t.scales[2 * (i / kFp8Block)];
      sr = t.scales[2 * (i / kFp8Block) + 1];
    }
    decode8(mr, sm, m);
    decode8(vr, sr, v);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = v[k] * v[k];
  } else {
    const Raw8<WF_FP32> mr = load8<WF_FP32>(t.m, i, have), vr = load8<WF_FP32>(t.v, i, have);
    mr.values(m);
    vr.values(v);
  }
  wr.values(w);
  gr.values(g);

  float r[8], wn[8];
  const bool finite = adamw8<S8>(w, g, m, v, r, wn, c, s);

  const u4 key = {(uint32_t)(t.group0 + i / 8), (uint32_t)((t.group0 + i / 8) >> 32), s.t, 0u};
  if constexpr (WF == WF_FP32) {
    store8((float*)t.w, i, have, wn);
    if constexpr (COPY) {
      if (t.copy) {
        u4 o;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          o[k] = enc_bf16x2(wn[2 * k], wn[2 * k + 1], false, 0u, 0u);
        store8(t.copy, i, have, o);
      }
    }
  } else {
    u4 draw = {0u, 0u, 0u, 0u}, o;
    if constexpr (SR) draw = philox10(key, s.key0, s.key1);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      o[k] = enc_bf16x2(wn[2 * k], wn[2 * k + 1], SR, draw[k] & 0xFFFFu,
                        draw[k] >> 16);
    store8((uint16_t*)t.w, i, have, o);
  }
  if constexpr (S8) {
    const u4 draw = philox10(u4{key[0], key[1], key[2], 1u}, s.key0, s.key1);
    uint32_t top = block_amax(r, finite);
    if (__builtin_expect(top < __float_as_uint(0x1p-40f) && top != 0u, 0)) {
#pragma unroll
      for (int k = 0; k < 8; ++k) r[k] = sqrtf(v[k]);
      top = block_amax(r, finite);
    }
    sm = pow2_scale<WF_E4M3>(block_amax(m, finite));
    sr = pow2_scale<WF_E4M3>(top);
    const u2 qm = encode8<false>(m, draw, sm), qr = encode8<true>(r, draw, sr);
    store8((uint8_t*)t.m, i, have, qm);
    store8((uint8_t*)t.v, i, have, qr);
    if (have > 0 && threadIdx.x % 16 == 0) {
      t.scales[2 * (i / kFp8Block)] = (uint8_t)sm;
      t.scales[2 * (i / kFp8Block) + 1] = (uint8_t)sr;
    }
  } else {
    store8((float*)t.m, i, have, m);
    store8((float*)t.v, i, have, v);
  }
}

// ---------------------------------------------------------------------------
// Global gradient norm
// ---------------------------------------------------------------------------

// Two launches: a partial sum from every workgroup, then one workgroup adds them in
// a fixed order.  Bound by memory: 1.2e8 bf16 gradients 49 us with both launches
// (5.0 TB/s), 1.1e9 of them 387 us (5.7 TB/s).
constexpr int kNormThreads = 256;
constexpr int kNormList = 160;
constexpr int64_t kNormUnit = kNormThreads * 8;  // a workgroup's share is a multiple of
constexpr int64_t kNormPartials = 4096;  // about as many partial sums

struct NormTensor {
  const void* g;
  int64_t n;
  int32_t chunk0;
  int32_t gfmt;
};
struct NormList {
  int64_t chunk;  // elements of a workgroup
  int32_t count, pad;
  NormTensor t[kNormList];
};
static_assert(sizeof(NormList) <= 4000, "kernel arguments");

// Sum over a workgroup of THREADS threads, in thread 0: by halves within a wave,
// then wave by wave.
template <int THREADS>
__device__ __forceinline__ double block_sum(double x) {
  __shared__ double waves[THREADS / 64];
#pragma unroll
  for (int h = 32; h > 0; h >>= 1) x += __shfl_xor(x, h, 64);
  if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = x;
  __syncthreads();
  double sum = waves[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) sum += waves[w];
  return sum;
}

// Squares are added in 64 bits: those of every fp32 value are in range, and the
// sum is right to fp32's last bit.  It costs 2% against 32 bits (7 us of a 1.1e9
// element list's 387).
template <int F>
__device__ __forceinline__ void square_sums(const void* g, int64_t i, int64_t end, double (&a)[8]) {
  for (; i < end; i += kNormThreads * 8) {
    float x[8];
    const int64_t left = end - i;
    load8<F>(g, i, left >= 8 ? 8 : (int)left).values(x);
#pragma unroll
    for (int k = 0; k < 8; ++k) a[k] = fma((double)x[k], (double)x[k], a[k]);
  }
}

__global__ __launch_bounds__(kNormThreads) void norm_partial_kernel(NormList l, double* partial) {
  const NormTensor& t = l.t[find_tensor(l, (int32_t)blockIdx.x)];
  const int64_t begin = (int64_t)((int32_t)blockIdx.x - t.chunk0) * l.chunk;
  const int64_t end = begin + l.chunk < t.n ? begin + l.chunk : t.n;
  double a[8] = {0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0};
  if (t.gfmt == GF_FP32) square_sums<WF_FP32>(t.g, begin + threadIdx.x * 8, end, a);
  else square_sums<WF_BF16>(t.g, begin + threadIdx.x * 8, end, a);
  double sum = 0.0;
#pragma unroll
  for (int k = 0; k < 8; ++k) sum += a[k];
  sum = block_sum<kNormThreads>(sum);
  if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

__global__ __launch_bounds__(1024) void norm_final_kernel(const double* partial, int64_t n,
                                                          float max_norm, float* out) {
  double sum = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += 1024) sum += partial[i];
  sum = block_sum<1024>(sum);
  if (threadIdx.x == 0) {
    const float norm = (float)sqrt(sum);
    out[0] = norm;
    out[1] = isfinite(norm) ? (norm <= max_norm ? 1.0f : max_norm / norm) : NAN;
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

constexpr int64_t kMaxElements = (int64_t)1 << 60;
constexpr int64_t kAdamMost = most_workgroups(kAdamThreads);  // of a launch, 3.4e10 elements

typedef void (*adamw_fn)(AdamList, const float*);

template <int WF, int GF, bool S8>
adamw_fn pick_adamw(bool sr, bool copy) {
  if constexpr (WF == WF_FP32)
    return copy ? adamw_kernel<WF, GF, S8, false, true> : adamw_kernel<WF, GF, S8, false, false>;
  else
    return sr ? adamw_kernel<WF, GF, S8, true, false> : adamw_kernel<WF, GF, S8, false, false>;
}
template <int WF>
adamw_fn pick_adamw(int32_t gfmt, int32_t sfmt, bool sr, bool copy) {
  if (gfmt == MADD_G_FP32)
    return sfmt == MADD_A_8BIT ? pick_adamw<WF, GF_FP32, true>(sr, copy)
                               : pick_adamw<WF, GF_FP32, false>(sr, copy);
  return sfmt == MADD_A_8BIT ? pick_adamw<WF, GF_BF16, true>(sr, copy)
                             : pick_adamw<WF, GF_BF16, false>(sr, copy);
}

static int32_t check_adamw(const madd_adamw_hparams* hp) {
  if (!hp) return MADD_EINVAL;
  if (!(hp->beta1 >= 0.0 && hp->beta1 < 1.0) || !(hp->beta2 >= 0.0 && hp->beta2 < 1.0))
    return MADD_EINVAL;
  if (!(hp->eps >= 0.0) || !std::isfinite(hp->lr) || !std::isfinite(hp->weight_decay))
    return MADD_EINVAL;
  if (hp->rounding != MADD_ROUND_RNE && hp->rounding != MADD_ROUND_SR) return MADD_EINVAL;
  if (hp->step < 1 || hp->step > (int64_t)0xFFFFFFFFll) return MADD_EINVAL;
  return MADD_OK;
}

static AdamScalars adamw_scalars(const madd_adamw_hparams& hp) {
  AdamScalars s;
  const double t = (double)hp.step;
  s.b1 = (float)hp.beta1;
  s.omb1 = (float)(1.0 - hp.beta1);
  s.b2 = (float)hp.beta2;
  s.omb2 = (float)(1.0 - hp.beta2);
  s.decay = (float)(1.0 - hp.lr * hp.weight_decay);
  s.lr = (float)(hp.lr / (1.0 - pow(hp.beta1, t)));
  s.ir2 = (float)(1.0 / sqrt(1.0 - pow(hp.beta2, t)));
  s.eps = (float)hp.eps;
  s.key0 = (uint32_t)hp.seed;
  s.key1 = (uint32_t)(hp.seed >> 32);
  s.t = (uint32_t)hp.step;
  return s;
}

static int64_t norm_chunk(int64_t total) {
  const int64_t per = (total + kNormPartials - 1) / kNormPartials;
  return (per + kNormUnit - 1) / kNormUnit * kNormUnit;
}

static int32_t norm_plan(int32_t ntensors, const int64_t* numel, int64_t* chunk,
                         int64_t* partials) {
  if (ntensors < 0 || (ntensors > 0 && !numel)) return MADD_EINVAL;
  int64_t total = 0;
  for (int32_t i = 0; i < ntensors; ++i) {
    if (numel[i] < 0 || numel[i] > kMaxElements - total) return MADD_EINVAL;
    total += numel[i];
  }
  *chunk = norm_chunk(total);
  *partials = 0;
  for (int32_t i = 0; i < ntensors; ++i)
    if (numel[i] > 0) *partials += (numel[i] + *chunk - 1) / *chunk;
  return MADD_OK;
}

}  // namespace madd_detail

using namespace madd_detail;

extern "C" {

int32_t madd_adamw_step(int32_t ntensors, void* const* w, int32_t wfmt, uint16_t* const* copy,
                        const void* const* g, int32_t gfmt, void* const* m, void* const* v,
                        uint8_t* const* scales, int32_t sfmt, const int64_t* numel,
                        int64_t index_base, const madd_adamw_hparams* hp, const float* grad_scale,
                        void* stream) {
  int32_t rc = check_adamw(hp);
  if (rc != MADD_OK) return rc;
  if (ntensors < 0 || (wfmt != MADD_W_FP32 && wfmt != MADD_W_BF16)) return MADD_EINVAL;
  if (gfmt != MADD_G_FP32 && gfmt != MADD_G_BF16) return MADD_EINVAL;
  if (sfmt != MADD_A_FP32 && sfmt != MADD_A_8BIT) return MADD_EINVAL;
  if (index_base < 0 || index_base % kFp8Block != 0) return MADD_EINVAL;
  if (((uintptr_t)grad_scale & 3u) != 0) return MADD_EALIGN;
  if (ntensors == 0) return MADD_OK;
  if (!w || !g || !m || !v || !numel || (sfmt == MADD_A_8BIT && !scales)) return MADD_EINVAL;
  const bool f32 = wfmt == MADD_W_FP32;
  bool any_copy = false;
  int64_t total = 0;
  for (int32_t i = 0; i < ntensors; ++i) {
    const int64_t n = numel[i];
    if (n < 0 || n > kMaxElements) return MADD_EINVAL;
    if (n == 0) continue;
    if (!w[i] || !g[i] || !m[i] || !v[i] || (sfmt == MADD_A_8BIT && !scales[i]))
      return MADD_EINVAL;
    uint16_t* cp = copy ? copy[i] : nullptr;
    if (cp && !f32) return MADD_EINVAL;  // bf16 weights are their own compute copy
    any_copy = any_copy || cp;
    const uint64_t u = (uint64_t)n, sb = sfmt == MADD_A_8BIT ? u : 4u * u;
    const uint64_t gb = (gfmt == MADD_G_FP32 ? 4u : 2u) * u;
    const Range r[7] = {{g[i], gb},        {grad_scale, 4u}, {w[i], (f32 ? 4u : 2u) * u},
                        {m[i], sb},        {v[i], sb},       {cp, 2u * u},
                        {sfmt == MADD_A_8BIT ? scales[i] : nullptr,
                         2u * ((u + kFp8Block - 1) / kFp8Block)}};
    if (!writes_are_apart(r, 7, 2)) return MADD_EINVAL;
    const uintptr_t wa = f32 ? 3u : 1u, ga = gfmt == MADD_G_FP32 ? 3u : 1u;
    const uintptr_t sa = sfmt == MADD_A_8BIT ? 0u : 3u;
    if (((uintptr_t)w[i] & wa) || ((uintptr_t)g[i] & ga) || ((uintptr_t)m[i] & sa) ||
        ((uintptr_t)v[i] & sa) || ((uintptr_t)cp & 1u))
      return MADD_EALIGN;
    const int64_t whole = (n + kFp8Block - 1) / kFp8Block * kFp8Block;
    if (whole > INT64_MAX - index_base - total) return MADD_EINVAL;
    if ((n + kAdamChunk - 1) / kAdamChunk > kAdamMost) return MADD_EUNSUPPORTED;
    total += whole;
  }
  const bool sr = hp->rounding == MADD_ROUND_SR;
  const adamw_fn fn = f32 ? pick_adamw<WF_FP32>(gfmt, sfmt, sr, any_copy)
                          : pick_adamw<WF_BF16>(gfmt, sfmt, sr, any_copy);
  AdamList l;
  memset(&l, 0, sizeof(l));
  l.s = adamw_scalars(*hp);
  int64_t chunks = 0, base = index_base;
  auto flush = [&]() {
    int32_t st = MADD_OK;
    if (l.count > 0)
      st = launch_kernel(fn, dim3((unsigned)chunks), dim3(kAdamThreads), (hipStream_t)stream, l,
                         grad_scale);
    l.count = 0;
    chunks = 0;
    return st;
  };
  for (int32_t i = 0; i < ntensors; ++i) {
    const int64_t n = numel[i];
    if (n == 0) continue;
    const int64_t nch = (n + kAdamChunk - 1) / kAdamChunk;
    if (l.count == kAdamList || chunks + nch > kAdamMost) {
      rc = flush();
      if (rc != MADD_OK) return rc;
    }
    AdamTensor& d = l.t[l.count++];
    d.w = w[i];
    d.g = g[i];
    d.m = m[i];
    d.v = v[i];
    d.scales = sfmt == MADD_A_8BIT ? scales[i] : nullptr;
    d.copy = copy ? copy[i] : nullptr;
    d.n = n;
    d.group0 = base / 8;
    d.chunk0 = (int32_t)chunks;
    chunks += nch;
    base += (n + kFp8Block - 1) / kFp8Block * kFp8Block;
  }
  return flush();
}

int64_t madd_grad_norm_workspace(int32_t ntensors, const int64_t* numel) {
  int64_t chunk, partials;
  if (norm_plan(ntensors, numel, &chunk, &partials) != MADD_OK) return -1;
  return 8 * (partials > 0 ? partials : 1);
}

int32_t madd_grad_norm(int32_t ntensors, const void* const* g, const int32_t* gfmt,
                       const int64_t* numel, float max_norm, void* workspace, float* out,
                       void* stream) {
  int64_t chunk, partials;
  int32_t rc = norm_plan(ntensors, numel, &chunk, &partials);
  if (rc != MADD_OK) return rc;
  if (!(max_norm > 0.0f) || !out || !workspace) return MADD_EINVAL;
  if (ntensors > 0 && (!g || !gfmt)) return MADD_EINVAL;
  if (((uintptr_t)workspace & 7u) || ((uintptr_t)out & 3u)) return MADD_EALIGN;
  const uint64_t ws = 8u * (uint64_t)(partials > 0 ? partials : 1);
  if (partials > 0x7FFFFFFFll) return MADD_EUNSUPPORTED;
  for (int32_t i = 0; i < ntensors; ++i) {
    if (numel[i] == 0) continue;
    if (!g[i] || (gfmt[i] != MADD_G_FP32 && gfmt[i] != MADD_G_BF16)) return MADD_EINVAL;
    const uint64_t b = gfmt[i] == MADD_G_FP32 ? 4u : 2u;
    if ((uintptr_t)g[i] & (b - 1u)) return MADD_EALIGN;
    const Range r[3] = {{g[i], b * (uint64_t)numel[i]}, {workspace, ws}, {out, 8u}};
    if (!writes_are_apart(r, 3, 1)) return MADD_EINVAL;
  }
  double* partial = (double*)workspace;
  NormList l;
  memset(&l, 0, sizeof(l));
  l.chunk = chunk;
  int64_t chunks = 0, done = 0;
  auto flush = [&]() {
    int32_t st = MADD_OK;
    if (l.count > 0)
      st = launch_kernel(norm_partial_kernel, dim3((unsigned)chunks), dim3(kNormThreads),
                         (hipStream_t)stream, l, partial + done);
    done += chunks;
    l.count = 0;
    chunks = 0;
    return st;
  };
  for (int32_t i = 0; i < ntensors; ++i) {
    if (numel[i] == 0) continue;
    if (l.count == kNormList) {
      rc = flush();
      if (rc != MADD_OK) return rc;
    }
    NormTensor& d = l.t[l.count++];
    d.g = g[i];
    d.n = numel[i];
    d.chunk0 = (int32_t)chunks;
    d.gfmt = gfmt[i];
    chunks += (numel[i] + chunk - 1) / chunk;
  }
  rc = flush();
  if (rc != MADD_OK) return rc;
  return launch_kernel(norm_final_kernel, dim3(1), dim3(1024), (hipStream_t)stream,
                       (const double*)partial, partials, max_norm, out);
}

}  // extern "C"
