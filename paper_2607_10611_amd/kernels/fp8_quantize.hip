// FP8 blocks of 128 with power-of-two scales, along the rows of a matrix, along
// its columns, or both in one pass (include/madd.h: madd_quantize_fp8):
//   e = the least integer in -127 .. 127 with max|x| <= FMAX 2^e,  q = round(x 2^-e)
// The maximum is one of bit patterns without their signs, so that NaN and infinities
// win it; 2^-e is exact, so q has one rounding (to nearest-even, by the hardware's
// conversion) but where x 2^-e is a denormal fp32 number.  Bound by memory.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "e8m0.h"
#include "elem.h"
#include "launch.h"
#include "madd.h"

namespace madd_detail {

constexpr int kQThreads = 256;
constexpr int kQTile = kFp8Block;  // a workgroup's tile: 128 rows by 128 columns

#define GLOBAL __attribute__((address_space(1)))
typedef u4 u4_half __attribute__((aligned(2)));

// Eight consecutive values of a row as they lie in memory.  They are converted
// apart from the branch that loads them: a conversion inside it would wait for
// this load before the next one is issued.
template <int GF>
struct Raw8;
template <>
struct Raw8<GF_FP32> {
  f4 a, b;
  __device__ __forceinline__ void load(const void* x, int64_t i) {
    a = *(const GLOBAL f4_any*)((const float*)x + i);
    b = *(const GLOBAL f4_any*)((const float*)x + i + 4);
  }
  // The first `have` (1 .. 7) of them and zeros; the last is read in place of those
  // past it, so that the loads need no branches.
  __device__ __forceinline__ void load(const void* x, int64_t i, int have) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float f = ((const GLOBAL float*)x)[i + (k < have ? k : have - 1)];
      (k < 4 ? a : b)[k & 3] = k < have ? f : 0.0f;
    }
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = (k < 4 ? a : b)[k & 3];
  }
};
template <>
struct Raw8<GF_BF16> {
  u4 a;
  __device__ __forceinline__ void load(const void* x, int64_t i) {
    a = *(const GLOBAL u4_half*)((const uint16_t*)x + i);
  }
  __device__ __forceinline__ void load(const void* x, int64_t i, int have) {
    uint32_t c[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint16_t f = ((const GLOBAL uint16_t*)x)[i + (k < have ? k : have - 1)];
      c[k] = k < have ? f : 0u;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) a[k] = c[2 * k] | c[2 * k + 1] << 16;
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      v[k] = __uint_as_float((k & 1) ? (a[k >> 1] & 0xFFFF0000u) : (a[k >> 1] << 16));
  }
};

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }

// Codes of eight values of a block with scale `code`; none if it is the NaN one.
template <int WF>
__device__ __forceinline__ u2 codes8(const float (&v)[8], uint32_t code) {
  const float inv = pow2_inverse(code);
  const uint32_t none[4] = {0u, 0u, 0u, 0u};
  u2 q;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float y[4] = {v[4 * h] * inv, v[4 * h + 1] * inv, v[4 * h + 2] * inv, v[4 * h + 3] * inv};
    q[h] = enc_fp8x4<WF, false>(y, none);
  }
  return code == 255u ? u2{0u, 0u} : q;
}

// Blocks along the rows: 16 lanes hold a block, so its maximum is four rotations
// within a row of lanes.  8192x4096 bf16: 17.9 us, 5.6 TB/s.
template <int WF, int GF>
__global__ __launch_bounds__(kQThreads) void quantize_rows_kernel(const void* x, int64_t rows,
                                                                  int64_t cols, int64_t ldx,
                                                                  uint8_t* q, uint8_t* s) {
  const int64_t kb = (cols + kFp8Block - 1) / kFp8Block, blocks = rows * kb;
  for (int64_t b = (int64_t)blockIdx.x * 16 + threadIdx.x / 16; b < blocks;
       b += (int64_t)gridDim.x * 16) {
    const int64_t row = b / kb, at = (b - row * kb) * kFp8Block + (threadIdx.x % 16) * 8;
    const int64_t left = cols - at;
    const int have = left >= 8 ? 8 : (left > 0 ? (int)left : 0);
    Raw8<GF> raw = {};
    if (have == 8) raw.load(x, row * ldx + at);
    else if (have > 0) raw.load(x, row * ldx + at, have);
    float v[8];
    raw.values(v);
    uint32_t amax = 0u;
#pragma unroll
    for (int k = 0; k < 8; ++k) amax = larger(amax, magnitude(v[k]));
    const uint32_t code = pow2_scale<WF>(row_max(amax));
    *(GLOBAL u2*)(q + row * kb * kFp8Block + at) = codes8<WF>(v, code);
    if (threadIdx.x % 16 == 0) s[b] = (uint8_t)code;
  }
}

// Blocks along the columns, and along the rows too with ROWS: a workgroup
// holds a 128x128 tile in registers, each thread eight rows of eight columns, so the
// matrix is read once; LDS joins the columns' maxima and turns their codes, that
// rows of 128 bytes are written.  8192x4096 bf16: columns 17.1 us (5.9 TB/s), both
// 26.4 us (5.1 TB/s); two launches in its place 35.
template <int WF, int GF, bool ROWS>
__global__ __launch_bounds__(kQThreads) void quantize_tile_kernel(const void* x, int64_t rows,
                                                                  int64_t cols, int64_t ldx,
                                                                  uint8_t* q, uint8_t* s,
                                                                  uint8_t* qt, uint8_t* st) {
  __shared__ __align__(16) uint32_t peak[16][kQTile];  // largest magnitude of eight rows
  __shared__ __align__(16) u2 turned[kQTile][16];  // column codes, eight rows each
  const int64_t kb = (cols + kQTile - 1) / kQTile, rb = (rows + kQTile - 1) / kQTile;
  const int64_t tr = blockIdx.x / kb, tc = blockIdx.x - tr * kb;
  const int lane = threadIdx.x % 16, group = threadIdx.x / 16;
  const int64_t row0 = tr * kQTile + group * 8, col0 = tc * kQTile + lane * 8;
  const int64_t left = cols - col0;
  const int have = left >= 8 ? 8 : (left > 0 ? (int)left : 0);
  Raw8<GF> raw[8] = {};
  const int64_t last = rows - 1;  // read in place of rows past it
  if (have == 8) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      raw[i].load(x, (row0 + i < last ? row0 + i : last) * ldx + col0);
  } else if (have > 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      raw[i].load(x, (row0 + i < last ? row0 + i : last) * ldx + col0, have);
  }
  if (row0 + 8 > rows) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (row0 + i >= rows) raw[i] = {};
  }
  float v[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) raw[i].values(v[i]);
  if constexpr (ROWS) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t amax = 0u;
#pragma unroll
      for (int k = 0; k < 8; ++k) amax = larger(amax, magnitude(v[i][k]));
      const uint32_t code = pow2_scale<WF>(row_max(amax));
      if (row0 + i < rows) {
        *(GLOBAL u2*)(q + (row0 + i) * kb * kFp8Block + col0) = codes8<WF>(v[i], code);
        if (lane == 0) s[(row0 + i) * kb + tc] = (uint8_t)code;
      }
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    u4 amax = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) amax[k] = larger(amax[k], magnitude(v[i][4 * h + k]));
    *(u4*)&peak[group][lane * 8 + 4 * h] = amax;
  }
  __syncthreads();
  if (threadIdx.x < kQTile) {
    uint32_t amax = 0u;
#pragma unroll
    for (int j = 0; j < 16; ++j) amax = larger(amax, peak[j][threadIdx.x]);
    const uint32_t code = pow2_scale<WF>(amax);
    peak[0][threadIdx.x] = code;
    const int64_t col = tc * kQTile + threadIdx.x;
    if (col < cols) st[col * rb + tr] = (uint8_t)code;
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const u4 code = *(const u4*)&peak[0][lane * 8 + 4 * h];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int k = 4 * h + i;
      const float c[8] = {v[0][k], v[1][k], v[2][k], v[3][k], v[4][k], v[5][k], v[6][k], v[7][k]};
      // eight columns apart, lanes would meet in the same banks: the slots of a
      // column are permuted by its lane
      turned[lane * 8 + k][group ^ lane] = codes8<WF>(c, code[i]);
    }
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int col = j * 32 + threadIdx.x / 8, part = threadIdx.x % 8, l = col / 8;
    const u2 a = turned[col][(2 * part) ^ l], b = turned[col][(2 * part + 1) ^ l];
    const int64_t at = tc * kQTile + col;
    if (at < cols) *(GLOBAL u4*)(qt + (at * rb + tr) * kFp8Block + part * 16) = u4{a.x, a.y, b.x, b.y};
  }
}

template <int WF, int GF>
int32_t quantize(const void* x, int64_t rows, int64_t cols, int64_t ldx, uint8_t* q, uint8_t* s,
                 uint8_t* qt, uint8_t* st, hipStream_t stream) {
  const int64_t kb = (cols + kQTile - 1) / kQTile, rb = (rows + kQTile - 1) / kQTile;
  if (!qt) {
    const int64_t want = (rows * kb + 15) / 16;
    const unsigned grid = (unsigned)(want < 65536 ? want : 65536);
    return launch_kernel(quantize_rows_kernel<WF, GF>, dim3(grid), dim3(kQThreads), stream, x,
                         rows, cols, ldx, q, s);
  }
  if (rb > 0x7FFFFFFFll / kb) return MADD_EUNSUPPORTED;
  const dim3 grid((unsigned)(rb * kb));
  return q ? launch_kernel(quantize_tile_kernel<WF, GF, true>, grid, dim3(kQThreads), stream, x,
                           rows, cols, ldx, q, s, qt, st)
           : launch_kernel(quantize_tile_kernel<WF, GF, false>, grid, dim3(kQThreads), stream, x,
                           rows, cols, ldx, q, s, qt, st);
}

}  // namespace madd_detail

using namespace madd_detail;

extern "C" int32_t madd_quantize_fp8(const void* x, int32_t xfmt, int64_t rows, int64_t cols,
                                     int64_t ldx, int32_t qfmt, uint8_t* q, uint8_t* qscale,
                                     uint8_t* qt, uint8_t* qtscale, void* stream) {
  if (xfmt != MADD_G_FP32 && xfmt != MADD_G_BF16) return MADD_EINVAL;
  if (qfmt != MADD_W_FP8_E4M3 && qfmt != MADD_W_FP8_E5M2) return MADD_EINVAL;
  constexpr int64_t kMaxDim = (int64_t)1 << 31;
  if (rows < 0 || cols < 0 || rows > kMaxDim || cols > kMaxDim) return MADD_EINVAL;
  if (rows == 0 || cols == 0) return MADD_OK;
  if ((!q && !qt) || !q != !qscale || !qt != !qtscale) return MADD_EINVAL;
  if (!x || ldx < cols || ldx > (int64_t)1 << 40) return MADD_EINVAL;
  const uint64_t xb = xfmt == MADD_G_FP32 ? 4u : 2u;
  if (!rows_fit(rows, ldx, (int64_t)xb)) return MADD_EINVAL;
  if ((uintptr_t)x & (xb - 1u)) return MADD_EALIGN;
  if (((uintptr_t)q & 15u) || ((uintptr_t)qt & 15u)) return MADD_EALIGN;
  const uint64_t r = (uint64_t)rows, c = (uint64_t)cols;
  const uint64_t kb = (c + kFp8Block - 1) / kFp8Block, rb = (r + kFp8Block - 1) / kFp8Block;
  const Range ranges[5] = {{x, xb * ((r - 1) * (uint64_t)ldx + c)},
                           {q, r * kb * kFp8Block}, {qscale, r * kb},
                           {qt, c * rb * kFp8Block}, {qtscale, c * rb}};
  if (!writes_are_apart(ranges, 5, 1)) return MADD_EINVAL;
  hipStream_t st = (hipStream_t)stream;
  if (qfmt == MADD_W_FP8_E4M3)
    return xfmt == MADD_G_FP32
               ? quantize<WF_E4M3, GF_FP32>(x, rows, cols, ldx, q, qscale, qt, qtscale, st)
               : quantize<WF_E4M3, GF_BF16>(x, rows, cols, ldx, q, qscale, qt, qtscale, st);
  return xfmt == MADD_G_FP32
             ? quantize<WF_E5M2, GF_FP32>(x, rows, cols, ldx, q, qscale, qt, qtscale, st)
             : quantize<WF_E5M2, GF_BF16>(x, rows, cols, ldx, q, qscale, qt, qtscale, st);
}
