// Quantiser of the 8-bit products: a matrix [rows, cols] of bf16 or float32 -> e4m3 or e5m2 values with a
// power-of-two scale for each 1 x 128 or 128 x 128 elements, as it stands and / or transposed.
//
//   s = min { 2^k >= 2^-126 : max |x| / s <= top } over the block's finite elements (1 for a block of zeros)
//   q = x / s, rounded to nearest even;  NaN where x is not finite
//
// Powers of two make the division exact, so the format's rounding is the only loss, and cost nothing
// against max / top as scale: the formats are floating point, only their last binade is used less.
//
// HBM-bound: one reading of x serves both outputs (a forward product wants activations in blocks along a
// row, the weight gradient wants them along the tokens, i.e. blocks down a column, transposed).  A thread
// block takes a 128 x 128 tile: 16 lanes hold a row's 128 elements, so that a row's maximum is four
// shuffles and each row is written as 128 consecutive bytes; the tile is kept in shared memory and
// read again down its columns for the transposed output.
#include "common.cuh"
#include "../../include/fax_ops.h"

#include <cuda_fp8.h>

namespace {

constexpr int QT = FAX_FP8_BLOCK;      // tile edge
constexpr int THREADS = 256;

struct QuantParams {
  int rows, cols;
  const void* x; long long ldx;
  uint8_t* q; long long ldq; float* s; long long lds;
  uint8_t* qt; long long ldqt; float* st; long long ldst;
  int square;                          // one scale for the whole tile
  int tiles_c;
};

__device__ __forceinline__ uint32_t finite_abs_bits(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
  return u < 0x7f800000u ? u : 0u;
}
template <int FMT> __device__ __forceinline__ uint32_t scale_field(uint32_t amax) {
  const int f = (int)((amax + 0x1fffffu) >> 23) - (FMT == FAX_FP8_E4M3 ? 8 : 15);
  return amax == 0u ? 127u : (f < 1 ? 1u : (uint32_t)f);
}
__device__ __forceinline__ float pow2_field(uint32_t f) { return __uint_as_float(f << 23); }

// Two values already divided by their scale -> two codes.
template <int FMT> __device__ __forceinline__ uint32_t code2(float a, float b) {
  return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, FMT == FAX_FP8_E4M3 ? __NV_E4M3 : __NV_E5M2);
}
// The conversion saturates: an infinite element is made NaN before it.
__device__ __forceinline__ float inf_to_nan(float x) { return x - x == 0.f ? x : __uint_as_float(0x7fffffffu); }

template <typename T> struct Row8;     // eight consecutive elements
template <> struct Row8<bf16> {
  static __device__ __forceinline__ void load(const bf16* p, float (&v)[8]) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&u);
#pragma unroll
    for (int e = 0; e < 4; ++e) { const float2 f = __bfloat1622float2(h[e]); v[2 * e] = f.x; v[2 * e + 1] = f.y; }
  }
};
template <> struct Row8<float> {
  static __device__ __forceinline__ void load(const float* p, float (&v)[8]) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
};

// VEC: x is 16-byte aligned with a pitch of whole 16-byte vectors.  Outputs: pitches are multiples of 16.
template <typename T, int FMT, bool VEC, bool STRAIGHT, bool TRANSPOSED>
__global__ void __launch_bounds__(THREADS)
fp8_quantize_kernel(const QuantParams p) {
  extern __shared__ uint4 tile_raw[];              // TRANSPOSED: the tile [128][128] of T
  T* tile = reinterpret_cast<T*>(tile_raw);
  __shared__ uint32_t red[THREADS / 32];
  __shared__ uint32_t col_max[TRANSPOSED ? 2 : 1][QT];
  fax_grid_dependency_wait();
  const int tr = blockIdx.x / p.tiles_c, tc = blockIdx.x - tr * p.tiles_c;
  const int r0 = tr * QT, c0 = tc * QT;
  const int sub = threadIdx.x & 15, grp = threadIdx.x >> 4;          // 16 lanes a row, 16 rows at a time
  const int c = c0 + 8 * sub;
  float v[8][8];
  uint32_t am[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + grp + 16 * i;
    const T* src = (const T*)p.x + (size_t)r * p.ldx + c;
    if (r < p.rows && VEC && c + 8 <= p.cols) {
      Row8<T>::load(src, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = (r < p.rows && c + j < p.cols) ? to_f32(src[j]) : 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    uint32_t m = 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, finite_abs_bits(v[i][j]));
    am[i] = m;
    if (TRANSPOSED) {
#pragma unroll
      for (int j = 0; j < 8; j += 16 / (int)sizeof(T)) {
        uint4 u;
        T* e = reinterpret_cast<T*>(&u);
#pragma unroll
        for (int k = 0; k < 16 / (int)sizeof(T); ++k) e[k] = from_f32<T>(v[i][j + k]);
        *reinterpret_cast<uint4*>(tile + (grp + 16 * i) * QT + 8 * sub + j) = u;
      }
    }
  }
  uint32_t all = 0u;                                                 // maximum of the whole tile
  if (p.square) {
#pragma unroll
    for (int i = 0; i < 8; ++i) all = max(all, am[i]);
    all = __reduce_max_sync(0xffffffffu, all);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = all;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) all = max(all, red[w]);
  }
  if (STRAIGHT) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = r0 + grp + 16 * i;
      uint32_t m = am[i];
      if (p.square) {
        m = all;
      } else {
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
      }
      const uint32_t f = scale_field<FMT>(m);
      const float inv = pow2_field(254u - f);
      if (r >= p.rows) continue;
      if (sub == 0 && !p.square) p.s[(size_t)tc * p.lds + r] = pow2_field(f);
      uint2 o;
      uint32_t h[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) h[j] = code2<FMT>(inf_to_nan(v[i][2 * j]) * inv, inf_to_nan(v[i][2 * j + 1]) * inv);
      o.x = h[0] | (h[1] << 16); o.y = h[2] | (h[3] << 16);
      uint8_t* dst = p.q + (size_t)r * p.ldq + c;
      if (c + 8 <= p.cols) {
        *reinterpret_cast<uint2*>(dst) = o;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (c + j < p.cols) dst[j] = (uint8_t)((j < 4 ? o.x : o.y) >> (8 * (j & 3)));
      }
    }
    if (p.square && threadIdx.x == 0) p.s[(size_t)tc * p.lds + tr] = pow2_field(scale_field<FMT>(all));
  }
  if (TRANSPOSED) {
    __syncthreads();
    // a thread takes one column and 16 consecutive rows of it at a time: 16 bytes of the transposed row
    const int col = threadIdx.x & 127, part = threadIdx.x >> 7;      // part 0: row groups 0..3, part 1: 4..7
    float x[4][16];
    uint32_t cm = 0u;
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        x[k][j] = to_f32(tile[(16 * (4 * part + k) + j) * QT + col]);
        cm = max(cm, finite_abs_bits(x[k][j]));
      }
    if (!p.square) {
      col_max[part][col] = cm;
      __syncthreads();
      cm = max(col_max[0][col], col_max[1][col]);
    } else {
      cm = all;
    }
    const uint32_t f = scale_field<FMT>(cm);
    const float inv = pow2_field(254u - f);
    if (c0 + col < p.cols) {
      if (part == 0 && !p.square) p.st[(size_t)tr * p.ldst + c0 + col] = pow2_field(f);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int r = r0 + 16 * (4 * part + k);
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          w[j] = code2<FMT>(inf_to_nan(x[k][4 * j]) * inv, inf_to_nan(x[k][4 * j + 1]) * inv) |
                 (code2<FMT>(inf_to_nan(x[k][4 * j + 2]) * inv, inf_to_nan(x[k][4 * j + 3]) * inv) << 16);
        uint8_t* dst = p.qt + (size_t)(c0 + col) * p.ldqt + r;
        if (r + 16 <= p.rows) {
          *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (r + j < p.rows) dst[j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
        }
      }
    }
    if (p.square && threadIdx.x == 0) p.st[(size_t)tr * p.ldst + tc] = pow2_field(scale_field<FMT>(all));
  }
}

template <typename T, int FMT, bool VEC>
fax_status launch(fax_ctx* ctx, const QuantParams& p, unsigned int blocks) {
  constexpr int tile_bytes = QT * QT * (int)sizeof(T);
  if (p.q && p.qt) {
    static bool done[FAX_MAX_DEVICES] = {};
    FAX_TRY(fax_opt_in_shared_memory(ctx, fp8_quantize_kernel<T, FMT, VEC, true, true>, tile_bytes, done));
    fax_launch(ctx, fp8_quantize_kernel<T, FMT, VEC, true, true>, dim3(blocks), dim3(THREADS), tile_bytes, p);
  } else if (p.q) {
    fax_launch(ctx, fp8_quantize_kernel<T, FMT, VEC, true, false>, dim3(blocks), dim3(THREADS), 0, p);
  } else {
    static bool done[FAX_MAX_DEVICES] = {};
    FAX_TRY(fax_opt_in_shared_memory(ctx, fp8_quantize_kernel<T, FMT, VEC, false, true>, tile_bytes, done));
    fax_launch(ctx, fp8_quantize_kernel<T, FMT, VEC, false, true>, dim3(blocks), dim3(THREADS), tile_bytes, p);
  }
  return fax_after_launch(ctx);
}

}  // namespace

extern "C" fax_status fax_op_fp8_quantize(fax_ctx* ctx, int32_t prec, const fax_fp8_quantize_desc* d) {
  if (!ctx || !d || !d->x || (!d->q && !d->qt)) return FAX_ERR_INVALID_ARG;
  if (prec != FAX_PREC_BF16 && prec != FAX_PREC_FP32_VALIDATE) return FAX_ERR_INVALID_ARG;
  if (d->format != FAX_FP8_E4M3 && d->format != FAX_FP8_E5M2) return FAX_ERR_INVALID_ARG;
  if (d->tile != 1 && d->tile != FAX_FP8_BLOCK) return FAX_ERR_INVALID_ARG;
  if (d->rows <= 0 || d->cols <= 0 || d->ldx < d->cols || !fax_aligned(d->x, fax_elem_size(prec))) return FAX_ERR_INVALID_ARG;
  const int64_t rb = ((int64_t)d->rows + FAX_FP8_BLOCK - 1) / FAX_FP8_BLOCK, cb = ((int64_t)d->cols + FAX_FP8_BLOCK - 1) / FAX_FP8_BLOCK;
  const bool square = d->tile == FAX_FP8_BLOCK;
  if (d->q && (!d->s || d->ldq < d->cols || d->ldq % 16 || !fax_aligned(d->q, 16) || !fax_aligned(d->s, 4) || d->lds < (square ? rb : d->rows)))
    return FAX_ERR_INVALID_ARG;
  if (d->qt && (!d->st || d->ldqt < d->rows || d->ldqt % 16 || !fax_aligned(d->qt, 16) || !fax_aligned(d->st, 4) || d->ldst < (square ? cb : d->cols)))
    return FAX_ERR_INVALID_ARG;
  if (rb * cb > 0x7fffffffLL) return FAX_ERR_UNSUPPORTED_SHAPE;
  QuantParams p;
  p.rows = d->rows; p.cols = d->cols; p.x = d->x; p.ldx = d->ldx;
  p.q = (uint8_t*)d->q; p.ldq = d->ldq; p.s = d->s; p.lds = d->lds;
  p.qt = (uint8_t*)d->qt; p.ldqt = d->ldqt; p.st = d->st; p.ldst = d->ldst;
  p.square = square ? 1 : 0;
  p.tiles_c = (int)cb;
  const size_t es = fax_elem_size(prec);
  FaxProfScope prof(ctx, KC_FP8_QUANT, 0.0, (double)d->rows * d->cols * (es + (d->q ? 1.0 : 0.0) + (d->qt ? 1.0 : 0.0)));
  const bool vec = fax_aligned(d->x, 16) && ((size_t)d->ldx * es) % 16 == 0;
  const unsigned int blocks = (unsigned int)(rb * cb);
  const bool e4 = d->format == FAX_FP8_E4M3;
  if (prec == FAX_PREC_BF16) {
    if (vec) return e4 ? launch<bf16, FAX_FP8_E4M3, true>(ctx, p, blocks) : launch<bf16, FAX_FP8_E5M2, true>(ctx, p, blocks);
    return e4 ? launch<bf16, FAX_FP8_E4M3, false>(ctx, p, blocks) : launch<bf16, FAX_FP8_E5M2, false>(ctx, p, blocks);
  }
  if (vec) return e4 ? launch<float, FAX_FP8_E4M3, true>(ctx, p, blocks) : launch<float, FAX_FP8_E5M2, true>(ctx, p, blocks);
  return e4 ? launch<float, FAX_FP8_E4M3, false>(ctx, p, blocks) : launch<float, FAX_FP8_E5M2, false>(ctx, p, blocks);
}
