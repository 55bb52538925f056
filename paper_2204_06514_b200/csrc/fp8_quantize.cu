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
// block takes a 128 x 128 tile: 8 lanes hold a row's 128 elements, so that a row's maximum is three
// shuffles and each row is written as 128 consecutive bytes; the tile is kept in shared memory and
// read again down its columns, 32 rows of a word a thread, for the transposed output.
//
// What costs is instructions: maxima are taken on the raw words (two bf16 at a time), and elements that are not
// finite are looked for once a tile (their bits are the largest); only a tile that holds one runs the code that
// leaves them out of the maximum and makes them NaN.
#include "common.cuh"
#include "../../include/fax_ops.h"

#include <cuda_fp8.h>

namespace {

constexpr int QT = FAX_FP8_BLOCK;      // tile edge
// Threads of a tile: each has 64 (bf16) or 32 (float) elements, 32 registers of them.
template <typename T> constexpr int THREADS = 128 * (int)sizeof(T);

struct QuantParams {
  int rows, cols;
  const void* x; long long ldx;
  uint8_t* q; long long ldq; float* s; long long lds;
  uint8_t* qt; long long ldqt; float* st; long long ldst;
  int square;                          // one scale for the whole tile
  int tiles_c;
};

template <int FMT> __device__ __forceinline__ uint32_t scale_field(uint32_t amax) {
  const int f = (int)((amax + 0x1fffffu) >> 23) - (FMT == FAX_FP8_E4M3 ? 8 : 15);
  return amax == 0u ? 127u : (f < 1 ? 1u : (uint32_t)f);
}
__device__ __forceinline__ float pow2_field(uint32_t f) { return __uint_as_float(f << 23); }

// Four values already divided by their scale -> four codes.  The conversion saturates: where elements may not be
// finite (BAD), infinities are made NaN before it.
template <int FMT, bool BAD> __device__ __forceinline__ uint32_t code4(float a, float b, float c, float d) {
  if (BAD) {
    const float nan = __uint_as_float(0x7fffffffu);
    a = a - a == 0.f ? a : nan; b = b - b == 0.f ? b : nan; c = c - c == 0.f ? c : nan; d = d - d == 0.f ? d : nan;
  }
  uint32_t r;
  if (FMT == FAX_FP8_E4M3)
    asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}"
        : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
  else
    asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e5m2x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e5m2x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}"
        : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}

// A 32-bit word of the matrix: two bf16 or one float.  Maxima are kept as words too (both halves of a bf16 word).
template <typename T> struct Word;
template <> struct Word<bf16> {
  static constexpr int N = 2;
  static constexpr uint32_t INF_BITS = 0x7f80u;
  template <bool BAD> static __device__ __forceinline__ uint32_t max_abs(uint32_t m, uint32_t w) {
    if (BAD) w = ((w & 0x7fffu) < INF_BITS ? w & 0x7fffu : 0u) | (((w >> 16) & 0x7fffu) < INF_BITS ? w & 0x7fff0000u : 0u);
    uint32_t d;                                    // the larger magnitudes, with signs that nobody reads; a NaN stays
    asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(m), "r"(w));
    return d;
  }
  static __device__ __forceinline__ uint32_t join(uint32_t m) { return max(m & 0x7fffu, (m >> 16) & 0x7fffu); }       // over both halves
  static __device__ __forceinline__ uint32_t half(uint32_t m, int i) { return (i ? m >> 16 : m) & 0x7fffu; }
  static __device__ __forceinline__ uint32_t float_bits(uint32_t m) { return m << 16; }
  static __device__ __forceinline__ float value(uint32_t w, int i) { return __uint_as_float(i ? w & 0xffff0000u : w << 16); }
};
template <> struct Word<float> {
  static constexpr int N = 1;
  static constexpr uint32_t INF_BITS = 0x7f800000u;
  template <bool BAD> static __device__ __forceinline__ uint32_t max_abs(uint32_t m, uint32_t w) {
    w &= 0x7fffffffu;
    if (BAD) w = w < INF_BITS ? w : 0u;
    return max(m, w);
  }
  static __device__ __forceinline__ uint32_t join(uint32_t m) { return m; }
  static __device__ __forceinline__ uint32_t half(uint32_t m, int) { return m; }
  static __device__ __forceinline__ uint32_t float_bits(uint32_t m) { return m; }
  static __device__ __forceinline__ float value(uint32_t w, int) { return __uint_as_float(w); }
};

// A lane holds 16 consecutive elements (RW words) of PASSES rows, ROW_STEP apart; the tile has WPR words a row.
template <typename T> constexpr int PASSES = QT * QT / (THREADS<T> * 16);
template <typename T> constexpr int ROW_STEP = THREADS<T> / 8;
template <typename T> constexpr int RW = 16 * (int)sizeof(T) / 4;
template <typename T> constexpr int WPR = QT * (int)sizeof(T) / 4;

// Place of a row's 16-byte unit in shared memory: eight lanes that write units 2 or 4 apart hit eight different bank groups,
// and 32 lanes that read consecutive words still do.
__device__ __forceinline__ int unit_at(int u) { return u ^ (u >> 3); }

// The rows of the tile in v, quantised; am: their lanes' maxima (taken again where some are not finite).  Returns the
// maximum of the whole tile (square blocks).
template <typename T, int FMT, bool STRAIGHT, bool BAD>
__device__ __forceinline__ uint32_t quantize_rows(const QuantParams& p, const uint32_t (&v)[PASSES<T>][RW<T>], uint32_t (&am)[PASSES<T>], uint32_t* red, int tr, int tc) {
  typedef Word<T> W;
  const int sub = threadIdx.x & 7;
  if (BAD) {
#pragma unroll
    for (int i = 0; i < PASSES<T>; ++i) {
      uint32_t m = 0u;
#pragma unroll
      for (int j = 0; j < RW<T>; ++j) m = W::template max_abs<true>(m, v[i][j]);
      am[i] = W::join(m);
    }
  }
  uint32_t all = 0u;
  if (p.square) {
#pragma unroll
    for (int i = 0; i < PASSES<T>; ++i) all = max(all, am[i]);
    all = __reduce_max_sync(0xffffffffu, all);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = all;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS<T> / 32; ++w) all = max(all, red[w]);
  }
  if (STRAIGHT) {
    const int c = tc * QT + 16 * sub, r0 = tr * QT + (threadIdx.x >> 3);
    uint8_t* dst = p.q + (size_t)r0 * p.ldq + c;
    float* sc = p.s + (size_t)tc * p.lds + r0;
#pragma unroll
    for (int i = 0; i < PASSES<T>; ++i, dst += ROW_STEP<T> * p.ldq) {
      uint32_t m = am[i];
      if (p.square) {
        m = all;
      } else {
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
      }
      const uint32_t f = scale_field<FMT>(W::float_bits(m));
      const float inv = pow2_field(254u - f);
      if (r0 + ROW_STEP<T> * i >= p.rows) continue;
      if (sub == 0 && !p.square) sc[ROW_STEP<T> * i] = pow2_field(f);
      uint32_t o[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = W::value(v[i][(4 * j + e) / W::N], e % W::N) * inv;
        o[j] = code4<FMT, BAD>(y[0], y[1], y[2], y[3]);
      }
      if (c <= p.cols - 16) {                          // c + 16 may pass 32 bits
        *reinterpret_cast<uint4*>(dst) = make_uint4(o[0], o[1], o[2], o[3]);
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (c + j < p.cols) dst[j] = (uint8_t)(o[j >> 2] >> (8 * (j & 3)));
      }
    }
    if (p.square && threadIdx.x == 0) p.s[(size_t)tc * p.lds + tr] = pow2_field(scale_field<FMT>(W::float_bits(all)));
  }
  return all;
}

// The columns of the tile in shared memory: a thread takes one word of each of 32 rows, 32 codes of each column in it.
// The codes go back to shared memory (16 KB over the tile, 16-byte units placed so that neighbouring columns hit different
// banks) and leave it as whole 128-byte rows: written from registers, 32 bytes a lane, the rows cost 5 us of 26.7 (8192 x 4096).
template <typename T, int FMT, bool BAD>
__device__ __forceinline__ void quantize_columns(const QuantParams& p, uint4* tile_raw, uint32_t* col_max, uint32_t all, int tr, int tc) {
  typedef Word<T> W;
  constexpr int GROUPS = QT / 32;
  static_assert(THREADS<T> == GROUPS * WPR<T>, "a word of 32 rows a thread");
  const uint32_t* tile = reinterpret_cast<const uint32_t*>(tile_raw);
  const int word = threadIdx.x % WPR<T>, group = threadIdx.x / WPR<T>;
  uint32_t w[32];
#pragma unroll
  for (int j = 0; j < 32; ++j) w[j] = tile[(group * 32 + j) * WPR<T> + 4 * unit_at(word >> 2) + (word & 3)];
  uint32_t m = 0u;
  if (!p.square) {
#pragma unroll
    for (int j = 0; j < 32; ++j) m = W::template max_abs<BAD>(m, w[j]);
    col_max[group * WPR<T> + word] = m;
  }
  __syncthreads();                                 // every thread has read the tile
  if (!p.square) {
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) m = W::template max_abs<false>(m, col_max[g * WPR<T> + word]);
  }
#pragma unroll
  for (int k = 0; k < W::N; ++k) {
    const uint32_t f = scale_field<FMT>(W::float_bits(p.square ? all : W::half(m, k)));
    const int col = word * W::N + k;
    const float inv = pow2_field(254u - f);
    if (group == 0 && !p.square && tc * QT + col < p.cols) p.st[(size_t)tr * p.ldst + tc * QT + col] = pow2_field(f);
    uint32_t o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      o[j] = code4<FMT, BAD>(W::value(w[4 * j], k) * inv, W::value(w[4 * j + 1], k) * inv, W::value(w[4 * j + 2], k) * inv, W::value(w[4 * j + 3], k) * inv);
#pragma unroll
    for (int h = 0; h < 2; ++h) tile_raw[col * 8 + ((2 * group + h) ^ (word & 7))] = make_uint4(o[4 * h], o[4 * h + 1], o[4 * h + 2], o[4 * h + 3]);
  }
  __syncthreads();
#pragma unroll
  for (int i = threadIdx.x; i < QT * 8; i += THREADS<T>) {
    const int col = i >> 3, unit = i & 7;
    const int c = tc * QT + col, r = tr * QT + 16 * unit;
    if (c >= p.cols) continue;
    const uint4 u = tile_raw[col * 8 + (unit ^ ((col / W::N) & 7))];
    uint8_t* dst = p.qt + (size_t)c * p.ldqt + r;
    if (r <= p.rows - 16) {
      *reinterpret_cast<uint4*>(dst) = u;
    } else {
      const uint32_t x[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (r + j < p.rows) dst[j] = (uint8_t)(x[j >> 2] >> (8 * (j & 3)));
    }
  }
  if (p.square && threadIdx.x == 0) p.st[(size_t)tr * p.ldst + tc] = pow2_field(scale_field<FMT>(W::float_bits(all)));
}

// VEC: x is 16-byte aligned with a pitch of whole 16-byte vectors.  Outputs: pitches are multiples of 16.
// Several blocks an SM: one's columns run under another's loads.
template <typename T, int FMT, bool VEC, bool STRAIGHT, bool TRANSPOSED>
__global__ void __launch_bounds__(THREADS<T>, sizeof(T) == 2 ? 4 : 2)
fp8_quantize_kernel(const QuantParams p) {
  typedef Word<T> W;
  extern __shared__ uint4 tile_raw[];              // TRANSPOSED: the tile [128][128] of T
  __shared__ uint32_t red[THREADS<T> / 32];
  __shared__ uint32_t col_max[TRANSPOSED ? THREADS<T> : 1];
  fax_grid_dependency_wait();
  const int tr = blockIdx.x / p.tiles_c, tc = blockIdx.x - tr * p.tiles_c;
  const int sub = threadIdx.x & 7, row = threadIdx.x >> 3;           // 8 lanes a row
  const int c = tc * QT + 16 * sub, r0 = tr * QT + row;
  uint32_t v[PASSES<T>][RW<T>];
#pragma unroll
  for (int i = 0; i < PASSES<T>; ++i) {
    const int r = r0 + ROW_STEP<T> * i;
    const T* src = (const T*)p.x + (size_t)r * p.ldx + c;
    if (VEC && r < p.rows && c <= p.cols - 16) {
#pragma unroll
      for (int j = 0; j < RW<T>; j += 4) {
        const uint4 u = __ldg(reinterpret_cast<const uint4*>(src) + j / 4);
        v[i][j] = u.x; v[i][j + 1] = u.y; v[i][j + 2] = u.z; v[i][j + 3] = u.w;
      }
    } else {
#pragma unroll
      for (int j = 0; j < RW<T>; ++j) {
        uint32_t w = 0u;
#pragma unroll
        for (int k = 0; k < W::N; ++k)
          if (r < p.rows && c + j * W::N + k < p.cols) {
            if (W::N == 2) w |= (uint32_t)reinterpret_cast<const uint16_t*>(src)[j * W::N + k] << (16 * k);
            else w = reinterpret_cast<const uint32_t*>(src)[j];
          }
        v[i][j] = w;
      }
    }
  }
  uint32_t am[PASSES<T>], most = 0u;
#pragma unroll
  for (int i = 0; i < PASSES<T>; ++i) {
    uint32_t m = 0u;
#pragma unroll
    for (int j = 0; j < RW<T>; ++j) m = W::template max_abs<false>(m, v[i][j]);
    am[i] = W::join(m);
    most = max(most, am[i]);
    if (TRANSPOSED) {
#pragma unroll
      for (int j = 0; j < RW<T>; j += 4)
        tile_raw[(row + ROW_STEP<T> * i) * (WPR<T> / 4) + unit_at((sub * RW<T> + j) / 4)] = make_uint4(v[i][j], v[i][j + 1], v[i][j + 2], v[i][j + 3]);
    }
  }
  // with a transposed output also the barrier between writing the tile and reading it
  const bool bad = (TRANSPOSED || p.square ? __syncthreads_or(most >= W::INF_BITS) : __any_sync(0xffffffffu, most >= W::INF_BITS)) != 0;
  uint32_t all = 0u;
  if (STRAIGHT || p.square)
    all = bad ? quantize_rows<T, FMT, STRAIGHT, true>(p, v, am, red, tr, tc) : quantize_rows<T, FMT, STRAIGHT, false>(p, v, am, red, tr, tc);
  if (TRANSPOSED) {
    if (bad) quantize_columns<T, FMT, true>(p, tile_raw, col_max, all, tr, tc);
    else quantize_columns<T, FMT, false>(p, tile_raw, col_max, all, tr, tc);
  }
}

template <typename T, int FMT, bool VEC>
fax_status launch(fax_ctx* ctx, const QuantParams& p, unsigned int blocks) {
  constexpr int tile_bytes = QT * QT * (int)sizeof(T);
  if (p.q && p.qt) {
    static bool done[FAX_MAX_DEVICES] = {};
    FAX_TRY(fax_opt_in_shared_memory(ctx, fp8_quantize_kernel<T, FMT, VEC, true, true>, tile_bytes, done));
    fax_launch(ctx, fp8_quantize_kernel<T, FMT, VEC, true, true>, dim3(blocks), dim3(THREADS<T>), tile_bytes, p);
  } else if (p.q) {
    fax_launch(ctx, fp8_quantize_kernel<T, FMT, VEC, true, false>, dim3(blocks), dim3(THREADS<T>), 0, p);
  } else {
    static bool done[FAX_MAX_DEVICES] = {};
    FAX_TRY(fax_opt_in_shared_memory(ctx, fp8_quantize_kernel<T, FMT, VEC, false, true>, tile_bytes, done));
    fax_launch(ctx, fp8_quantize_kernel<T, FMT, VEC, false, true>, dim3(blocks), dim3(THREADS<T>), tile_bytes, p);
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
  if (rb * cb > 0x40000000LL) return FAX_ERR_UNSUPPORTED_SHAPE;
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
