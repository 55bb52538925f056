// Positions by rotation: pairs of a head's elements turned by position * frequency (see fax_ops.h).
//
// The angle.  A frequency is held as turns in units of 2^-64, so that position * frequency modulo 2^64 is the angle modulo a
// turn with no rounding at all: one 64-bit integer product, right at any position (a float32 angle is off by 0.06 rad at
// position 10^6).  The nearest quarter turn is split off exactly, what is left (within an eighth of a turn, 34 bits behind the
// point of the turn) goes through sincospif: the two factors are within 1e-7 of their values.
//
// The work.  Each element is read and written once; memory bounds it.  The factors are the same for every head of a token, so
// a block first works out those of its rows (rows * rot_dim / 2 of them) into shared memory and then goes over its rows' heads
// 16 bytes a side at a time; the first loads are on their way while the factors are made.
#include <cmath>

#include "stream_common.cuh"
#include "../../include/fax_ops.h"

namespace {

constexpr int THREADS = 256;
constexpr int UNITS = 4;                          // pairs of vectors that a thread holds at a time
constexpr int TABLE_BYTES = 32 * 1024;

struct RotaryParams {
  const void* x; void* y; int64_t ldx, ldy;
  const int32_t* positions;
  const uint64_t* freq;
  int32_t rows, block_rows, half, head_dim, first, seq;
  int32_t turned;                                 // units of a head that turn; those behind are copied
  FastDiv row_units, head_units;                  // units of a row and of a head
  float amplitude; int32_t backward;
};

// Cosine and sine of a turn's fraction held in units of 2^-64.
__device__ __forceinline__ void turn(uint64_t angle, float* c, float* s) {
  const uint64_t quarter = (angle + (1ull << 61)) >> 62;
  const int64_t rest = (int64_t)(angle - (quarter << 62));                     // [-2^61, 2^61)
  float sn, cs;
  sincospif((float)(int32_t)(rest >> 30) * 0x1p-33f, &sn, &cs);                // half turns
  const bool odd = quarter & 1;
  const float a = odd ? sn : cs, b = odd ? cs : sn;
  *c = (quarter == 1 || quarter == 2) ? -a : a;
  *s = (quarter >= 2) ? -b : b;
}

// NP: pairs of a unit.  A unit is two vectors of NP elements: HALVES: NP first and NP second elements; PAIRS: 2 NP elements in a row.
template <typename T, int LAYOUT, int NP>
__global__ void __launch_bounds__(THREADS) rotary_kernel(const RotaryParams p) {
  extern __shared__ float table[];
  float* const cosines = table;
  float* const sines = table + p.block_rows * p.half;
  fax_grid_dependency_wait();
  const int row0 = blockIdx.x * p.block_rows;
  const int rows = min(p.block_rows, p.rows - row0);
  const uint32_t units = (uint32_t)rows * p.row_units.d;
  const T* const x = (const T*)p.x;
  T* const y = (T*)p.y;
  for (uint32_t base = 0; base < units; base += THREADS * UNITS) {
    Pack<T, NP> a[UNITS], b[UNITS];
    int64_t at[UNITS]; int32_t entry[UNITS], second[UNITS];
#pragma unroll
    for (int k = 0; k < UNITS; ++k) {
      const uint32_t u = base + k * THREADS + threadIdx.x;
      at[k] = -1;
      if (u < units) {
        const uint32_t r = p.row_units.div(u), in_row = p.row_units.mod(u, r);
        const uint32_t head = p.head_units.div(in_row), j = p.head_units.mod(in_row, head);
        const bool turns = (int)j < p.turned;
        const int col = LAYOUT == FAX_ROTARY_HALVES && turns ? (int)j * NP : (int)j * 2 * NP;
        second[k] = LAYOUT == FAX_ROTARY_HALVES && turns ? p.half : NP;
        entry[k] = turns ? (int)(r * p.half + j * NP) : -1;
        const int64_t row = row0 + (int)r;
        const int64_t in = (int64_t)head * p.head_dim + col;
        const T* src = x + row * p.ldx + in;
        a[k] = load_pack<T, NP>(src);
        b[k] = load_pack<T, NP>(src + second[k]);
        at[k] = row * p.ldy + in;
      }
    }
    if (base == 0) {
      for (int i = threadIdx.x; i < rows * p.half; i += THREADS) {
        const int r = i / p.half, f = i - r * p.half;
        const int row = row0 + r;
        const int64_t pos = p.positions ? (int64_t)p.positions[row] : (int64_t)p.first + (p.seq ? row % p.seq : row);
        float c, s;
        turn((uint64_t)pos * p.freq[f], &c, &s);
        cosines[i] = p.amplitude * c;
        sines[i] = p.backward ? -(p.amplitude * s) : p.amplitude * s;
      }
      __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < UNITS; ++k) {
      if (at[k] < 0) continue;
      if (entry[k] >= 0) {
        const Pack<float, NP> c = load_pack<float, NP>(cosines + entry[k]), s = load_pack<float, NP>(sines + entry[k]);
        float v[2 * NP], w[2 * NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) { v[i] = to_f32(a[k].e[i]); v[NP + i] = to_f32(b[k].e[i]); }
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int ia = LAYOUT == FAX_ROTARY_HALVES ? i : 2 * i, ib = LAYOUT == FAX_ROTARY_HALVES ? NP + i : 2 * i + 1;
          w[ia] = v[ia] * c.e[i] - v[ib] * s.e[i];
          w[ib] = v[ib] * c.e[i] + v[ia] * s.e[i];
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) { a[k].e[i] = from_f32<T>(w[i]); b[k].e[i] = from_f32<T>(w[NP + i]); }
      }
      store_pack<T, NP>(y + at[k], a[k]);
      store_pack<T, NP>(y + at[k] + second[k], b[k]);
    }
  }
}

template <typename T, int NP>
void launch(fax_ctx* ctx, int layout, int grid, size_t smem, const RotaryParams& p) {
  if (layout == FAX_ROTARY_HALVES) fax_launch(ctx, rotary_kernel<T, FAX_ROTARY_HALVES, NP>, dim3(grid), dim3(THREADS), smem, p);
  else fax_launch(ctx, rotary_kernel<T, FAX_ROTARY_PAIRS, NP>, dim3(grid), dim3(THREADS), smem, p);
}

}  // namespace

extern "C" fax_status fax_rotary_frequencies(int32_t rot_dim, double base, double factor, int32_t original_seq, double low_turns,
                                             double high_turns, uint64_t* out) {
  if (!out || rot_dim < 2 || rot_dim % 2 || rot_dim > FAX_ROTARY_MAX_DIM) return FAX_ERR_INVALID_ARG;
  if (!(base >= 1.0) || !(factor >= 1.0) || std::isinf(base) || std::isinf(factor) || original_seq < 0) return FAX_ERR_INVALID_ARG;
  if (factor > 1.0 && original_seq > 0 && !(low_turns < high_turns && std::isfinite(low_turns) && std::isfinite(high_turns))) return FAX_ERR_INVALID_ARG;
  const double two_pi = 6.283185307179586476925286766559;
  for (int i = 0; i < rot_dim / 2; ++i) {
    double turns = std::pow(base, -2.0 * i / rot_dim) / two_pi;                 // a position
    if (factor > 1.0) {
      double keep = 0.0;
      if (original_seq > 0) keep = std::fmin(1.0, std::fmax(0.0, (original_seq * turns - low_turns) / (high_turns - low_turns)));
      turns *= keep + (1.0 - keep) / factor;
    }
    out[i] = (uint64_t)std::rint(std::ldexp(turns, 64));                        // turns <= 1 / (2 pi)
  }
  return FAX_OK;
}

extern "C" fax_status fax_op_rotary(fax_ctx* ctx, int32_t prec, const fax_rotary_desc* d) {
  if (!ctx || !d || (prec != FAX_PREC_BF16 && prec != FAX_PREC_FP32_VALIDATE)) return FAX_ERR_INVALID_ARG;
  if (d->rows < 0 || d->heads < 1 || d->head_dim < 2 || d->rot_dim < 2 || d->rot_dim % 2 || d->rot_dim > d->head_dim || d->seq < 0) return FAX_ERR_INVALID_ARG;
  if (d->layout != FAX_ROTARY_HALVES && d->layout != FAX_ROTARY_PAIRS) return FAX_ERR_INVALID_ARG;
  const int64_t width = (int64_t)d->heads * d->head_dim;
  if (d->ldx < width || d->ldy < width) return FAX_ERR_INVALID_ARG;
  if (d->head_dim > FAX_ROTARY_MAX_DIM || width > (1 << 24) || d->rows > (1 << 30)) return FAX_ERR_UNSUPPORTED_SHAPE;
  if (d->rows == 0) return FAX_OK;
  if (!d->x || !d->y || !d->frequencies) return FAX_ERR_INVALID_ARG;
  const size_t es = fax_elem_size(prec);
  if (!fax_aligned(d->x, es) || !fax_aligned(d->y, es) || !fax_aligned(d->positions, 4) || !fax_aligned(d->frequencies, 8)) return FAX_ERR_INVALID_ARG;
  const bool in_place = d->x == d->y;
  if (in_place && d->ldx != d->ldy) return FAX_ERR_INVALID_ARG;

  // Elements a side of a unit: as many as fill 16 bytes, or 8 of them, where heads, pairs and rows divide into such vectors.
  const int half = d->rot_dim / 2, moved = in_place ? d->rot_dim : d->head_dim;
  auto fits = [&](int np) {
    return half % np == 0 && moved % (2 * np) == 0 && d->head_dim % np == 0 && fax_rows_aligned(d->x, d->ldx, es, np * es) && fax_rows_aligned(d->y, d->ldy, es, np * es);
  };
  const int np = es == 2 && fits(8) ? 8 : fits(4) ? 4 : 1;
  // Odd head_dim: the copied rest has a last element without a partner.
  if (moved % 2) return FAX_ERR_UNSUPPORTED_SHAPE;

  RotaryParams p;
  p.x = d->x; p.y = d->y; p.ldx = d->ldx; p.ldy = d->ldy; p.positions = d->positions; p.freq = d->frequencies;
  p.rows = d->rows; p.half = half; p.head_dim = d->head_dim; p.first = d->first; p.seq = d->seq;
  p.turned = half / np;
  p.head_units = FastDiv((uint32_t)(moved / (2 * np)));
  p.row_units = FastDiv((uint32_t)d->heads * p.head_units.d);
  p.amplitude = d->amplitude; p.backward = d->backward != 0;
  // Rows of a block: about as many as its threads hold at a time, within the table, and no fewer blocks than SMs.
  int64_t rows = (THREADS * UNITS + p.row_units.d - 1) / p.row_units.d;
  rows = rows < 1 ? 1 : rows;
  const int64_t table_rows = TABLE_BYTES / ((int64_t)half * 8), even = (d->rows + ctx->sm_count - 1) / ctx->sm_count;
  if (rows > table_rows) rows = table_rows;
  if (rows > even) rows = even;
  p.block_rows = (int32_t)rows;
  const int grid = (int)((d->rows + rows - 1) / rows);
  const size_t smem = (size_t)rows * half * 8;
  FaxProfScope prof(ctx, KC_ROTARY, 3.0 * d->rows * d->heads * d->rot_dim, 2.0 * d->rows * d->heads * moved * es + (d->positions ? 4.0 * d->rows : 0.0));
  if (prec == FAX_PREC_BF16) {
    if (np == 8) launch<bf16, 8>(ctx, d->layout, grid, smem, p);
    else if (np == 4) launch<bf16, 4>(ctx, d->layout, grid, smem, p);
    else launch<bf16, 1>(ctx, d->layout, grid, smem, p);
  } else {
    if (np == 4) launch<float, 4>(ctx, d->layout, grid, smem, p);
    else launch<float, 1>(ctx, d->layout, grid, smem, p);
  }
  return fax_after_launch(ctx);
}
