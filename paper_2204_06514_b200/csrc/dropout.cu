// Dropout whose mask is never stored: y = resid + (kept ? x / (1 - p) : 0) (see fax_ops.h for the bits).
//
// Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): ten rounds of two
// 32 x 32 -> 64 bit products over a counter of four words; the rounds' keys are the same for all and come with the launch.
// One counter gives the 16 bits of eight elements, which are one 16-byte vector of bf16, so that a thread draws once for what
// it loads.  Memory bounds it, the instructions come next: some 15 an element beside 4 to 6 bytes of traffic.
#include <cmath>

#include "stream_common.cuh"
#include "../../include/fax_ops.h"

namespace {

constexpr int THREADS = 256;
constexpr int ROUNDS = 10;

struct DropoutParams {
  const void* x; const void* resid; void* y;
  int64_t ldx, ldr, ldy;
  int64_t units;                   // rows * groups
  FastDiv groups;                  // of eight columns in a row
  uint32_t step_rows, step_groups; // THREADS groups further
  int32_t cols;
  uint32_t limit;                  // dropped below it
  uint32_t above;                  // 2^16 limit - 1
  float scale;
  uint32_t k0[ROUNDS], k1[ROUNDS];
  uint64_t offset;
  const uint64_t* offset_device;
};

// N counters at once, so that a round's keys are fetched once for all.
template <int N>
__device__ __forceinline__ void philox(const DropoutParams& p, const uint32_t (&c0)[N], const uint32_t (&c1)[N], uint64_t offset, uint32_t (&w)[N][4]) {
#pragma unroll
  for (int n = 0; n < N; ++n) { w[n][0] = c0[n]; w[n][1] = c1[n]; w[n][2] = (uint32_t)offset; w[n][3] = (uint32_t)(offset >> 32); }
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const uint32_t k0 = p.k0[r], k1 = p.k1[r];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const uint64_t p0 = (uint64_t)w[n][0] * 0xD2511F53u, p1 = (uint64_t)w[n][2] * 0xCD9E8D57u;
      w[n][0] = (uint32_t)(p1 >> 32) ^ w[n][1] ^ k0;
      w[n][1] = (uint32_t)p1;
      w[n][2] = (uint32_t)(p0 >> 32) ^ w[n][3] ^ k1;
      w[n][3] = (uint32_t)p0;
    }
  }
}

// How the rows lie.  FLAT: one after the other without gaps, in whole vectors; PITCHED: whole vectors a pitch apart; SHORT: the same with a last
// group that is short of columns; LOOSE: anything, element by element.
enum Rows { FLAT, PITCHED, SHORT, LOOSE };

// Groups of eight columns of a thread: several of bf16 in whole vectors share the fetching of keys (8192 x 4096: 28.6 us with one, 24.3 with two, 23.1
// with four; with residual 16384 x 768: 14.0, 13.4, 13.4 us; a pitch of 4104: 25.1 us with four, 33.6 with one and branches between its loads); else
// one, with more warps to hide the loads (float 22.1 against 22.7 us).
template <typename T> constexpr int units_of(bool resid, int rows) { return (rows == FLAT || rows == PITCHED) && sizeof(T) == 2 ? (resid ? 2 : 4) : 1; }
template <typename T, bool RESID, int ROWS>
__global__ void __launch_bounds__(THREADS, units_of<T>(RESID, ROWS) > 1 ? 4 : 1) dropout_kernel(const __grid_constant__ DropoutParams p) {
  constexpr int UNITS = units_of<T>(RESID, ROWS);
  fax_grid_dependency_wait();
  const uint64_t offset = p.offset + (p.offset_device ? *p.offset_device : 0);
  const int64_t first = (int64_t)blockIdx.x * (THREADS * UNITS);
  uint32_t row[UNITS], group[UNITS];
  {
    const uint32_t row0 = (uint32_t)(first / p.groups.d), at = (uint32_t)(first - (int64_t)row0 * p.groups.d) + threadIdx.x, down = p.groups.div(at);
    row[0] = row0 + down;
    group[0] = p.groups.mod(at, down);
#pragma unroll
    for (int k = 1; k < UNITS; ++k) {
      row[k] = row[k - 1] + p.step_rows;
      group[k] = group[k - 1] + p.step_groups;
      if (group[k] >= p.groups.d) { group[k] -= p.groups.d; ++row[k]; }
    }
  }
  auto place = [&](int k, int64_t ld) { return ROWS == FLAT ? (first + threadIdx.x + k * THREADS) * 8 : (int64_t)row[k] * ld + group[k] * 8; };
  Pack<T, 8> x[UNITS], r[RESID ? UNITS : 1];
  bool live[UNITS], whole[UNITS];
#pragma unroll
  for (int k = 0; k < UNITS; ++k) {
    live[k] = first + threadIdx.x + k * THREADS < p.units;
    whole[k] = ROWS == FLAT || ROWS == PITCHED || (ROWS == SHORT && (int)group[k] * 8 + 8 <= p.cols);
    if (!live[k]) continue;
    const T* px = (const T*)p.x + place(k, p.ldx);
    const T* pr = RESID ? (const T*)p.resid + place(k, p.ldr) : nullptr;
    if (whole[k]) {
      x[k] = load_pack<T, 8>(px);
      if constexpr (RESID) r[k] = load_pack<T, 8>(pr);
    } else if (ROWS == LOOSE && (int)group[k] * 8 + 8 <= p.cols) {               // no branches between the loads
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[k].e[i] = px[i];
        if constexpr (RESID) r[k].e[i] = pr[i];
      }
    } else if (ROWS == SHORT || ROWS == LOOSE) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if ((int)group[k] * 8 + i < p.cols) {
          x[k].e[i] = px[i];
          if constexpr (RESID) r[k].e[i] = pr[i];
        }
    }
  }
  uint32_t bits[UNITS][4];
  if (p.limit) {
    philox<UNITS>(p, group, row, offset, bits);
  } else {                                         // keeps everything: whatever is above 0
#pragma unroll
    for (int k = 0; k < UNITS; ++k) bits[k][0] = bits[k][1] = bits[k][2] = bits[k][3] = ~0u;
  }
#pragma unroll
  for (int k = 0; k < UNITS; ++k) {
    if (!live[k]) continue;
    const uint32_t (&w)[4] = bits[k];
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool keep = (i % 2 ? w[i / 2] : w[i / 2] << 16) > p.above;       // the 16 bits against the limit, in the upper half of a word
      const float kept = keep ? to_f32(x[k].e[i]) : 0.f;      // whatever x is
      if constexpr (RESID) y[i] = fmaf(kept, p.scale, to_f32(r[k].e[i]));
      else y[i] = kept * p.scale;
    }
    Pack<T, 8> out;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 8; i += 2) reinterpret_cast<__nv_bfloat162*>(out.e)[i / 2] = __floats2bfloat162_rn(y[i], y[i + 1]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) out.e[i] = from_f32<T>(y[i]);
    }
    T* py = (T*)p.y + place(k, p.ldy);
    if (whole[k]) {
      store_pack<T, 8>(py, out);
    } else if (ROWS == LOOSE && (int)group[k] * 8 + 8 <= p.cols) {
#pragma unroll
      for (int i = 0; i < 8; ++i) py[i] = out.e[i];
    } else if (ROWS == SHORT || ROWS == LOOSE) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if ((int)group[k] * 8 + i < p.cols) py[i] = out.e[i];
    }
  }
}

template <typename T, int ROWS>
void launch(fax_ctx* ctx, bool resid, const DropoutParams& p) {
  const int64_t per_block = THREADS * units_of<T>(resid, ROWS);
  fax_launch(ctx, resid ? dropout_kernel<T, true, ROWS> : dropout_kernel<T, false, ROWS>, dim3((unsigned)((p.units + per_block - 1) / per_block)), dim3(THREADS), 0, p);
}
template <typename T>
void launch(fax_ctx* ctx, bool resid, Rows rows, const DropoutParams& p) {
  if (rows == FLAT) launch<T, FLAT>(ctx, resid, p);
  else if (rows == PITCHED) launch<T, PITCHED>(ctx, resid, p);
  else if (rows == SHORT) launch<T, SHORT>(ctx, resid, p);
  else launch<T, LOOSE>(ctx, resid, p);
}

}  // namespace

extern "C" fax_status fax_op_dropout(fax_ctx* ctx, int32_t prec, const fax_dropout_desc* d) {
  if (!ctx || !d || (prec != FAX_PREC_BF16 && prec != FAX_PREC_FP32_VALIDATE)) return FAX_ERR_INVALID_ARG;
  if (d->rows < 0 || d->cols < 1 || !(d->p >= 0.f && d->p <= 1.f)) return FAX_ERR_INVALID_ARG;
  if (d->ldx < d->cols || d->ldy < d->cols || (d->resid && d->ldr < d->cols)) return FAX_ERR_INVALID_ARG;
  if (d->cols > (1 << 30)) return FAX_ERR_UNSUPPORTED_SHAPE;
  if (d->rows == 0) return FAX_OK;
  if (!d->x || !d->y) return FAX_ERR_INVALID_ARG;
  const size_t es = fax_elem_size(prec);
  if (!fax_aligned(d->x, es) || !fax_aligned(d->y, es) || !fax_aligned(d->resid, es) || !fax_aligned(d->offset_device, 8)) return FAX_ERR_INVALID_ARG;
  if ((d->x == d->y && d->ldx != d->ldy) || (d->resid == d->y && d->ldr != d->ldy)) return FAX_ERR_INVALID_ARG;
  const uint32_t groups = ((uint32_t)d->cols + 7) / 8;
  const int64_t units = (int64_t)d->rows * groups;
  if (units / THREADS >= 0x7fffffff) return FAX_ERR_UNSUPPORTED_SHAPE;

  DropoutParams p;
  p.x = d->x; p.resid = d->resid; p.y = d->y; p.ldx = d->ldx; p.ldr = d->ldr; p.ldy = d->ldy;
  p.units = units; p.groups = FastDiv(groups); p.cols = d->cols;
  p.limit = (uint32_t)std::rint((double)d->p * 65536.0);
  p.above = p.limit ? (p.limit << 16) - 1u : 0u;            // (all ones for 65536: nothing is above)
  p.scale = p.limit < 65536 ? (float)(65536.0 / (65536.0 - p.limit)) : 0.f;
  for (int r = 0; r < ROUNDS; ++r) {
    p.k0[r] = (uint32_t)d->seed + (uint32_t)r * 0x9E3779B9u;
    p.k1[r] = (uint32_t)(d->seed >> 32) + (uint32_t)r * 0xBB67AE85u;
  }
  p.offset = d->offset; p.offset_device = d->offset_device;
  p.step_rows = THREADS / groups; p.step_groups = THREADS % groups;
  const bool vec = fax_rows_aligned(d->x, d->ldx, es, 16) && fax_rows_aligned(d->y, d->ldy, es, 16) && (!d->resid || fax_rows_aligned(d->resid, d->ldr, es, 16));
  const bool flat = d->cols % 8 == 0 && d->ldx == d->cols && d->ldy == d->cols && (!d->resid || d->ldr == d->cols);
  const Rows rows = !vec ? LOOSE : flat ? FLAT : d->cols % 8 == 0 ? PITCHED : SHORT;
  const double n = (double)d->rows * d->cols;
  FaxProfScope prof(ctx, KC_DROPOUT, 2.0 * n, (d->resid ? 3.0 : 2.0) * n * es);
  if (prec == FAX_PREC_BF16) launch<bf16>(ctx, d->resid != nullptr, rows, p);
  else launch<float>(ctx, d->resid != nullptr, rows, p);
  return fax_after_launch(ctx);
}
