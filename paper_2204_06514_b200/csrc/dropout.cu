// Dropout whose mask is never stored: y = resid + (kept ? x / (1 - p) : 0) (see fax_ops.h for the bits).
//
// Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): ten rounds of two
// 32 x 32 -> 64 bit products over a counter of four words.  One counter gives the 16 bits of eight elements, which are one
// 16-byte vector of bf16, so that a thread draws once for what it loads: about 6 integer instructions an element beside 4
// to 6 bytes of traffic, which bound the kernel.
#include <cmath>

#include "stream_common.cuh"
#include "../../include/fax_ops.h"

namespace {

constexpr int THREADS = 256;
constexpr int UNITS = 2;           // groups of eight columns a thread has in flight

struct DropoutParams {
  const void* x; const void* resid; void* y;
  int64_t ldx, ldr, ldy;
  int64_t units;                   // rows * groups
  FastDiv groups;                  // of eight columns in a row
  int32_t cols;
  uint32_t limit;                  // dropped below it
  float scale;
  uint64_t seed, offset;
  const uint64_t* offset_device;
};

__device__ __forceinline__ uint4 philox(uint32_t c0, uint32_t c1, uint64_t offset, uint64_t key) {
  uint32_t x0 = c0, x1 = c1, x2 = (uint32_t)offset, x3 = (uint32_t)(offset >> 32);
  uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p0 = (uint64_t)x0 * 0xD2511F53u, p1 = (uint64_t)x2 * 0xCD9E8D57u;
    x0 = (uint32_t)(p1 >> 32) ^ x1 ^ k0;
    x1 = (uint32_t)p1;
    x2 = (uint32_t)(p0 >> 32) ^ x3 ^ k1;
    x3 = (uint32_t)p0;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(x0, x1, x2, x3);
}

// VEC: rows and pitches are whole vectors; otherwise a group is handled element by element.
template <typename T, bool RESID, bool VEC>
__global__ void __launch_bounds__(THREADS) dropout_kernel(const DropoutParams p) {
  fax_grid_dependency_wait();
  const uint64_t offset = p.offset + (p.offset_device ? *p.offset_device : 0);
  const int64_t first = (int64_t)blockIdx.x * (THREADS * UNITS);
  const uint32_t row0 = (uint32_t)(first / p.groups.d), group0 = (uint32_t)(first - (int64_t)row0 * p.groups.d);
  Pack<T, 8> x[UNITS], r[UNITS];
  uint32_t row[UNITS], group[UNITS];
#pragma unroll
  for (int k = 0; k < UNITS; ++k) {
    const uint32_t u = threadIdx.x + k * THREADS;
    const uint32_t at = group0 + u, down = p.groups.div(at);
    row[k] = row0 + down;
    group[k] = p.groups.mod(at, down);
    if (first + u < p.units) {
      const int64_t in = (int64_t)row[k] * p.ldx + group[k] * 8, rin = (int64_t)row[k] * p.ldr + group[k] * 8;
      if (VEC) {
        x[k] = load_pack<T, 8>((const T*)p.x + in);
        if (RESID) r[k] = load_pack<T, 8>((const T*)p.resid + rin);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if ((int)group[k] * 8 + i < p.cols) {
            x[k].e[i] = ((const T*)p.x)[in + i];
            if (RESID) r[k].e[i] = ((const T*)p.resid)[rin + i];
          }
      }
    }
  }
#pragma unroll
  for (int k = 0; k < UNITS; ++k) {
    const uint32_t u = threadIdx.x + k * THREADS;
    if (first + u >= p.units) break;
    const uint4 bits = philox(group[k], row[k], offset, p.seed);
    const uint32_t w[4] = {bits.x, bits.y, bits.z, bits.w};
    Pack<T, 8> y;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t draw = i % 2 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu;
      const float kept = draw >= p.limit ? to_f32(x[k].e[i]) : 0.f;      // whatever x is
      y.e[i] = from_f32<T>(RESID ? fmaf(kept, p.scale, to_f32(r[k].e[i])) : kept * p.scale);
    }
    T* out = (T*)p.y + (int64_t)row[k] * p.ldy + group[k] * 8;
    if (VEC) {
      store_pack<T, 8>(out, y);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if ((int)group[k] * 8 + i < p.cols) out[i] = y.e[i];
    }
  }
}

template <typename T>
void launch(fax_ctx* ctx, bool resid, bool vec, int grid, const DropoutParams& p) {
  auto kernel = resid ? (vec ? dropout_kernel<T, true, true> : dropout_kernel<T, true, false>) : (vec ? dropout_kernel<T, false, true> : dropout_kernel<T, false, false>);
  fax_launch(ctx, kernel, dim3(grid), dim3(THREADS), 0, p);
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
  const int64_t units = (int64_t)d->rows * groups, blocks = (units + THREADS * UNITS - 1) / (THREADS * UNITS);
  if (blocks > 0x7fffffff) return FAX_ERR_UNSUPPORTED_SHAPE;

  DropoutParams p;
  p.x = d->x; p.resid = d->resid; p.y = d->y; p.ldx = d->ldx; p.ldr = d->ldr; p.ldy = d->ldy;
  p.units = units; p.groups = FastDiv(groups); p.cols = d->cols;
  p.limit = (uint32_t)std::rint((double)d->p * 65536.0);
  p.scale = p.limit < 65536 ? (float)(65536.0 / (65536.0 - p.limit)) : 0.f;
  p.seed = d->seed; p.offset = d->offset; p.offset_device = d->offset_device;
  const bool vec = d->cols % 8 == 0 && fax_rows_aligned(d->x, d->ldx, es, 16) && fax_rows_aligned(d->y, d->ldy, es, 16) &&
                   (!d->resid || fax_rows_aligned(d->resid, d->ldr, es, 16));
  const double n = (double)d->rows * d->cols;
  FaxProfScope prof(ctx, KC_DROPOUT, 2.0 * n, (d->resid ? 3.0 : 2.0) * n * es);
  if (prec == FAX_PREC_BF16) launch<bf16>(ctx, d->resid != nullptr, vec, (int)blocks, p);
  else launch<float>(ctx, d->resid != nullptr, vec, (int)blocks, p);
  return fax_after_launch(ctx);
}
