// Positions by rotation: pairs of a head's elements turned by position * frequency (see fax_ops.h).
//
// The angle.  A frequency is held as turns in units of 2^-64, so that position * frequency modulo 2^64 is the angle modulo a
// turn with no rounding at all: one 64-bit integer product, right at any position (a float32 angle is off by 0.06 rad at
// position 10^6).  The nearest quarter turn is split off exactly; sine and cosine of what is left (within an eighth of a turn, 34
// bits behind the point of the turn) are the first five terms of their series each, whose remainder is below 2^-24; with the roundings of
// the angle and of the terms they are within 2^-22 of their values (3.2 and 2.2 times 2^-24 over millions of angles).
//
// The work.  Each element is read and written once; memory bounds it, the instructions come next (two pairs share one where the hardware has
// it).  The factors are the same for every head of a token, so a thread works out those of one 16-byte vector of one token,
// keeps them in registers and goes over the heads (or a part of them where tokens are few), several heads' loads on their way
// together.  With HALVES the vector's partner lies half of rot_dim further: the lanes of a token cover whole lines of a head with both.
#include <cmath>

#include "stream_common.cuh"
#include "../../include/fax_ops.h"

namespace {

constexpr int THREADS = 256;

struct RotaryParams {
  const void* x; void* y; int64_t ldx, ldy;
  const int32_t* positions;
  const uint64_t* freq;
  int32_t heads, head_dim, half, first, seq;
  int64_t row0;                                   // of the launch's first row
  int32_t turned;                                 // units of a head that turn; those behind are copied
  int32_t per;                                    // heads of a thread
  FastDiv units, tokens;                          // units of a head; rows
  int64_t threads;
  float amplitude; int32_t backward;
};

// Cosine and sine of a turn's fraction held in units of 2^-64.
__device__ __forceinline__ void turn(uint64_t angle, float* c, float* s) {
  const uint64_t quarter = (angle + (1ull << 61)) >> 62;
  const int32_t rest = (int32_t)((int64_t)(angle - (quarter << 62)) >> 30);    // [-2^31, 2^31): units of 2^-34 turns
  const float t = (float)rest * (6.28318531f * 0x1p-34f);                      // within pi / 4
  const float q = t * t;
  const float sn = fmaf(t * q, fmaf(q, fmaf(q, fmaf(q, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), t);
  const float cs = fmaf(q, fmaf(q, fmaf(q, fmaf(q, 1.f / 40320, -1.f / 720), 1.f / 24), -0.5f), 1.f);
  const bool odd = quarter & 1;
  const float a = odd ? sn : cs, b = odd ? cs : sn;
  *c = (quarter == 1 || quarter == 2) ? -a : a;
  *s = (quarter >= 2) ? -b : b;
}

// N elements as floats.
template <typename T, int N>
__device__ __forceinline__ void widen(const Pack<T, N>& p, float* f) {
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = to_f32(p.e[i]);
}
template <typename T, int N>
__device__ __forceinline__ Pack<T, N> narrow(const float* f) {
  Pack<T, N> p;
  if constexpr (sizeof(T) == 2 && N % 2 == 0) {
#pragma unroll
    for (int i = 0; i + 1 < N; i += 2) reinterpret_cast<__nv_bfloat162*>(p.e)[i / 2] = __floats2bfloat162_rn(f[i], f[i + 1]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) p.e[i] = from_f32<T>(f[i]);
  }
  return p;
}
// VEC: one access; else element by element.
template <typename T, int N, bool VEC>
__device__ __forceinline__ Pack<T, N> load(const T* p) {
  Pack<T, N> v;
  if constexpr (VEC) {
    v = load_pack<T, N>(p);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v.e[i] = p[i];
  }
  return v;
}
template <typename T, int N, bool VEC>
__device__ __forceinline__ void store(T* p, const Pack<T, N>& v) {
  if constexpr (VEC) {
    store_pack<T, N>(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = v.e[i];
  }
}

// Two floats an instruction.
typedef unsigned long long two;
__device__ __forceinline__ two pack2(float a, float b) { two r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void unpack2(two v, float* f) { asm("mov.b64 {%0, %1}, %2;" : "=f"(f[0]), "=f"(f[1]) : "l"(v)); }
__device__ __forceinline__ two mul2(two a, two b) { two r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ two fma2(two a, two b, two c) { two r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }

// A unit is N elements and, with HALVES, the N that turn with them; with PAIRS the N elements are N / 2 pairs.
template <typename T, int LAYOUT, int N, bool VEC>
__global__ void __launch_bounds__(THREADS, 3) rotary_kernel(const RotaryParams p) {
  constexpr bool HALVES = LAYOUT == FAX_ROTARY_HALVES;
  constexpr int PAIRS_ = HALVES ? N : N / 2;                                     // pairs of a unit
  constexpr int HEADS = HALVES ? 2 : 4;                                          // on their way together: 80 registers, three blocks an SM
  fax_grid_dependency_wait();
  const int64_t id = (int64_t)blockIdx.x * THREADS + threadIdx.x;
  if (id >= p.threads) return;
  const uint32_t rest = p.units.div((uint32_t)id), j = p.units.mod((uint32_t)id, rest);
  const uint32_t part = p.tokens.div(rest), row = p.tokens.mod(rest, part);
  const int head0 = (int)part * p.per, heads = min(p.per, p.heads - head0);
  const bool turns = (int)j < p.turned;
  // (behind the turning elements a unit is 2 N elements with HALVES)
  const int col = (int)j * (HALVES && !turns ? 2 * N : N), partner = turns ? p.half : N;
  const T* x = (const T*)p.x + row * p.ldx + (int64_t)head0 * p.head_dim + col;
  T* y = (T*)p.y + row * p.ldy + (int64_t)head0 * p.head_dim + col;

  Pack<T, N> a[HEADS], b[HALVES ? HEADS : 1];
  auto fetch = [&](int h0) {
#pragma unroll
    for (int h = 0; h < HEADS; ++h)
      if (h0 + h < heads) {
        a[h] = load<T, N, VEC>(x + h * p.head_dim);
        if constexpr (HALVES) b[h] = load<T, N, VEC>(x + h * p.head_dim + partner);
      }
    x += HEADS * p.head_dim;
  };
  fetch(0);                                       // on its way while the factors are made
  float c[PAIRS_], s[PAIRS_];
  if (turns) {
    const uint64_t pos = (uint64_t)(p.positions ? (int64_t)p.positions[row] : (int64_t)p.first + (p.seq ? (p.row0 + row) % p.seq : p.row0 + row));
    const float amplitude = p.amplitude, signed_amplitude = p.backward ? -p.amplitude : p.amplitude;
#pragma unroll
    for (int i = 0; i < PAIRS_; ++i) {
      turn(pos * p.freq[j * PAIRS_ + i], &c[i], &s[i]);
      c[i] *= amplitude;
      s[i] *= signed_amplitude;
    }
  }
  for (int h0 = 0; h0 < heads; h0 += HEADS) {
    if (h0) fetch(h0);
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      if (h0 + h >= heads) break;
      if (turns) {
        float v[HALVES ? 2 * N : N];
        widen<T, N>(a[h], v);
        if constexpr (HALVES) widen<T, N>(b[h], v + N);
        if constexpr (HALVES && N % 2 == 0) {
#pragma unroll
          for (int i = 0; i < N; i += 2) {
            const two va = pack2(v[i], v[i + 1]), vb = pack2(v[N + i], v[N + i + 1]), cc = pack2(c[i], c[i + 1]), ss = pack2(s[i], s[i + 1]);
            unpack2(fma2(vb, pack2(-s[i], -s[i + 1]), mul2(va, cc)), v + i);
            unpack2(fma2(va, ss, mul2(vb, cc)), v + N + i);
          }
        } else {
#pragma unroll
          for (int i = 0; i < PAIRS_; ++i) {
            const int ia = HALVES ? i : 2 * i, ib = HALVES ? N + i : 2 * i + 1;
            const float va = v[ia], vb = v[ib];
            v[ia] = fmaf(-vb, s[i], va * c[i]);
            v[ib] = fmaf(va, s[i], vb * c[i]);
          }
        }
        a[h] = narrow<T, N>(v);
        if constexpr (HALVES) b[h] = narrow<T, N>(v + N);
      }
      store<T, N, VEC>(y + h * p.head_dim, a[h]);
      if constexpr (HALVES) store<T, N, VEC>(y + h * p.head_dim + partner, b[h]);
    }
    y += HEADS * p.head_dim;
  }
}

template <typename T, int N>
void launch(fax_ctx* ctx, int layout, bool vec, int grid, const RotaryParams& p) {
  void (*kernel)(RotaryParams);
  if (layout == FAX_ROTARY_HALVES) kernel = rotary_kernel<T, FAX_ROTARY_HALVES, N, true>;
  else if (vec) kernel = rotary_kernel<T, FAX_ROTARY_PAIRS, (N > 1 ? N : 2), true>;
  else kernel = rotary_kernel<T, FAX_ROTARY_PAIRS, 2, false>;
  fax_launch(ctx, kernel, dim3(grid), dim3(THREADS), 0, p);
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

  if (!in_place && d->head_dim % 2) return FAX_ERR_UNSUPPORTED_SHAPE;         // the copied rest has a last element without a partner

  // Elements of a vector: as many as fill 16 bytes, or 8, where heads, pairs and rows divide into such vectors; else single
  // elements (HALVES) or pairs (PAIRS).
  const int half = d->rot_dim / 2, moved = in_place ? d->rot_dim : d->head_dim;
  const bool halves = d->layout == FAX_ROTARY_HALVES;
  auto fits = [&](int n) {
    return (halves ? half % n == 0 && moved % (2 * n) == 0 : d->rot_dim % n == 0 && moved % n == 0) && d->head_dim % n == 0 && fax_rows_aligned(d->x, d->ldx, es, n * es) &&
           fax_rows_aligned(d->y, d->ldy, es, n * es);
  };
  const int full = (int)(16 / es), n = fits(full) ? full : fits(full / 2) ? full / 2 : halves ? 1 : 2;
  const bool vec = n > 2 || halves || fits(n);

  RotaryParams p;
  p.ldx = d->ldx; p.ldy = d->ldy; p.freq = d->frequencies;
  p.heads = d->heads; p.half = half; p.head_dim = d->head_dim; p.first = d->first; p.seq = d->seq;
  p.turned = halves ? half / n : d->rot_dim / n;
  p.amplitude = d->amplitude; p.backward = d->backward != 0;
  const int64_t units = halves ? moved / (2 * n) : moved / n;
  // Heads of a thread: all of them, or so few that there are 32 warps an SM (16384 x 24 x 64 in place: 25 us with 16, 22 us with 32, 23 us
  // with 48 of them; a thread's factors cost as much as a few heads).
  const int64_t want = 32 * 32 * (int64_t)ctx->sm_count;
  int64_t parts = (want + units * d->rows - 1) / (units * d->rows);
  if (parts > d->heads) parts = d->heads;
  p.per = (int32_t)((d->heads + parts - 1) / parts);
  const int64_t row_threads = units * ((d->heads + p.per - 1) / p.per);
  p.units = FastDiv((uint32_t)units);
  FaxProfScope prof(ctx, KC_ROTARY, 3.0 * d->rows * d->heads * d->rot_dim, 2.0 * d->rows * d->heads * moved * es + (d->positions ? 4.0 * d->rows : 0.0));
  // threads are counted in 31 bits
  const int64_t most = 0x7fffff00 / row_threads;
  for (int64_t r0 = 0; r0 < d->rows; r0 += most) {
    const int64_t rows = d->rows - r0 < most ? d->rows - r0 : most;
    p.x = (const char*)d->x + r0 * d->ldx * es; p.y = (char*)d->y + r0 * d->ldy * es;
    p.positions = d->positions ? d->positions + r0 : nullptr;
    p.row0 = r0;
    p.threads = row_threads * rows;
    p.tokens = FastDiv((uint32_t)rows);
    const int grid = (int)((p.threads + THREADS - 1) / THREADS);
    if (prec == FAX_PREC_BF16) {
      if (n == 8) launch<bf16, 8>(ctx, d->layout, vec, grid, p);
      else if (n == 4) launch<bf16, 4>(ctx, d->layout, vec, grid, p);
      else launch<bf16, 1>(ctx, d->layout, vec, grid, p);
    } else {
      if (n == 4) launch<float, 4>(ctx, d->layout, vec, grid, p);
      else if (n == 2 && vec) launch<float, 2>(ctx, d->layout, vec, grid, p);
      else launch<float, 1>(ctx, d->layout, vec, grid, p);
    }
    FAX_TRY(fax_after_launch(ctx));
  }
  return FAX_OK;
}
