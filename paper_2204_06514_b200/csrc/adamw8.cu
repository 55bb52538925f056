// Multi-tensor AdamW whose moments are held in 8 bits: m in e4m3, v in e5m2, each block of 128
// elements with a power-of-two scale of its own.
//
//   m = s_m q_m, v = s_v q_v                       (exact: a power of two times a value of the format)
//   m <- b1 m + (1 - b1) g;  v <- b2 v + (1 - b2) g^2
//   w <- w - lr wd w - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
//   s = min { 2^k >= 2^-126 : max |m| / s <= 448 } over the block, q_m = SR(m / s); v likewise with 57344
//
// Why the moments are rounded stochastically: one step moves v by a share (1 - b2) of itself, far less
// than half the distance between neighbouring 8-bit floats (12 % of the value), so the nearest value
// would never move again.  SR(y) is the neighbour above with probability (y - below) / (above -
// below): right on average.  A v above zero never becomes zero (its smallest value is kept instead):
// m / (sqrt(0) + eps) would be a step out of all proportion.  Why e5m2 for v: it is a square, so it
// needs twice the exponent range of m.  Why powers of two: m / s is then exact, the rounding is the
// only loss, and the moments after a step are one well-defined bit pattern (their float operations are each
// rounded on its own, in the order written; no contraction).  The update of w takes root and quotient from the
// hardware's approximations and one correction each by the exact remainder, which a fused multiply-add gives
// (Markstein, "Computation of elementary functions on the IBM RISC System/6000 processor", 1990): rounded right but
// for rare halfway cases, so that w's bf16 copy is the definition's too.  Two elements share an instruction (f32x2)
// where no product is added to: the assembler contracts packed products and sums, which the moments must not be.
//
// The rounding in integers: y 2^-120 (2^-112 for e5m2) puts the format's smallest normal value on
// float32's, so that the float's bits, cut off after the format's mantissa, are the format's code,
// subnormals included; adding 16 random bits below the cut carries into it with the right probability.
// The largest moment is at most the format's largest value times the scale, which is where the cut falls, so
// that the sum never carries past the last code.
//
// HBM-bound if the instructions are few: 18 bytes per element (w 8, g 4, m 2, v 2, bf16 copy 2) against 30 with
// float32 moments.  A warp takes one block of 128 elements at a time, four elements a lane, so that a block's
// maximum is one warp reduction (redux) and every access is a full 32-byte sector or more.  Moments that are
// not finite are looked for once a block (their bits are the largest), not element by element.  201M elements: 615 us,
// 5.9 TB/s (in a run of a second 670 us), some 80 instructions an element; 900 us with every check and IEEE operation an element of its own.
#include "common.cuh"

#include <cuda_fp8.h>

#include <algorithm>
#include <cstdlib>

namespace {

constexpr int QB = FAX_ADAMW8_BLOCK;   // elements per scale
constexpr int THREADS = 128;
constexpr int UNROLL = 2;              // blocks of 128 a warp has in flight
constexpr int CHUNK = THREADS / 32 * UNROLL * QB;
constexpr int MAX_T = 40;              // tensors per launch (kernel-parameter space)

struct Adam8Tensor {
  float* w; uint8_t* m; uint8_t* v; float* ms; float* vs; const void* g; bf16* wc;
  unsigned long long n;
  float wd;
  uint32_t key;                        // random key of this tensor at this step
  unsigned int first_chunk;            // prefix sum of chunk counts
};
struct Adam8Batch {
  Adam8Tensor t[MAX_T];
  int n_tensors;
  unsigned int total_chunks;
};
struct Adam8Scalars { float lr, b1, b2, eps, inv_bc1, inv_bc2; };

static inline uint32_t mix32(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x7feb352du;
  x = (x ^ (x >> 15)) * 0x846ca68bu;
  return x ^ (x >> 16);
}

// Exponent field of the scale: the smallest power of two that brings the maximum to (1.75 2^TOP_EXP).
template <int TOP_EXP>
__device__ __forceinline__ int scale_field(uint32_t amax_bits) {
  const int f = (int)((amax_bits + 0x1fffffu) >> 23) - TOP_EXP;
  return amax_bits == 0u ? 127 : (f < 1 ? 1 : f);
}
// Stochastic rounding: y is the moment times 2^(127 - field) 2^-120 (2^-112 for e5m2); the codes are the top bytes
// of the words returned.  e4m3: sign, then bits 26 .. 20 of the float's magnitude; e5m2 (never negative): bits 28 .. 21.
__device__ __forceinline__ uint32_t sr_e4m3(float y, uint32_t h) {
  const uint32_t t = __float_as_uint(y) + ((h >> 12) & 0xffff0u) + 8u;
  return (t & 0x80000000u) | ((t << 4) & 0x7f000000u);
}
__device__ __forceinline__ uint32_t sr_e5m2(float y, uint32_t h) {
  return (__float_as_uint(y) + ((h & 0xffffu) << 5) + 16u) << 3;
}
__device__ __forceinline__ uint32_t top_bytes(const uint32_t (&c)[4]) {
  return __byte_perm(__byte_perm(c[0], c[1], 0x0073), __byte_perm(c[2], c[3], 0x0073), 0x5410);
}
__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7fffffffu) < 0x7f800000u; }
__device__ __forceinline__ uint32_t max4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) { return max(__vimax3_u32(a, b, c), d); }
// Bits of the largest magnitude; a NaN stays.
__device__ __forceinline__ uint32_t max4_abs(float a, float b, float c, float d) {
  float m;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(m), "f"(d), "f"(d));
  return __float_as_uint(m) & 0x7fffffffu;
}

// Two float32 in one register pair; one instruction for both.
typedef unsigned long long f2;
__device__ __forceinline__ f2 pair(float a, float b) {
  f2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void split(f2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
  f2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
  f2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
  f2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
// What a root is taken of: at least 2^-126 (a NaN stays), because the approximation takes smaller numbers for zero.
__device__ __forceinline__ float root_arg(float x) {
  asm("max.NaN.f32 %0, %0, 0f00800000;" : "+f"(x));
  return x;
}
// sqrt(x) of the raised x: s = x y, y ~ 1 / sqrt(x);  s + (x - s s) y / 2.
__device__ __forceinline__ f2 sqrt2(f2 x) {
  float a, b, ya, yb;
  split(x, a, b);
  a = root_arg(a); b = root_arg(b);
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(ya) : "f"(a));
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(yb) : "f"(b));
  const f2 c = pair(a, b), y = pair(ya, yb), minus = pair(-1.f, -1.f), half = pair(0.5f, 0.5f);
  const f2 s = mul2(c, y);
  return fma2(fma2(mul2(s, minus), s, c), mul2(y, half), s);
}
// a / b: r = 1 / b with one Newton step, q = a r;  q + (a - b q) r.
__device__ __forceinline__ f2 div2(f2 a, f2 b) {
  float u, v, ru, rv;
  split(b, u, v);
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(ru) : "f"(u));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(rv) : "f"(v));
  const f2 r0 = pair(ru, rv), bn = mul2(b, pair(-1.f, -1.f));
  const f2 r = fma2(r0, fma2(bn, r0, pair(1.f, 1.f)), r0);
  const f2 q = mul2(a, r);
  return fma2(fma2(bn, q, a), r, q);
}
// Four moments: values of the format times their scale.
__device__ __forceinline__ void decode4(uint32_t q, __nv_fp8_interpretation_t fmt, float scale, float (&x)[4]) {
  const float2 a = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(q & 0xffffu), fmt)));
  const float2 b = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(q >> 16), fmt)));
  const f2 s = pair(scale, scale);
  split(mul2(pair(a.x, a.y), s), x[0], x[1]);
  split(mul2(pair(b.x, b.y), s), x[2], x[3]);
}

// One warp's UNROLL blocks of a chunk.  FULL: the chunk lies wholly inside its tensor.
template <bool G_BF16, bool FULL>
__device__ __forceinline__ void update_blocks(const Adam8Tensor& t, const Adam8Scalars& sc, unsigned long long blk0, int lane) {
  constexpr int WARPS = THREADS / 32, NEXT = WARPS * QB;           // blocks, elements from one of the warp's blocks to its next
  const float omb1 = __fsub_rn(1.f, sc.b1), omb2 = __fsub_rn(1.f, sc.b2);
  const float lrwd = __fmul_rn(sc.lr, t.wd);
  auto both = [](float x) { return pair(x, x); };
  const unsigned long long e0 = blk0 * QB + 4 * lane;
  float* const wp = t.w + e0;
  uint8_t* const mp = t.m + e0;
  uint8_t* const vp = t.v + e0;
  bf16* const cp = t.wc + e0;
  float* const msp = t.ms + blk0;
  float* const vsp = t.vs + blk0;
  const float* const gp = (const float*)t.g + e0;
  const bf16* const hp = (const bf16*)t.g + e0;
  // elements of this lane's group that are inside (only the last block's group can be cut)
  auto inside = [&](int u) { return FULL ? 4 : (e0 + u * NEXT >= t.n ? 0 : (t.n - (e0 + u * NEXT) < 4 ? (int)(t.n - (e0 + u * NEXT)) : 4)); };
  auto block_in = [&](int u) { return FULL || (blk0 + u * WARPS) * QB < t.n; };

  float w[UNROLL][4], g[UNROLL][4];
  uint32_t mq[UNROLL], vq[UNROLL];
  float sm[UNROLL], sv[UNROLL];
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    const int in = inside(u);
    if (in == 4) {
      const float4 f = *reinterpret_cast<const float4*>(wp + u * NEXT);
      w[u][0] = f.x; w[u][1] = f.y; w[u][2] = f.z; w[u][3] = f.w;
      if (G_BF16) {
        const uint2 raw = *reinterpret_cast<const uint2*>(hp + u * NEXT);
        g[u][0] = __uint_as_float(raw.x << 16); g[u][1] = __uint_as_float(raw.x & 0xffff0000u);
        g[u][2] = __uint_as_float(raw.y << 16); g[u][3] = __uint_as_float(raw.y & 0xffff0000u);
      } else {
        const float4 h = *reinterpret_cast<const float4*>(gp + u * NEXT);
        g[u][0] = h.x; g[u][1] = h.y; g[u][2] = h.z; g[u][3] = h.w;
      }
      mq[u] = *reinterpret_cast<const uint32_t*>(mp + u * NEXT);
      vq[u] = *reinterpret_cast<const uint32_t*>(vp + u * NEXT);
    } else {
      mq[u] = vq[u] = 0u;                            // past the end: zeros, which leave the block's maximum alone
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        w[u][j] = j < in ? wp[u * NEXT + j] : 0.f;
        g[u][j] = j < in ? (G_BF16 ? __bfloat162float(hp[u * NEXT + j]) : gp[u * NEXT + j]) : 0.f;
        if (j < in) { mq[u] |= (uint32_t)mp[u * NEXT + j] << (8 * j); vq[u] |= (uint32_t)vp[u * NEXT + j] << (8 * j); }
      }
    }
    sm[u] = block_in(u) ? msp[u * WARPS] : 0.f;
    sv[u] = block_in(u) ? vsp[u * WARPS] : 0.f;
  }
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    if (!block_in(u)) continue;                      // the whole warp at once
    float m[4], v[4];
    decode4(mq[u], __NV_E4M3, sm[u], m);
    decode4(vq[u], __NV_E5M2, sv[u], v);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m[j] = __fadd_rn(__fmul_rn(sc.b1, m[j]), __fmul_rn(omb1, g[u][j]));
      v[j] = __fadd_rn(__fmul_rn(sc.b2, v[j]), __fmul_rn(__fmul_rn(omb2, g[u][j]), g[u][j]));
    }
    f2 upd[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const f2 den = add2(sqrt2(mul2(pair(v[2 * k], v[2 * k + 1]), both(sc.inv_bc2))), both(sc.eps));
      upd[k] = div2(mul2(both(sc.lr), mul2(pair(m[2 * k], m[2 * k + 1]), both(sc.inv_bc1))), den);
    }
    uint32_t am = __reduce_max_sync(0xffffffffu, max4_abs(m[0], m[1], m[2], m[3]));
    uint32_t av = __reduce_max_sync(0xffffffffu, max4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])));
    uint32_t bad_m = 0u, bad_v = 0u;                 // bytes that become NaN
    if (max(am, av) >= 0x6f800000u) {                // from 2^96 on, the whole warp: the update by the functions that take any
      float d[4];                                    // number, and what is not finite left out of the maxima
      am = av = 0u;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float den = __fadd_rn(__fsqrt_rn(root_arg(__fmul_rn(v[j], sc.inv_bc2))), sc.eps);
        d[j] = __fdiv_rn(__fmul_rn(sc.lr, __fmul_rn(m[j], sc.inv_bc1)), den);
        if (finite(m[j])) am = max(am, __float_as_uint(m[j]) & 0x7fffffffu);
        else { bad_m |= (m[j] < 0.f ? 0xffu : 0x7fu) << (8 * j); m[j] = 0.f; }
        if (finite(v[j])) av = max(av, __float_as_uint(v[j]));
        else { bad_v |= 0x7fu << (8 * j); v[j] = 0.f; }
      }
      am = __reduce_max_sync(0xffffffffu, am);
      av = __reduce_max_sync(0xffffffffu, av);
      upd[0] = pair(d[0], d[1]); upd[1] = pair(d[2], d[3]);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float d0, d1;
      split(upd[k], d0, d1);
      w[u][2 * k] = __fsub_rn(__fsub_rn(w[u][2 * k], __fmul_rn(lrwd, w[u][2 * k])), d0);
      w[u][2 * k + 1] = __fsub_rn(__fsub_rn(w[u][2 * k + 1], __fmul_rn(lrwd, w[u][2 * k + 1])), d1);
    }
    const int fm = scale_field<8>(am), fv = scale_field<15>(av);
    // moment times 2^(127 - field), then 2^-120 or 2^-112: one factor unless it is below 2^-126 itself
    float ym[4], yv[4];
    if (fm <= 133 && fv <= 141) {
      const float km = __uint_as_float((uint32_t)(134 - fm) << 23), kv = __uint_as_float((uint32_t)(142 - fv) << 23);
#pragma unroll
      for (int j = 0; j < 4; ++j) { ym[j] = __fmul_rn(m[j], km); yv[j] = __fmul_rn(v[j], kv); }
    } else {
      const float im = __uint_as_float((uint32_t)(254 - fm) << 23), iv = __uint_as_float((uint32_t)(254 - fv) << 23);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        ym[j] = __fmul_rn(__fmul_rn(m[j], im), __uint_as_float(7u << 23));
        yv[j] = __fmul_rn(__fmul_rn(v[j], iv), __uint_as_float(15u << 23));
      }
    }
    // mix32 of (element index ^ key): the index ends in two bits j, which the first shift leaves alone
    const unsigned long long e = e0 + u * NEXT;
    uint32_t x0 = (uint32_t)e ^ (t.key + (uint32_t)(e >> 32) * 0x85ebca77u);
    x0 ^= x0 >> 16;
    uint32_t cm[4], cv[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t h = (x0 ^ (uint32_t)j) * 0x7feb352du;
      h = (h ^ (h >> 15)) * 0x846ca68bu;
      h ^= h >> 16;
      cm[j] = sr_e4m3(ym[j], h);
      cv[j] = sr_e5m2(yv[j], h);
    }
    // a v above zero keeps at least its format's smallest value; looked at only where some code came out as 0
    if (__any_sync(0xffffffffu, min(min(cv[0], cv[1]), min(cv[2], cv[3])) < (1u << 24))) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (v[j] > 0.f) cv[j] = max(cv[j], 1u << 24);
    }
    const uint32_t qm = top_bytes(cm) | bad_m, qv = top_bytes(cv) | bad_v;
    const int in = inside(u);
    if (in == 4) {
      *reinterpret_cast<float4*>(wp + u * NEXT) = make_float4(w[u][0], w[u][1], w[u][2], w[u][3]);
      *reinterpret_cast<uint32_t*>(mp + u * NEXT) = qm;
      *reinterpret_cast<uint32_t*>(vp + u * NEXT) = qv;
      if (t.wc) {
        uint2 o;
        *reinterpret_cast<__nv_bfloat162*>(&o.x) = __floats2bfloat162_rn(w[u][0], w[u][1]);
        *reinterpret_cast<__nv_bfloat162*>(&o.y) = __floats2bfloat162_rn(w[u][2], w[u][3]);
        *reinterpret_cast<uint2*>(cp + u * NEXT) = o;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < in) {
          wp[u * NEXT + j] = w[u][j];
          mp[u * NEXT + j] = (uint8_t)(qm >> (8 * j)); vp[u * NEXT + j] = (uint8_t)(qv >> (8 * j));
          if (t.wc) cp[u * NEXT + j] = __float2bfloat16_rn(w[u][j]);
        }
    }
    if (lane == 0) { msp[u * WARPS] = __uint_as_float((uint32_t)fm << 23); vsp[u * WARPS] = __uint_as_float((uint32_t)fv << 23); }
  }
}

template <bool G_BF16>
__global__ void __launch_bounds__(THREADS, 8)
adamw8_kernel(const __grid_constant__ Adam8Batch batch, Adam8Scalars sc) {
  fax_grid_dependency_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (unsigned int chunk = blockIdx.x; chunk < batch.total_chunks; chunk += gridDim.x) {
    int lo = 0, hi = batch.n_tensors - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (batch.t[mid].first_chunk <= chunk) lo = mid; else hi = mid - 1;
    }
    const Adam8Tensor& t = batch.t[lo];
    const unsigned long long c = chunk - t.first_chunk;
    if ((c + 1) * CHUNK <= t.n) update_blocks<G_BF16, true>(t, sc, c * (CHUNK / QB) + warp, lane);
    else update_blocks<G_BF16, false>(t, sc, c * (CHUNK / QB) + warp, lane);
  }
}

// Do two tensors update the same weights?  Their blocks would race.
fax_status check_distinct(const fax_adamw8_tensor* tensors, int n) {
  const float* few[MAX_T];
  const float** w = n <= MAX_T ? few : (const float**)malloc((size_t)n * sizeof(*w));
  if (!w) return FAX_ERR_WORKSPACE_TOO_SMALL;          // host memory
  int k = 0;
  for (int i = 0; i < n; ++i)
    if (tensors[i].n) w[k++] = tensors[i].w;
  std::sort(w, w + k);
  const bool twice = std::adjacent_find(w, w + k) != w + k;
  if (w != few) free(w);
  return twice ? FAX_ERR_INVALID_ARG : FAX_OK;
}

}  // namespace

extern "C" fax_status fax_adamw8_step(fax_ctx* ctx, const fax_adamw8_tensor* tensors, int32_t n, const fax_adamw_hparams* hp) {
  if (!ctx || !hp || n < 0 || (n > 0 && !tensors)) return FAX_ERR_INVALID_ARG;
  FAX_TRY(fax_adamw_check_hparams(hp));
  double total = 0;
  for (int i = 0; i < n; ++i) {
    const fax_adamw8_tensor& t = tensors[i];
    if (t.n == 0) continue;
    if (!t.w || !t.m || !t.v || !t.m_scale || !t.v_scale || !t.g) return FAX_ERR_INVALID_ARG;
    if (!fax_aligned(t.w, 16) || !fax_aligned(t.g, 16) || !fax_aligned(t.m, 4) || !fax_aligned(t.v, 4) ||
        !fax_aligned(t.m_scale, 4) || !fax_aligned(t.v_scale, 4) || (t.w_compute && !fax_aligned(t.w_compute, 8)))
      return FAX_ERR_INVALID_ARG;
    if ((t.n + CHUNK - 1) / CHUNK > 0xffffffffull) return FAX_ERR_UNSUPPORTED_SHAPE;
    total += (double)t.n;
  }
  FAX_TRY(check_distinct(tensors, n));
  Adam8Scalars sc;
  sc.lr = hp->lr; sc.b1 = hp->beta1; sc.b2 = hp->beta2; sc.eps = hp->eps;
  sc.inv_bc1 = (float)(1.0 / (1.0 - pow((double)hp->beta1, (double)hp->step)));
  sc.inv_bc2 = (float)(1.0 / (1.0 - pow((double)hp->beta2, (double)hp->step)));
  FaxProfScope prof(ctx, KC_ADAMW, 0.0, total * (hp->grad_is_bf16 ? 16.0 : 18.0));
  int i = 0;
  while (i < n) {
    Adam8Batch batch;
    int k = 0;
    unsigned long long chunks = 0;
    while (i < n && k < MAX_T) {
      const fax_adamw8_tensor& t = tensors[i];
      const unsigned long long c = (t.n + CHUNK - 1) / CHUNK;
      if (chunks + c > 0xffffffffull) break;                 // the next launch takes it
      ++i;
      if (t.n == 0) continue;
      Adam8Tensor& b = batch.t[k];
      b.w = t.w; b.m = (uint8_t*)t.m; b.v = (uint8_t*)t.v; b.ms = t.m_scale; b.vs = t.v_scale; b.g = t.g; b.wc = (bf16*)t.w_compute;
      b.n = t.n; b.wd = t.weight_decay;
      b.key = mix32(t.seed + (uint32_t)hp->step * 0x9e3779b9u);
      b.first_chunk = (unsigned int)chunks;
      chunks += c;
      ++k;
    }
    if (k == 0) continue;                                    // only empty tensors were left
    batch.n_tensors = k;
    batch.total_chunks = (unsigned int)chunks;
    // a dozen and more rounds of blocks even the SMs out (201M elements: 642 us with two rounds, 615 us with 16, 640 us a chunk a block)
    const unsigned long long cap = (unsigned long long)ctx->sm_count * 128;
    const unsigned int grid = (unsigned int)(chunks < cap ? chunks : cap);
    if (hp->grad_is_bf16) fax_launch(ctx, adamw8_kernel<true>, dim3(grid), dim3(THREADS), 0, batch, sc);
    else fax_launch(ctx, adamw8_kernel<false>, dim3(grid), dim3(THREADS), 0, batch, sc);
    FAX_TRY(fax_after_launch(ctx));
  }
  return FAX_OK;
}
