// Gated linear recurrence over sequences, forward and backward (see fax_ops.h): h_t = a_t h_{t-1} + b_t for each channel.
//
// A stretch of tokens maps the state before it to the state behind it as h -> A h + B, and two stretches join as
// (A2 A1, A2 B1 + B2), so that time can be split: a thread folds 16 tokens of its channels into (A, B), the (A, B) of
// the stretches before it are joined in their order, and with the state that gives it goes over its 16 tokens again, which
// are still in its registers.  Backward the same runs from the end: e_t = a_t (u_t + e_{t+1}) with u_t = dy_t gate_t is what token t
// hands to the one before it, dh_t = u_t + e_{t+1}; h itself is worked out again from the state the forward pass kept
// for every 16th token.  Inputs are read once and outputs written once, which bounds both passes by memory.
//
// A warp has 32 * V channels (V = 2: a 128-byte line of bf16 a row) and 16 tokens at a time.  Where sequences are few, a
// cluster of CTAs shares one: each CTA has 8 warps, one after the other in time, and the CTAs of a cluster follow one
// another; (A, B) of a CTA goes to the others through distributed shared memory, one cluster barrier a stretch of
// (CTAs * 128) tokens.  Where channels and sequences alone fill the GPU (or a sequence is one stretch), each warp takes a whole sequence by itself.
// The order of joining is fixed by the sizes: the same inputs give the same bits.
#include "stream_common.cuh"
#include "../../include/fax_ops.h"

namespace {

constexpr int WARPS = 8;
constexpr int STEPS = FAX_RECURRENCE_BLOCK;      // tokens of a thread
constexpr int MAX_CLUSTER = 8;                   // portable

struct RecurrenceParams {
  int32_t rows, d, n_seq, seq, tiles;
  const int32_t* offsets;
  const void *f, *x, *g, *dy;
  void *y, *df, *dx, *dg;
  int64_t ldf, ldx, ldg, lddy, ldy, lddf, lddx, lddg;
  const float *h0, *dh_last;
  float *h_last, *states, *dh0;
  int32_t units;                                 // sequences * tiles
};

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cluster_size() { uint32_t r; asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void store_remote(const float2* here, uint32_t rank, float2 v) {
  uint32_t a = (uint32_t)__cvta_generic_to_shared(here), r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(r), "f"(v.x), "f"(v.y) : "memory");
}

// sigmoid(f) and sigmoid(-f), both with a small relative error (where a is close to 1, 1 - a is what a channel forgets): the
// larger one is 1 / (1 + e) with e = exp(-|f|), the smaller one e times that.  bf16 inputs take the hardware's exponential and
// reciprocal (4e-7 of the value at |f| = 8, against 2e-3 of f's and the outputs' own rounding), float inputs the library's.
template <typename T>
__device__ __forceinline__ void gates(float f, float* a, float* rest) {
  float e, big;
  if constexpr (sizeof(T) == 2) {
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fabsf(f) * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(big) : "f"(1.f + e));
  } else {
    e = expf(-fabsf(f));
    big = 1.f / (1.f + e);
  }
  const float small = e * big;
  *a = f < 0.f ? small : big;
  *rest = f < 0.f ? big : small;
}
// g sigmoid(g)
template <typename T>
__device__ __forceinline__ float silu(float g) { float s, r; gates<T>(g, &s, &r); return g * s; }

template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load_row(const T* p, bool live) {
  Pack<T, V> v;
  if (live) v = load_pack<T, V>(p);
  else {
#pragma unroll
    for (int i = 0; i < V; ++i) v.e[i] = from_f32<T>(0.f);
  }
  return v;
}

// The same value, of which the compiler knows nothing: what was worked out from it before is worked out again instead of
// being kept in registers that are not there.
template <typename P>
__device__ __forceinline__ void forget(P& v) {
  if constexpr (sizeof(P) == 2) asm volatile("" : "+h"(reinterpret_cast<unsigned short&>(v)));
  else asm volatile("" : "+r"(reinterpret_cast<unsigned&>(v)));
}

// Which stretch of which sequence a warp works on.
template <int V, bool CLUSTER>
struct Place {
  int warp, lane, unit, seq, channel, slot, n;   // slot: place in time among the warps that share the sequence
  uint32_t rank, ctas;
  int64_t lo;                                    // first row
  int64_t block0;                                // first kept state
  bool channel_live;
  int span;                                      // tokens of a round
  __device__ __forceinline__ bool set(const RecurrenceParams& p) {
    warp = threadIdx.x / 32; lane = threadIdx.x % 32;
    if (CLUSTER) {
      rank = cluster_rank(); ctas = cluster_size();
      unit = blockIdx.x / ctas;
      slot = rank * WARPS + warp;
      span = ctas * WARPS * STEPS;
    } else {
      rank = 0; ctas = 1;
      unit = blockIdx.x * WARPS + warp;
      slot = 0;
      span = STEPS;
      if (unit >= p.units) return false;
    }
    seq = unit / p.tiles;
    channel = ((unit - seq * p.tiles) * 32 + lane) * V;
    channel_live = channel < p.d;
    if (p.offsets) {
      const int a = min(max(p.offsets[seq], 0), p.rows), b = min(max(p.offsets[seq + 1], a), p.rows);
      lo = a; n = b - a;
    } else {
      lo = (int64_t)seq * p.seq; n = p.seq;
    }
    block0 = lo / STEPS + seq;
    return true;
  }
};

// What the warps and CTAs of a cluster tell one another: (A, B) of each warp, and of each CTA.  Two of each in turn, so that one
// barrier a round is enough: nobody writes a place again before all have passed the barrier after its reading.
template <int V>
struct Exchange {
  float2 warps[2][WARPS][32 * V];
  float2 ctas[2][MAX_CLUSTER][32 * V];
};

// Joins the stretches of a round.  (A, B): this warp's; carry: the state before the round, afterwards the state behind it;
// returns the state before this warp's stretch in `start`.  FORWARD: earlier slots come first; else later ones.
template <int V, bool FORWARD>
__device__ __forceinline__ void join(Exchange<V>& ex, const Place<V, true>& at, int parity, const float* A, const float* B, float* carry, float* start) {
#pragma unroll
  for (int v = 0; v < V; ++v) ex.warps[parity][at.warp][at.lane * V + v] = make_float2(A[v], B[v]);
  __syncthreads();
  float pa[V], pb[V], ta[V], tb[V];
#pragma unroll
  for (int v = 0; v < V; ++v) { pa[v] = ta[v] = 1.f; pb[v] = tb[v] = 0.f; }
#pragma unroll
  for (int i = 0; i < WARPS; ++i) {
    const int w = FORWARD ? i : WARPS - 1 - i;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (w == at.warp) { pa[v] = ta[v]; pb[v] = tb[v]; }
      const float2 s = ex.warps[parity][w][at.lane * V + v];
      ta[v] *= s.x;
      tb[v] = fmaf(s.x, tb[v], s.y);
    }
  }
  if (at.ctas == 1) {
#pragma unroll
    for (int v = 0; v < V; ++v) { start[v] = fmaf(pa[v], carry[v], pb[v]); carry[v] = fmaf(ta[v], carry[v], tb[v]); }
    return;
  }
  for (uint32_t r = at.warp; r < at.ctas; r += WARPS) {
#pragma unroll
    for (int v = 0; v < V; ++v) store_remote(&ex.ctas[parity][at.rank][at.lane * V + v], r, make_float2(ta[v], tb[v]));
  }
  cluster_sync();
  for (uint32_t i = 0; i < at.ctas; ++i) {
    const uint32_t c = FORWARD ? i : at.ctas - 1 - i;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (c == at.rank) start[v] = fmaf(pa[v], carry[v], pb[v]);
      const float2 s = ex.ctas[parity][c][at.lane * V + v];
      carry[v] = fmaf(s.x, carry[v], s.y);
    }
  }
}

template <typename T, int V, bool GATE, bool COMPLEMENT, bool CLUSTER>
__global__ void __launch_bounds__(WARPS * 32, 2) recurrence_forward_kernel(const RecurrenceParams p) {
  __shared__ Exchange<V> ex;                      // of clusters only
  if (CLUSTER && cluster_size() > 1) cluster_sync();                             // the others run: their shared memory can be written
  fax_grid_dependency_wait();
  Place<V, CLUSTER> at;
  if (!at.set(p)) return;
  const int64_t sc = (int64_t)at.seq * p.d + at.channel;
  float carry[V];
#pragma unroll
  for (int v = 0; v < V; ++v) carry[v] = at.channel_live && p.h0 ? p.h0[sc + v] : 0.f;
  int parity = 0;
  for (int t0 = 0; t0 < at.n; t0 += at.span, parity ^= 1) {
    const int ts = t0 + at.slot * STEPS;
    const int left = at.channel_live ? at.n - ts : 0;           // tokens of this thread's stretch: those up to `left`
    const int64_t row = at.lo + ts;
    const T* pf = (const T*)p.f + row * p.ldf + at.channel;
    const T* px = (const T*)p.x + row * p.ldx + at.channel;
    const T* pg = GATE ? (const T*)p.g + row * p.ldg + at.channel : nullptr;
    Pack<T, V> f[STEPS], x[STEPS], g[STEPS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      f[i] = load_row<T, V>(pf + i * p.ldf, i < left);
      x[i] = load_row<T, V>(px + i * p.ldx, i < left);
      if (GATE) g[i] = load_row<T, V>(pg + i * p.ldg, i < left);
    }
    T* py = (T*)p.y + row * p.ldy + at.channel;
    float* state = p.states + (at.block0 + ts / STEPS) * p.d + at.channel;
    const bool keep = p.states && left > 0;
    if constexpr (CLUSTER) {
      float a[STEPS][V], b[STEPS][V], A[V], B[V], h[V];
#pragma unroll
      for (int v = 0; v < V; ++v) { A[v] = 1.f; B[v] = 0.f; }
#pragma unroll
      for (int i = 0; i < STEPS; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          float rest;
          gates<T>(to_f32(f[i].e[v]), &a[i][v], &rest);
          b[i][v] = COMPLEMENT ? rest * to_f32(x[i].e[v]) : to_f32(x[i].e[v]);
          if (i >= left) { a[i][v] = 1.f; b[i][v] = 0.f; }
          A[v] *= a[i][v];
          B[v] = fmaf(a[i][v], B[v], b[i][v]);
        }
      join<V, true>(ex, at, parity, A, B, carry, h);
      if (keep) {
#pragma unroll
        for (int v = 0; v < V; ++v) state[v] = h[v];
      }
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        Pack<T, V> y;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          h[v] = fmaf(a[i][v], h[v], b[i][v]);
          y.e[v] = from_f32<T>(GATE ? h[v] * silu<T>(to_f32(g[i].e[v])) : h[v]);
        }
        if (i < left) store_pack<T, V>(py + i * p.ldy, y);
      }
    } else {
      if (keep) {
#pragma unroll
        for (int v = 0; v < V; ++v) state[v] = carry[v];
      }
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        if (i >= left) break;
        Pack<T, V> y;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          float a, rest;
          gates<T>(to_f32(f[i].e[v]), &a, &rest);
          carry[v] = fmaf(a, carry[v], COMPLEMENT ? rest * to_f32(x[i].e[v]) : to_f32(x[i].e[v]));
          y.e[v] = from_f32<T>(GATE ? carry[v] * silu<T>(to_f32(g[i].e[v])) : carry[v]);
        }
        store_pack<T, V>(py + i * p.ldy, y);
      }
    }
  }
  if (p.h_last && at.slot == 0 && at.channel_live) {
#pragma unroll
    for (int v = 0; v < V; ++v) p.h_last[sc + v] = carry[v];
  }
}

template <typename T, int V, bool GATE, bool COMPLEMENT, bool CLUSTER>
__global__ void __launch_bounds__(WARPS * 32, 2) recurrence_backward_kernel(const RecurrenceParams p) {
  __shared__ Exchange<V> ex;
  __shared__ float before[STEPS][WARPS][32 * V];  // h before each token: a thread's own places (kept in registers beside four rows of inputs they spill)
  if (CLUSTER && cluster_size() > 1) cluster_sync();
  fax_grid_dependency_wait();
  Place<V, CLUSTER> at;
  if (!at.set(p)) return;
  const int64_t sc = (int64_t)at.seq * p.d + at.channel;
  float carry[V];                                                // e behind the round: what its last token receives
#pragma unroll
  for (int v = 0; v < V; ++v) carry[v] = at.channel_live && p.dh_last ? p.dh_last[sc + v] : 0.f;
  int parity = 0;
  for (int t0 = at.n > 0 ? (at.n - 1) / at.span * at.span : -1; t0 >= 0; t0 -= at.span, parity ^= 1) {
    const int ts = t0 + at.slot * STEPS;
    const int left = at.channel_live ? at.n - ts : 0;
    const int64_t row = at.lo + ts;
    const T* pf = (const T*)p.f + row * p.ldf + at.channel;
    const T* px = (const T*)p.x + row * p.ldx + at.channel;
    const T* pg = GATE ? (const T*)p.g + row * p.ldg + at.channel : nullptr;
    const T* pdy = (const T*)p.dy + row * p.lddy + at.channel;
    Pack<T, V> f[STEPS], x[STEPS], g[STEPS], dy[STEPS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      f[i] = load_row<T, V>(pf + i * p.ldf, i < left);
      x[i] = load_row<T, V>(px + i * p.ldx, i < left);
      if (GATE) g[i] = load_row<T, V>(pg + i * p.ldg, i < left);
      dy[i] = load_row<T, V>(pdy + i * p.lddy, i < left);
    }
    float h[V];
    const float* s = p.states + (at.block0 + ts / STEPS) * p.d + at.channel;
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = left > 0 ? s[v] : 0.f;
    float e[V];
#pragma unroll
    for (int i = 0; i < STEPS; ++i)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        before[i][at.warp][at.lane * V + v] = h[v];
        float a, rest;
        gates<T>(to_f32(f[i].e[v]), &a, &rest);
        h[v] = fmaf(a, h[v], COMPLEMENT ? rest * to_f32(x[i].e[v]) : to_f32(x[i].e[v]));
      }
    if constexpr (CLUSTER) {
      float A[V], B[V];                                           // the stretch's, from its end
#pragma unroll
      for (int v = 0; v < V; ++v) { A[v] = 1.f; B[v] = 0.f; }
#pragma unroll
      for (int i = STEPS - 1; i >= 0; --i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          float a, rest;
          if (v == 0) forget(f[i]);
          gates<T>(to_f32(f[i].e[v]), &a, &rest);
          const float u = GATE ? to_f32(dy[i].e[v]) * silu<T>(to_f32(g[i].e[v])) : to_f32(dy[i].e[v]);
          if (i >= left) a = 1.f;                                 // u is 0 there
          A[v] *= a;
          B[v] = a * (u + B[v]);
        }
      join<V, false>(ex, at, parity, A, B, carry, e);
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) e[v] = carry[v];
    }
    T* pdf = (T*)p.df + row * p.lddf + at.channel;
    T* pdx = (T*)p.dx + row * p.lddx + at.channel;
    T* pdg = GATE ? (T*)p.dg + row * p.lddg + at.channel : nullptr;
#pragma unroll
    for (int i = STEPS - 1; i >= 0; --i) {
      Pack<T, V> df, dx, dg;
      forget(f[i]);
      if (GATE) forget(g[i]);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float a, rest, u = to_f32(dy[i].e[v]);
        gates<T>(to_f32(f[i].e[v]), &a, &rest);
        const float xv = to_f32(x[i].e[v]), hb = before[i][at.warp][at.lane * V + v];
        if (GATE) {
          const float gv = to_f32(g[i].e[v]);
          float sg, sr;
          gates<T>(gv, &sg, &sr);
          const float ht = fmaf(a, hb, COMPLEMENT ? rest * xv : xv);
          dg.e[v] = from_f32<T>(u * ht * fmaf(gv * sg, sr, sg));
          u *= gv * sg;
        }
        const float dh = u + e[v];
        df.e[v] = from_f32<T>(dh * (COMPLEMENT ? hb - xv : hb) * (a * rest));
        dx.e[v] = from_f32<T>(COMPLEMENT ? dh * rest : dh);
        if (i < left) e[v] = a * dh;
      }
      if (i < left) {
        store_pack<T, V>(pdf + i * p.lddf, df);
        store_pack<T, V>(pdx + i * p.lddx, dx);
        if (GATE) store_pack<T, V>(pdg + i * p.lddg, dg);
      }
    }
    if constexpr (!CLUSTER) {
#pragma unroll
      for (int v = 0; v < V; ++v) carry[v] = e[v];
    }
  }
  if (p.dh0 && at.slot == 0 && at.channel_live) {
#pragma unroll
    for (int v = 0; v < V; ++v) p.dh0[sc + v] = carry[v];
  }
}

// fax_launch, with clusters of `cluster` CTAs where there is more than one.
fax_status launch(fax_ctx* ctx, void (*kernel)(RecurrenceParams), int64_t grid, int cluster, const RecurrenceParams& p) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid); cfg.blockDim = dim3(WARPS * 32); cfg.stream = ctx->stream;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = ctx->use_pdl ? 2 : 1;
  (void)cudaLaunchKernelEx(&cfg, kernel, p);          // errors surface in fax_after_launch
  return fax_after_launch(ctx);
}

template <bool BACKWARD, typename T, int V, bool CLUSTER>
void (*pick(bool gate, bool complement))(RecurrenceParams) {
  if constexpr (BACKWARD) {
    if (gate) return complement ? recurrence_backward_kernel<T, V, true, true, CLUSTER> : recurrence_backward_kernel<T, V, true, false, CLUSTER>;
    return complement ? recurrence_backward_kernel<T, V, false, true, CLUSTER> : recurrence_backward_kernel<T, V, false, false, CLUSTER>;
  } else {
    if (gate) return complement ? recurrence_forward_kernel<T, V, true, true, CLUSTER> : recurrence_forward_kernel<T, V, true, false, CLUSTER>;
    return complement ? recurrence_forward_kernel<T, V, false, true, CLUSTER> : recurrence_forward_kernel<T, V, false, false, CLUSTER>;
  }
}

template <bool BACKWARD>
fax_status run(fax_ctx* ctx, int prec, RecurrenceParams p, bool complement, bool pairs) {
  const int v = pairs ? 2 : 1;
  p.tiles = (p.d + 32 * v - 1) / (32 * v);
  const int64_t units = (int64_t)p.n_seq * p.tiles;
  if (units > 0x7fffffff / MAX_CLUSTER) return FAX_ERR_UNSUPPORTED_SHAPE;
  p.units = (int32_t)units;
  // A warp for each sequence and channel tile where that is 8 warps an SM or a sequence is one stretch; else CTAs up to
  // two an SM, as far as the longest sequence has stretches of 128 tokens for them.
  const bool alone = units >= 8 * ctx->sm_count || p.seq <= STEPS;
  int cluster = 1;
  while (!alone && cluster < MAX_CLUSTER && cluster * WARPS * STEPS < p.seq && units * cluster < 2 * ctx->sm_count) cluster *= 2;
  const int64_t grid = alone ? (units + WARPS - 1) / WARPS : units * cluster;
  const bool gate = p.g != nullptr;
  void (*kernel)(RecurrenceParams);
  if (prec == FAX_PREC_BF16) {
    if (pairs) kernel = alone ? pick<BACKWARD, bf16, 2, false>(gate, complement) : pick<BACKWARD, bf16, 2, true>(gate, complement);
    else kernel = alone ? pick<BACKWARD, bf16, 1, false>(gate, complement) : pick<BACKWARD, bf16, 1, true>(gate, complement);
  } else {
    kernel = alone ? pick<BACKWARD, float, 1, false>(gate, complement) : pick<BACKWARD, float, 1, true>(gate, complement);
  }
  return launch(ctx, kernel, grid, cluster, p);
}

// Sizes, sequences and inputs that both passes share; `ok` with rows = 0 as well.
template <typename D>
fax_status check(fax_ctx* ctx, int prec, const D* d) {
  if (!ctx || !d || (prec != FAX_PREC_BF16 && prec != FAX_PREC_FP32_VALIDATE)) return FAX_ERR_INVALID_ARG;
  if (d->rows < 0 || d->d < 1 || d->n_seq < 0 || d->seq < 0) return FAX_ERR_INVALID_ARG;
  if (d->input != FAX_RECURRENCE_PLAIN && d->input != FAX_RECURRENCE_COMPLEMENT) return FAX_ERR_INVALID_ARG;
  if (!d->offsets && (int64_t)d->n_seq * d->seq != d->rows) return FAX_ERR_INVALID_ARG;
  if (d->ldf < d->d || d->ldx < d->d || (d->g && d->ldg < d->d)) return FAX_ERR_INVALID_ARG;
  if (d->rows > 0 && (!d->f || !d->x)) return FAX_ERR_INVALID_ARG;
  const size_t es = fax_elem_size(prec);
  if (!fax_aligned(d->f, es) || !fax_aligned(d->x, es) || !fax_aligned(d->g, es) || !fax_aligned(d->offsets, 4) || !fax_aligned(d->h0, 4) || !fax_aligned(d->states, 4))
    return FAX_ERR_INVALID_ARG;
  if (d->rows > (1 << 30) || d->d > (1 << 24)) return FAX_ERR_UNSUPPORTED_SHAPE;
  return FAX_OK;
}

template <typename D>
RecurrenceParams params(const D* d) {
  RecurrenceParams p = {};
  p.rows = d->rows; p.d = d->d; p.n_seq = d->n_seq; p.seq = d->seq; p.offsets = d->offsets;
  p.f = d->f; p.x = d->x; p.g = d->g; p.ldf = d->ldf; p.ldx = d->ldx; p.ldg = d->ldg;
  p.h0 = d->h0;
  return p;
}

// Two bf16 channels a lane: even widths and pitches, addresses of whole pairs.
bool pair(const void* p, int64_t ld) { return !p || fax_rows_aligned(p, ld, 2, 4); }

}  // namespace

extern "C" fax_status fax_op_recurrence_states_floats(int32_t rows, int32_t n_seq, int32_t d, size_t* floats) {
  if (!floats || rows < 0 || n_seq < 0 || d < 1) return FAX_ERR_INVALID_ARG;
  *floats = ((size_t)rows / STEPS + (size_t)n_seq) * (size_t)d;
  return FAX_OK;
}

extern "C" fax_status fax_op_recurrence_forward(fax_ctx* ctx, int32_t prec, const fax_recurrence_desc* d) {
  FAX_TRY(check(ctx, prec, d));
  if (d->rows > 0 && (!d->y || d->ldy < d->d)) return FAX_ERR_INVALID_ARG;
  if (!fax_aligned(d->y, fax_elem_size(prec)) || !fax_aligned(d->h_last, 4)) return FAX_ERR_INVALID_ARG;
  if (d->n_seq == 0) return FAX_OK;
  RecurrenceParams p = params(d);
  p.y = d->y; p.ldy = d->ldy; p.h_last = d->h_last; p.states = d->states;
  const double n = (double)d->rows * d->d, es = (double)fax_elem_size(prec);
  FaxProfScope prof(ctx, KC_RECURRENCE, 4.0 * n, (3.0 + (d->g != nullptr)) * n * es + (d->states ? n / 4 : 0.0));
  const bool pairs = prec == FAX_PREC_BF16 && d->d % 2 == 0 && pair(d->f, d->ldf) && pair(d->x, d->ldx) && pair(d->g, d->ldg) && pair(d->y, d->ldy);
  return run<false>(ctx, prec, p, d->input == FAX_RECURRENCE_COMPLEMENT, pairs);
}

extern "C" fax_status fax_op_recurrence_backward(fax_ctx* ctx, int32_t prec, const fax_recurrence_backward_desc* d) {
  FAX_TRY(check(ctx, prec, d));
  const size_t esz = fax_elem_size(prec);
  if (d->rows > 0 && (!d->dy || !d->df || !d->dx || !d->states || (d->g && !d->dg))) return FAX_ERR_INVALID_ARG;
  if (d->rows > 0 && (d->lddy < d->d || d->lddf < d->d || d->lddx < d->d || (d->g && d->lddg < d->d))) return FAX_ERR_INVALID_ARG;
  if (!fax_aligned(d->dy, esz) || !fax_aligned(d->df, esz) || !fax_aligned(d->dx, esz) || !fax_aligned(d->dg, esz) || !fax_aligned(d->dh_last, 4) || !fax_aligned(d->dh0, 4))
    return FAX_ERR_INVALID_ARG;
  if ((d->df == d->f && d->lddf != d->ldf) || (d->dx == d->x && d->lddx != d->ldx) || (d->g && d->dg == d->g && d->lddg != d->ldg)) return FAX_ERR_INVALID_ARG;
  if (d->n_seq == 0) return FAX_OK;
  RecurrenceParams p = params(d);
  p.states = const_cast<float*>(d->states);
  p.dy = d->dy; p.lddy = d->lddy; p.dh_last = d->dh_last; p.dh0 = d->dh0;
  p.df = d->df; p.lddf = d->lddf; p.dx = d->dx; p.lddx = d->lddx; p.dg = d->dg; p.lddg = d->lddg;
  const double n = (double)d->rows * d->d, es = (double)esz;
  FaxProfScope prof(ctx, KC_RECURRENCE, 10.0 * n, (5.0 + 2.0 * (d->g != nullptr)) * n * es + n / 4);
  const bool pairs = prec == FAX_PREC_BF16 && d->d % 2 == 0 && pair(d->f, d->ldf) && pair(d->x, d->ldx) && pair(d->g, d->ldg) && pair(d->dy, d->lddy) &&
                     pair(d->df, d->lddf) && pair(d->dx, d->lddx) && (!d->g || pair(d->dg, d->lddg));
  return run<true>(ctx, prec, p, d->input == FAX_RECURRENCE_COMPLEMENT, pairs);
}
