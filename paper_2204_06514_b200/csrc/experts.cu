// Tokens to their experts and back (see fax_ops.h).
//
// The places: a counting sort that keeps the order, in one launch of one cluster.  Each CTA has a consecutive part of the choices,
// each of its warps a consecutive part of that, and each warp counts its experts 32 choices at a time (the lanes with the same expert
// find one another by a ballot for each bit of the expert's number).  The counts are summed over warps in shared memory and over CTAs through distributed shared
// memory, which gives every warp the first slot of each expert for its own choices; a second walk over the (cached) ids hands the slots out.
// Nothing is stored in between and nothing depends on an order of atomics.  Latency bounds it.
//
// The rows: memory bounds them.  A group of threads has a token: its row is read once and written to (or read from) the slots of all
// its choices, a 16-byte vector at a time; groups before the tokens' look for empty slots and zero them.
#include "stream_common.cuh"
#include "../../include/fax_ops.h"

namespace {

// ---- the places ----

constexpr int SORT_WARPS = 32;                  // of a CTA at most
constexpr int SORT_CLUSTER = 16;
constexpr int GROUPS = 4;                       // of 32 choices that a warp has in registers at a time

struct SortParams {
  int32_t choices, experts, capacity, align, slots;
  const int32_t* ids;
  int32_t *slot_of, *source, *offsets, *counts;
};

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cluster_size() { uint32_t r; asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void store_remote(const int32_t* here, uint32_t rank, int32_t v) {
  uint32_t a = (uint32_t)__cvta_generic_to_shared(here), r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(r), "r"(v) : "memory");
}

// The lanes with the same x as this one, x of `bits` bits: a ballot a bit (match.any takes longer the more values there are).
__device__ __forceinline__ uint32_t alike(int x, int bits) {
  uint32_t same = 0xffffffffu;
  for (int b = 0; b < bits; ++b) {
    const uint32_t ones = __ballot_sync(0xffffffffu, (x >> b) & 1);
    same &= ((x >> b) & 1) ? ones : ~ones;
  }
  return same;
}

__device__ __forceinline__ int warp_inclusive(int v) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, v, o);
    if ((int)(threadIdx.x % 32) >= o) v += u;
  }
  return v;
}

// Shared memory: counts of each warp [warps][experts], of each CTA [CTAs][experts], first slots [experts].
__global__ void __launch_bounds__(SORT_WARPS * 32) expert_sort_kernel(const SortParams p) {
  extern __shared__ int32_t mem[];
  const uint32_t rank = cluster_rank(), n_ctas = cluster_size();
  const int threads = blockDim.x, n_warps = threads / 32, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  int32_t* const mine = mem;
  int32_t* const ctas = mem + n_warps * p.experts;
  int32_t* const first = ctas + n_ctas * p.experts;
  __shared__ int32_t sums[SORT_WARPS + 1];
  const uint32_t before_me = (1u << lane) - 1;
  for (int i = threadIdx.x; i < n_warps * p.experts; i += threads) mine[i] = 0;
  __syncthreads();
  if (n_ctas > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  fax_grid_dependency_wait();

  // this warp's choices: whole groups of 32, GROUPS of them read at a time; the first ones stay for the second walk
  const int64_t groups = ((int64_t)p.choices + 31) / 32, warps = (int64_t)n_ctas * n_warps, me = (int64_t)rank * n_warps + warp;
  const int64_t lo = groups * me / warps * 32, hi = min(groups * (me + 1) / warps * 32, (int64_t)p.choices);
  int32_t* const count = mine + warp * p.experts;
  const int bits = 32 - __clz(p.experts);         // of 0 to experts
  int x[GROUPS];
  uint32_t same[GROUPS];
  auto read = [&](int64_t c) {
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) {
      const int64_t at = c + 32 * k + lane;
      x[k] = at < hi ? p.ids[at] : -1;
      if ((uint32_t)x[k] >= (uint32_t)p.experts) x[k] = p.experts;                // none
    }
#pragma unroll
    for (int k = 0; k < GROUPS; ++k)
      if (c + 32 * k < hi) same[k] = alike(x[k], bits);
  };
  // (from the end, so that the first ones are read last)
  const int64_t last = lo < hi ? lo + (hi - lo - 1) / (32 * GROUPS) * (32 * GROUPS) : lo - 1;
  for (int64_t c = last; c >= lo; c -= 32 * GROUPS) {
    read(c);
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) {
      if (c + 32 * k >= hi) break;
      if (x[k] < p.experts && (same[k] & before_me) == 0) count[x[k]] += __popc(same[k]);
      __syncwarp();
    }
  }
  __syncthreads();
  // over the warps: what each starts from within the CTA, and the CTA's counts for everyone
  if (n_ctas > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");              // the others run: their shared memory can be written
  for (int e = threadIdx.x; e < p.experts; e += threads) {
    int sum = 0;
#pragma unroll 8
    for (int w = 0; w < n_warps; ++w) {
      const int n = mine[w * p.experts + e];
      mine[w * p.experts + e] = sum;
      sum += n;
    }
    if (n_ctas == 1) ctas[e] = sum;
    else for (uint32_t r = 0; r < n_ctas; ++r) store_remote(&ctas[rank * p.experts + e], r, sum);
  }
  if (n_ctas > 1) cluster_sync(); else __syncthreads();
  // each expert's first slot: a thread has one expert
  const int e = threadIdx.x;
  int total = 0, earlier = 0, room = 0;
  if (e < p.experts) {
    for (uint32_t r = 0; r < n_ctas; ++r) {
      if (r == rank) earlier = total;
      total += ctas[r * p.experts + e];
    }
    room = p.capacity ? p.capacity : (total + p.align - 1) / p.align * p.align;
  }
  const int through = warp_inclusive(room);
  if (lane == 31) sums[warp] = through;
  __syncthreads();
  // (every warp adds up the warps before it)
  const int v = warp_inclusive(lane < n_warps ? sums[lane] : 0);
  const int before = __shfl_sync(0xffffffffu, v, (warp + 31) % 32), end = __shfl_sync(0xffffffffu, v, 31);
  const int slot0 = (warp ? before : 0) + through - room;
  if (e < p.experts) {
    first[e] = (int)((uint32_t)slot0 + (uint32_t)earlier);
    if (rank == 0) {
      p.counts[e] = total;
      p.offsets[e] = slot0;
      if (e == p.experts - 1) p.offsets[p.experts] = end;
    }
  }
  __syncthreads();
  // the slots
  for (int64_t c = lo; c < hi; c += 32 * GROUPS) {
    if (c > lo) read(c);
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) {
      if (c + 32 * k >= hi) break;
      int slot = -1;
      if (x[k] < p.experts) {
        const uint32_t next = (uint32_t)first[x[k]] + (uint32_t)count[x[k]] + __popc(same[k] & before_me);     // below 2^32: slots and choices are below 2^31
        slot = p.capacity && next >= (int64_t)(x[k] + 1) * p.capacity ? -1 : (int)next;
      }
      __syncwarp();
      if (x[k] < p.experts && (same[k] & before_me) == 0) count[x[k]] += __popc(same[k]);
      __syncwarp();
      const int64_t at = c + 32 * k + lane;
      if (at < hi) {
        p.slot_of[at] = slot;
        if (slot >= 0) p.source[slot] = (int32_t)at;
      }
    }
  }
  // empty slots: behind an expert's choices (a warp an expert), and behind the last expert
  for (int q = rank * n_warps + warp; q < p.experts; q += n_ctas * n_warps) {
    int all = 0, others = 0;
    for (uint32_t r = 0; r < n_ctas; ++r) {
      if (r == rank) others = all;
      all += ctas[r * p.experts + q];
    }
    const uint32_t start = (uint32_t)first[q] - (uint32_t)others;
    const int64_t stop = (int64_t)start + (p.capacity ? p.capacity : (all + p.align - 1) / p.align * p.align);
    for (int64_t s = (int64_t)start + all + lane; s < stop; s += 32) p.source[s] = -1;
  }
  for (int64_t s = end + (int64_t)rank * threads + threadIdx.x; s < p.slots; s += (int64_t)n_ctas * threads) p.source[s] = -1;
}

// ---- the rows ----

constexpr int ROW_THREADS = 256;

struct RowParams {
  int32_t n_tokens, top_k, d, slots;
  int64_t slot_groups;                // groups of threads that look for empty slots; those behind have a token each
  const int32_t* slot_of; const int32_t* source;
  const float* weights;
  const void *in, *resid, *z; void *out;
  int64_t ld_in, ld_resid, ld_z, ld_out;
  float* dw;
};

__device__ __forceinline__ int slot_at(const RowParams& p, int64_t token, int j) {
  const int s = j < p.top_k ? p.slot_of[token * p.top_k + j] : -1;
  return (uint32_t)s < (uint32_t)p.slots ? s : -1;
}

// Zeros in the empty ones of the 32 slots from s0 on: the group's warps look at them together and take a row in turn.
template <typename T, int N, int GROUP>
__device__ __forceinline__ void zero_slots(const RowParams& p, int64_t s0) {
  const int lane = threadIdx.x % 32, in_group = threadIdx.x % GROUP;
  const int64_t s = s0 + lane;
  uint32_t empty = __ballot_sync(0xffffffffu, s < p.slots && p.source[s] < 0);
  Pack<T, N> zero;
#pragma unroll
  for (int i = 0; i < N; ++i) zero.e[i] = from_f32<T>(0.f);
  for (; empty; empty &= empty - 1) {
    T* row = (T*)p.out + (s0 + __ffs(empty) - 1) * p.ld_out;
    for (int v = in_group; v < p.d / N; v += GROUP) store_pack<T, N>(row + v * N, zero);
  }
}

// K: choices of a token that a thread works on at a time.  GROUP: threads of a token, a warp or the block.
template <typename T, int N, int GROUP, int K>
__global__ void __launch_bounds__(ROW_THREADS, 4) dispatch_kernel(const RowParams p) {
  constexpr int U = 4;                            // vectors on their way together
  fax_grid_dependency_wait();
  const int lane = threadIdx.x % GROUP;
  int64_t item = (int64_t)blockIdx.x * (ROW_THREADS / GROUP) + threadIdx.x / GROUP;
  if (item < p.slot_groups) { zero_slots<T, N, GROUP>(p, item * 32); return; }
  item -= p.slot_groups;
  if (item >= p.n_tokens) return;
  const T* row = (const T*)p.in + item * p.ld_in;
  const int vectors = p.d / N;
  for (int j0 = 0; j0 < p.top_k; j0 += K) {
    int slot[K];
#pragma unroll
    for (int j = 0; j < K; ++j) slot[j] = slot_at(p, item, j0 + j);
    for (int v0 = lane; v0 < vectors; v0 += GROUP * U) {
      Pack<T, N> x[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (v0 + u * GROUP < vectors) x[u] = load_pack<T, N>(row + (v0 + u * GROUP) * N);
#pragma unroll
      for (int j = 0; j < K; ++j)
        if (slot[j] >= 0) {
          T* out = (T*)p.out + (int64_t)slot[j] * p.ld_out + v0 * N;
#pragma unroll
          for (int u = 0; u < U; ++u)
            if (v0 + u * GROUP < vectors) store_pack<T, N>(out + u * GROUP * N, x[u]);
        }
    }
  }
}

template <typename T, int N, int GROUP, int K>
__global__ void __launch_bounds__(ROW_THREADS, K > 4 ? 2 : 4) combine_kernel(const RowParams p) {
  fax_grid_dependency_wait();
  const int lane = threadIdx.x % GROUP;
  const int64_t item = (int64_t)blockIdx.x * (ROW_THREADS / GROUP) + threadIdx.x / GROUP;
  if (item >= p.n_tokens) return;
  int slot[K]; float w[K];
  auto fetch = [&](int j0) {
#pragma unroll
    for (int j = 0; j < K; ++j) {
      slot[j] = slot_at(p, item, j0 + j);
      w[j] = slot[j] >= 0 && p.weights ? p.weights[item * p.top_k + j0 + j] : 1.f;
    }
  };
  fetch(0);
  for (int v = lane; v < p.d / N; v += GROUP) {
    float sum[N];
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = 0.f;
    Pack<T, N> r;
    if (p.resid) r = load_pack<T, N>((const T*)p.resid + item * p.ld_resid + v * N);
    for (int j0 = 0; j0 < p.top_k; j0 += K) {
      if (p.top_k > K) fetch(j0);
      Pack<T, N> z[K];
#pragma unroll
      for (int j = 0; j < K; ++j)
        if (slot[j] >= 0) z[j] = load_pack<T, N>((const T*)p.z + (int64_t)slot[j] * p.ld_z + v * N);
#pragma unroll
      for (int j = 0; j < K; ++j)
        if (slot[j] >= 0) {
#pragma unroll
          for (int i = 0; i < N; ++i) sum[i] = fmaf(w[j], to_f32(z[j].e[i]), sum[i]);
        }
    }
    Pack<T, N> y;
#pragma unroll
    for (int i = 0; i < N; ++i) y.e[i] = from_f32<T>(p.resid ? to_f32(r.e[i]) + sum[i] : sum[i]);
    store_pack<T, N>((T*)p.out + item * p.ld_out + v * N, y);
  }
}

// in: dy; out: dz.  The products of a choice are summed over a thread's vectors, the group's lanes by halves, its warps in order.
template <typename T, int N, int GROUP, int K>
__global__ void __launch_bounds__(ROW_THREADS, 4) combine_backward_kernel(const RowParams p) {
  __shared__ float sums[GROUP > 32 ? ROW_THREADS / 32 : 1][K];
  fax_grid_dependency_wait();
  const int lane = threadIdx.x % GROUP;
  int64_t item = (int64_t)blockIdx.x * (ROW_THREADS / GROUP) + threadIdx.x / GROUP;
  if (item < p.slot_groups) { zero_slots<T, N, GROUP>(p, item * 32); return; }
  item -= p.slot_groups;
  if (item >= p.n_tokens) return;
  const T* row = (const T*)p.in + item * p.ld_in;
  for (int j0 = 0; j0 < p.top_k; j0 += K) {
    int slot[K]; float w[K], dot[K];
#pragma unroll
    for (int j = 0; j < K; ++j) {
      slot[j] = slot_at(p, item, j0 + j);
      w[j] = slot[j] >= 0 ? p.weights[item * p.top_k + j0 + j] : 0.f;
      dot[j] = 0.f;
    }
    constexpr int U = K == 2 ? 2 : 1;             // vectors on their way together (two choices, 16384 x 1024: 37.1 -> 34.7 us; one choice loses by it, 36 -> 40 us)
    const int vectors = p.d / N;
    for (int v0 = lane; v0 < vectors; v0 += GROUP * U) {
      Pack<T, N> g[U], z[U][K];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (v0 + u * GROUP >= vectors) break;
        g[u] = load_pack<T, N>(row + (v0 + u * GROUP) * N);
        if (p.dw) {
#pragma unroll
          for (int j = 0; j < K; ++j)
            // (one choice: a row in any case, so that no branch stands before the load: 16384 x 2048 45 -> 36 us; with more choices it
            // costs.  What is read for a choice without a slot is not looked at, whoever writes there where dz is z.)
            if (K == 1 ? p.slots > 0 : slot[j] >= 0) z[u][j] = load_pack<T, N>((const T*)p.z + (int64_t)max(slot[j], 0) * p.ld_z + (v0 + u * GROUP) * N);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (v0 + u * GROUP >= vectors) break;
#pragma unroll
        for (int j = 0; j < K; ++j)
          if (slot[j] >= 0) {
            Pack<T, N> dz;
#pragma unroll
            for (int i = 0; i < N; ++i) {
              const float gi = to_f32(g[u].e[i]);
              if (p.dw) dot[j] = fmaf(to_f32(z[u][j].e[i]), gi, dot[j]);
              dz.e[i] = from_f32<T>(w[j] * gi);
            }
            store_pack<T, N>((T*)p.out + (int64_t)slot[j] * p.ld_out + (v0 + u * GROUP) * N, dz);
          }
      }
    }
    if (!p.dw) continue;
#pragma unroll
    for (int j = 0; j < K; ++j) dot[j] = warp_sum(dot[j]);
    if (GROUP > 32) {
      __syncthreads();                            // GROUP is the block then: its threads are all here
      if (threadIdx.x % 32 == 0) {
#pragma unroll
        for (int j = 0; j < K; ++j) sums[threadIdx.x / 32][j] = dot[j];
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < K; ++j) {
        dot[j] = 0.f;
#pragma unroll
        for (int q = 0; q < ROW_THREADS / 32; ++q) dot[j] += sums[q][j];
      }
    }
    if (lane == 0) {
#pragma unroll
      for (int j = 0; j < K; ++j)
        if (j0 + j < p.top_k) p.dw[item * p.top_k + j0 + j] = slot[j] >= 0 ? dot[j] : 0.f;
    }
  }
}

enum RowOp { DISPATCH, COMBINE, COMBINE_BACKWARD };

// Choices at a time (K): as many loads on their way as registers hold beside four blocks an SM; more of them in two blocks' worth
// pays where a sum is all there is to keep (6 of 64, 8191 x 2048: combine 58 us with 4 or 3 at a time, 50 us with 6; its gradient 98 us with
// 8 at a time, 82 us with 3; 4 of 16, 8192 x 2048: 33 and 60 us with 4 at a time in four blocks, 42 and 72 us in two).
template <typename T, int N, int GROUP>
fax_status launch_rows(fax_ctx* ctx, RowOp op, RowParams p) {
  constexpr int PER_BLOCK = ROW_THREADS / GROUP;
  p.slot_groups = op == COMBINE ? 0 : (((int64_t)p.slots + 31) / 32 + PER_BLOCK - 1) / PER_BLOCK * PER_BLOCK;      // whole blocks, so that none has both kinds of work
  const int64_t groups = p.slot_groups + p.n_tokens;
  const dim3 grid((unsigned)((groups + PER_BLOCK - 1) / PER_BLOCK)), threads(ROW_THREADS);
  const int k = p.top_k;
  void (*kernel)(RowParams);
  if (op == DISPATCH) kernel = k <= 2 ? dispatch_kernel<T, N, GROUP, 2> : k <= 4 ? dispatch_kernel<T, N, GROUP, 4> : dispatch_kernel<T, N, GROUP, 8>;
  else if (op == COMBINE) kernel = k == 1 ? combine_kernel<T, N, GROUP, 1> : k == 2 ? combine_kernel<T, N, GROUP, 2> : k <= 4 ? combine_kernel<T, N, GROUP, 4> : k <= 6 ? combine_kernel<T, N, GROUP, 6> : combine_kernel<T, N, GROUP, 8>;
  else kernel = k == 1 ? combine_backward_kernel<T, N, GROUP, 1> : k == 2 ? combine_backward_kernel<T, N, GROUP, 2> : k == 3 || k == 5 || k == 6 ? combine_backward_kernel<T, N, GROUP, 3> : combine_backward_kernel<T, N, GROUP, 4>;
  fax_launch(ctx, kernel, grid, threads, 0, p);
  return fax_after_launch(ctx);
}
template <typename T, int N>
fax_status launch_rows(fax_ctx* ctx, RowOp op, bool block, const RowParams& p) {
  return block ? launch_rows<T, N, ROW_THREADS>(ctx, op, p) : launch_rows<T, N, 32>(ctx, op, p);
}

// Vectors of 16 bytes where every row is whole vectors, else single elements; a block a token where tokens are few.
fax_status rows(fax_ctx* ctx, int prec, RowOp op, const RowParams& p) {
  const size_t es = fax_elem_size(prec);
  auto fits = [&](const void* q, int64_t ld) { return !q || fax_rows_aligned(q, ld, es, 16); };
  const int n = (int)(16 / es);
  const bool vec = p.d % n == 0 && fits(p.in, p.ld_in) && fits(p.resid, p.ld_resid) && fits(p.z, p.ld_z) && fits(p.out, p.ld_out);
  const bool block = (int64_t)p.n_tokens < 8 * (int64_t)ctx->sm_count && p.d > 32 * n;
  if (prec == FAX_PREC_BF16) return vec ? launch_rows<bf16, 8>(ctx, op, block, p) : launch_rows<bf16, 1>(ctx, op, block, p);
  return vec ? launch_rows<float, 4>(ctx, op, block, p) : launch_rows<float, 1>(ctx, op, block, p);
}

fax_status check(fax_ctx* ctx, int prec, const void* desc, int n_tokens, int top_k, int d, int slots) {
  if (!ctx || !desc || (prec != FAX_PREC_BF16 && prec != FAX_PREC_FP32_VALIDATE)) return FAX_ERR_INVALID_ARG;
  if (n_tokens < 0 || top_k < 1 || d < 1 || slots < 0) return FAX_ERR_INVALID_ARG;
  if ((int64_t)n_tokens * top_k > 0x7fffffff || (int64_t)n_tokens + slots > 0x7fffffff || d > (1 << 30)) return FAX_ERR_UNSUPPORTED_SHAPE;
  return FAX_OK;
}

}  // namespace

extern "C" fax_status fax_op_expert_slots(int32_t n_tokens, int32_t top_k, int32_t n_experts, int32_t capacity, int32_t align, int32_t* slots) {
  if (!slots || n_tokens < 0 || top_k < 1 || n_experts < 1 || capacity < 0 || (capacity == 0 && align < 1)) return FAX_ERR_INVALID_ARG;
  if (n_experts > FAX_EXPERT_MAX) return FAX_ERR_UNSUPPORTED_SHAPE;
  const int64_t n = (int64_t)n_tokens * top_k, used = n < n_experts ? n : n_experts;
  const int64_t s = capacity ? (int64_t)n_experts * capacity : n + used * (align - 1);
  if (n > 0x7fffffff || s > 0x7fffffff) return FAX_ERR_UNSUPPORTED_SHAPE;
  *slots = (int32_t)s;
  return FAX_OK;
}

extern "C" fax_status fax_op_expert_sort(fax_ctx* ctx, const fax_expert_sort_desc* d) {
  if (!ctx || !d) return FAX_ERR_INVALID_ARG;
  int32_t need = 0;
  FAX_TRY(fax_op_expert_slots(d->n_tokens, d->top_k, d->n_experts, d->capacity, d->align, &need));
  if (d->slots < need) return FAX_ERR_WORKSPACE_TOO_SMALL;
  if (!d->offsets || !d->counts || (d->slots > 0 && !d->source) || (d->n_tokens > 0 && (!d->ids || !d->slot_of))) return FAX_ERR_INVALID_ARG;
  if (!fax_aligned(d->ids, 4) || !fax_aligned(d->slot_of, 4) || !fax_aligned(d->source, 4) || !fax_aligned(d->offsets, 4) || !fax_aligned(d->counts, 4)) return FAX_ERR_INVALID_ARG;
  SortParams p;
  p.choices = d->n_tokens * d->top_k; p.experts = d->n_experts; p.capacity = d->capacity; p.align = d->capacity ? 1 : d->align; p.slots = d->slots;
  p.ids = d->ids; p.slot_of = d->slot_of; p.source = d->source; p.offsets = d->offsets; p.counts = d->counts;
  // Warps for every 64 choices, threads for every expert; one CTA of them, 8 or 16 (4000 choices, 128 experts: 9.9 us on one CTA, 5.1 us on 8;
  // 49146 choices, 64 experts: 15.5 us on 8, 11.4 us on 16: the slots' scattered stores).
  const int cluster = p.choices <= 1024 ? 1 : p.choices <= 8192 ? 8 : SORT_CLUSTER;
  int warps = (p.choices / cluster + 63) / 64;
  if (warps < (p.experts + 31) / 32) warps = (p.experts + 31) / 32;
  if (warps < 4) warps = 4;
  if (warps > SORT_WARPS) warps = SORT_WARPS;
  const int smem_max = (SORT_WARPS + SORT_CLUSTER + 1) * FAX_EXPERT_MAX * 4, smem = (warps + cluster + 1) * p.experts * 4;
  static bool done[FAX_MAX_DEVICES] = {};
  FAX_TRY(fax_opt_in_shared_memory(ctx, expert_sort_kernel, smem_max, done));
  static bool wide[FAX_MAX_DEVICES] = {};
  const bool tracked = ctx->device >= 0 && ctx->device < FAX_MAX_DEVICES;
  if (cluster > 8 && !(tracked && wide[ctx->device])) {
    FAX_CUDA_TRY(ctx, cudaFuncSetAttribute(expert_sort_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    if (tracked) wide[ctx->device] = true;
  }
  FaxProfScope prof(ctx, KC_EXPERT, 0.0, 4.0 * (2.0 * p.choices + p.slots + 2.0 * p.experts));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(cluster); cfg.blockDim = dim3(warps * 32); cfg.dynamicSmemBytes = smem; cfg.stream = ctx->stream;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = ctx->use_pdl ? 2 : 1;
  (void)cudaLaunchKernelEx(&cfg, expert_sort_kernel, p);          // errors surface in fax_after_launch
  return fax_after_launch(ctx);
}

extern "C" fax_status fax_op_expert_dispatch(fax_ctx* ctx, int32_t prec, const fax_expert_dispatch_desc* d) {
  FAX_TRY(d ? check(ctx, prec, d, d->n_tokens, d->top_k, d->d, d->slots) : FAX_ERR_INVALID_ARG);
  if (d->ldo < d->d || d->ldx < d->d) return FAX_ERR_INVALID_ARG;
  if (d->n_tokens == 0 && d->slots == 0) return FAX_OK;
  if ((d->n_tokens > 0 && (!d->slot_of || !d->x)) || (d->slots > 0 && (!d->source || !d->out))) return FAX_ERR_INVALID_ARG;
  const size_t es = fax_elem_size(prec);
  if (!fax_aligned(d->slot_of, 4) || !fax_aligned(d->source, 4) || !fax_aligned(d->x, es) || !fax_aligned(d->out, es)) return FAX_ERR_INVALID_ARG;
  RowParams p = {};
  p.n_tokens = d->n_tokens; p.top_k = d->top_k; p.d = d->d; p.slots = d->slots; p.slot_of = d->slot_of; p.source = d->source;
  p.in = d->x; p.ld_in = d->ldx; p.out = d->out; p.ld_out = d->ldo;
  FaxProfScope prof(ctx, KC_EXPERT, 0.0, ((double)d->n_tokens + d->slots) * d->d * es + 4.0 * ((double)d->n_tokens * d->top_k + d->slots));
  return rows(ctx, prec, DISPATCH, p);
}

extern "C" fax_status fax_op_expert_combine(fax_ctx* ctx, int32_t prec, const fax_expert_combine_desc* d) {
  FAX_TRY(d ? check(ctx, prec, d, d->n_tokens, d->top_k, d->d, d->slots) : FAX_ERR_INVALID_ARG);
  if (d->ldz < d->d || d->ldy < d->d || (d->resid && d->ldr < d->d)) return FAX_ERR_INVALID_ARG;
  if (d->n_tokens == 0) return FAX_OK;
  if (!d->slot_of || !d->y || (d->slots > 0 && !d->z)) return FAX_ERR_INVALID_ARG;
  const size_t es = fax_elem_size(prec);
  if (!fax_aligned(d->slot_of, 4) || !fax_aligned(d->weights, 4) || !fax_aligned(d->z, es) || !fax_aligned(d->resid, es) || !fax_aligned(d->y, es)) return FAX_ERR_INVALID_ARG;
  if (d->resid == d->y && d->ldr != d->ldy) return FAX_ERR_INVALID_ARG;
  RowParams p = {};
  p.n_tokens = d->n_tokens; p.top_k = d->top_k; p.d = d->d; p.slots = d->slots; p.slot_of = d->slot_of; p.weights = d->weights;
  p.z = d->z; p.ld_z = d->ldz; p.resid = d->resid; p.ld_resid = d->ldr; p.out = d->y; p.ld_out = d->ldy;
  const double n = (double)d->n_tokens, k = n * d->top_k;
  FaxProfScope prof(ctx, KC_EXPERT, 2.0 * k * d->d, (k + n + (d->resid ? n : 0.0)) * d->d * es + (d->weights ? 8.0 : 4.0) * k);
  return rows(ctx, prec, COMBINE, p);
}

extern "C" fax_status fax_op_expert_combine_backward(fax_ctx* ctx, int32_t prec, const fax_expert_combine_backward_desc* d) {
  FAX_TRY(d ? check(ctx, prec, d, d->n_tokens, d->top_k, d->d, d->slots) : FAX_ERR_INVALID_ARG);
  if (d->lddy < d->d || d->lddz < d->d || (d->dw && d->ldz < d->d)) return FAX_ERR_INVALID_ARG;
  if (d->n_tokens == 0 && d->slots == 0) return FAX_OK;
  if ((d->n_tokens > 0 && (!d->slot_of || !d->weights || !d->dy)) || (d->slots > 0 && (!d->source || !d->dz || (d->dw && !d->z)))) return FAX_ERR_INVALID_ARG;
  const size_t es = fax_elem_size(prec);
  if (!fax_aligned(d->slot_of, 4) || !fax_aligned(d->source, 4) || !fax_aligned(d->weights, 4) || !fax_aligned(d->z, es) || !fax_aligned(d->dy, es) || !fax_aligned(d->dz, es) || !fax_aligned(d->dw, 4))
    return FAX_ERR_INVALID_ARG;
  if (d->dw && d->dz == d->z && d->lddz != d->ldz) return FAX_ERR_INVALID_ARG;
  RowParams p = {};
  p.n_tokens = d->n_tokens; p.top_k = d->top_k; p.d = d->d; p.slots = d->slots; p.slot_of = d->slot_of; p.source = d->source; p.weights = d->weights;
  p.in = d->dy; p.ld_in = d->lddy; p.z = d->dw ? d->z : nullptr; p.ld_z = d->ldz; p.out = d->dz; p.ld_out = d->lddz; p.dw = d->dw;
  const double n = (double)d->n_tokens, k = n * d->top_k;
  FaxProfScope prof(ctx, KC_EXPERT, 4.0 * k * d->d, ((d->dw ? k : 0.0) + d->slots + n) * d->d * es + 12.0 * k);
  return rows(ctx, prec, COMBINE_BACKWARD, p);
}
