// Token table lookup with scaling, and its gradient by sorted tokens.
//
//   forward   out[i] = scale * table[ids[i]]                     (a zero row where ids[i] is outside the table)
//   backward  dtable[v] (+)= scale * sum_{i : ids[i] = v} dout[i]
//
// The gradient's sums run over tokens sorted by id, in the order in which the tokens stand: every row of
// the table is written once, nothing is added by float atomics, and the same call gives the same bits.
//
//  1. A least-significant-digit radix sort of the ids (8 bits a pass at most, as many passes as the
//     vocabulary needs: two for 50,304 ids).  embed_sort_count zeroes the counters and counts the first
//     digit per tile of tokens; embed_sort_scatter places a tile's tokens behind those of the tiles before
//     it, keeping their order (rank within a warp by match, then warps, then tiles), and counts the next
//     digit of the tile each token lands in (whole-number atomics: the sums do not depend on their order).
//  2. embed_grad: chunks of consecutive sorted tokens.  A run of equal ids inside a chunk is summed in
//     registers and written; a run that crosses a chunk's edge leaves partial sums (at most a first and
//     a last one per chunk).  When the table is overwritten, further blocks of the same launch zero the rows
//     that no token touches.
//  3. embed_join: adds the partial sums of each run that crossed an edge, in chunk order.
#include "common.cuh"

namespace {

constexpr int SORT_THREADS = 512;
constexpr int SORT_WARPS = SORT_THREADS / 32;
constexpr int DIGITS = 256;
constexpr int TILE_UNIT = 512;         // tokens per tile: a multiple of this
constexpr int MAX_TILES = 256;         // a scatter block reads every tile's counts of its pass
constexpr int MAX_TOKENS = 1 << 30;    // token and tile positions stay within 32 bits
constexpr int GRAD_THREADS = 128;
constexpr int JOIN_GROUPS = 8;

struct SortPlan {
  int n, tile, tiles, passes, bits;    // bits per pass
  int chunk, chunks;                   // sorted tokens per gradient chunk
};

SortPlan plan_for(int n, int vocab) {
  SortPlan p;
  p.n = n;
  const int units = (n + TILE_UNIT - 1) / TILE_UNIT;
  p.tile = TILE_UNIT * ((units + MAX_TILES - 1) / MAX_TILES);
  p.tiles = (n + p.tile - 1) / p.tile;
  int bits = 1;
  while (bits < 32 && ((uint32_t)vocab >> bits) != 0u) ++bits;      // keys 0 .. vocab (vocab: outside the table)
  p.passes = (bits + 7) / 8;
  p.bits = (bits + p.passes - 1) / p.passes;
  // Chunks of 32 sorted tokens keep the launch wide; longer ones for large batches keep the partial sums few.
  p.chunk = 32;
  while (p.chunk < 1024 && (n + p.chunk - 1) / p.chunk > 2048) p.chunk *= 2;
  p.chunks = (n + p.chunk - 1) / p.chunk;
  return p;
}

struct EmbedScratch {
  uint32_t* counts;                    // [passes][tiles][DIGITS]
  uint8_t* touched;                    // [vocab]
  uint2* a; uint2* b;                  // (id, token) before and after a pass
  float* partial;                      // [chunks][2][d]: first run's part, last run's part
  size_t count_words;
};

void carve(FaxArena& ar, const SortPlan& p, int vocab, int d, EmbedScratch* s) {
  s->count_words = (size_t)p.passes * p.tiles * DIGITS;
  s->counts = (uint32_t*)ar.take(s->count_words * 4);
  s->touched = (uint8_t*)ar.take(fax_round_up((size_t)vocab, 16));
  s->a = (uint2*)ar.take((size_t)p.n * sizeof(uint2));
  s->b = (uint2*)ar.take((size_t)p.n * sizeof(uint2));
  s->partial = (float*)ar.take((size_t)p.chunks * 2 * d * sizeof(float));
}

__device__ __forceinline__ uint32_t key_of(int32_t id, int vocab) { return (id < 0 || id >= vocab) ? (uint32_t)vocab : (uint32_t)id; }

// ---- forward: a warp takes 32 * U vectors of one row ----
template <typename T, int V> struct Vec;
template <> struct Vec<bf16, 8> { typedef uint4 type; };
template <> struct Vec<bf16, 1> { typedef bf16 type; };
template <> struct Vec<float, 4> { typedef float4 type; };
template <> struct Vec<float, 1> { typedef float type; };

template <typename T, int V>
__device__ __forceinline__ void widen(const typename Vec<T, V>::type& x, float (&f)[V]) {
  const T* e = reinterpret_cast<const T*>(&x);
#pragma unroll
  for (int j = 0; j < V; ++j) f[j] = to_f32(e[j]);
}

template <typename T, int V>
__global__ void __launch_bounds__(256)
embed_lookup_kernel(int n, int vocab, int nvec, int parts, const int32_t* __restrict__ ids, const T* __restrict__ table,
                    float scale, T* __restrict__ out) {
  typedef typename Vec<T, V>::type vec;
  constexpr int U = 4;
  fax_grid_dependency_wait();
  const long long item = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  const long long row = item / parts;
  const int c0 = (int)(item - row * parts) * (32 * U) + lane;
  if (row >= n) return;
  const int id = ids[row];
  const bool in = id >= 0 && id < vocab;
  const vec* src = reinterpret_cast<const vec*>(table) + (size_t)(in ? id : 0) * nvec;
  vec* dst = reinterpret_cast<vec*>(out) + (size_t)row * nvec;
  vec x[U];
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (in && c0 + 32 * u < nvec) x[u] = src[c0 + 32 * u];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = c0 + 32 * u;
    if (c >= nvec) continue;
    vec y;
    T* ye = reinterpret_cast<T*>(&y);
    float f[V];
    if (in) widen<T, V>(x[u], f);
#pragma unroll
    for (int j = 0; j < V; ++j) ye[j] = from_f32<T>(in ? scale * f[j] : 0.f);
    dst[c] = y;
  }
}

// ---- sort ----
__global__ void __launch_bounds__(SORT_THREADS)
embed_sort_count_kernel(SortPlan p, int vocab, const int32_t* __restrict__ ids, uint32_t* __restrict__ counts,
                        unsigned long long later_words, uint4* __restrict__ touched, unsigned long long touched_vecs) {
  __shared__ uint32_t hist[DIGITS];
  for (int i = threadIdx.x; i < DIGITS; i += SORT_THREADS) hist[i] = 0u;
  __syncthreads();
  fax_grid_dependency_wait();
  const unsigned long long tid = (unsigned long long)blockIdx.x * SORT_THREADS + threadIdx.x, step = (unsigned long long)gridDim.x * SORT_THREADS;
  uint32_t* later = counts + (size_t)p.tiles * DIGITS;              // the counts of the passes after the first
  for (unsigned long long i = tid; i < later_words; i += step) later[i] = 0u;
  for (unsigned long long i = tid; i < touched_vecs; i += step) touched[i] = make_uint4(0u, 0u, 0u, 0u);
  for (int t = blockIdx.x; t < p.tiles; t += gridDim.x) {
    const int lo = t * p.tile, hi = min(p.n, lo + p.tile);
    for (int i = lo + threadIdx.x; i < hi; i += SORT_THREADS)
      atomicAdd(&hist[key_of(ids[i], vocab) & ((1u << p.bits) - 1u)], 1u);
    __syncthreads();
    for (int i = threadIdx.x; i < DIGITS; i += SORT_THREADS) { counts[(size_t)t * DIGITS + i] = hist[i]; hist[i] = 0u; }
    __syncthreads();
  }
}

// One tile per block.  FIRST: the tokens are read from ids, and the table rows they touch are marked.
template <bool FIRST>
__global__ void __launch_bounds__(SORT_THREADS)
embed_sort_scatter_kernel(SortPlan p, int pass, int vocab, const int32_t* __restrict__ ids, const uint2* __restrict__ in,
                          uint2* __restrict__ out, uint32_t* __restrict__ counts, uint8_t* __restrict__ touched) {
  __shared__ uint32_t before[2][DIGITS], total[2][DIGITS];          // two halves of the tiles
  __shared__ uint32_t warp_total[8];
  __shared__ uint32_t off[SORT_WARPS][DIGITS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < SORT_WARPS * DIGITS; i += SORT_THREADS) (&off[0][0])[i] = 0u;
  fax_grid_dependency_wait();
  const int t = blockIdx.x;
  const int shift = pass * p.bits;
  const uint32_t mask = (1u << p.bits) - 1u;
  const int lo = t * p.tile, hi = min(p.n, lo + p.tile);
  const int per_warp = p.tile / SORT_WARPS;                          // a multiple of 32
  const int w_lo = lo + warp * per_warp, w_hi = min(hi, w_lo + per_warp);

  // counts of the tiles before this one, and of all tiles, by digit
  {
    const uint32_t* c = counts + (size_t)pass * p.tiles * DIGITS;
    const int dgt = threadIdx.x & (DIGITS - 1), half = threadIdx.x >> 8;
    const int mid = (p.tiles + 1) / 2, t0 = half ? mid : 0, t1 = half ? p.tiles : mid;
    uint32_t b = 0u, all = 0u;
#pragma unroll 8
    for (int i = t0; i < t1; ++i) {
      const uint32_t x = c[(size_t)i * DIGITS + dgt];
      b += i < t ? x : 0u;
      all += x;
    }
    before[half][dgt] = b;
    total[half][dgt] = all;
  }
  __syncthreads();
  // this tile's digits, by warp
  auto load = [&](int i) { return FIRST ? make_uint2(key_of(ids[i], vocab), (uint32_t)i) : in[i]; };
  for (int i = w_lo + lane; i < w_hi; i += 32) atomicAdd(&off[warp][(load(i).x >> shift) & mask], 1u);
  // exclusive sum of all tiles' totals over the digits
  uint32_t x = 0u, incl = 0u;
  if (threadIdx.x < DIGITS) {
    x = total[0][threadIdx.x] + total[1][threadIdx.x];
    incl = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    if (lane == 31) warp_total[warp] = incl;
  }
  __syncthreads();
  if (threadIdx.x < DIGITS) {
    uint32_t add = 0u;
    for (int w = 0; w < warp; ++w) add += warp_total[w];
    uint32_t at = add + incl - x + before[0][threadIdx.x] + before[1][threadIdx.x];
    for (int w = 0; w < SORT_WARPS; ++w) {                           // where each warp's tokens of this digit begin
      const uint32_t c = off[w][threadIdx.x];
      off[w][threadIdx.x] = at;
      at += c;
    }
  }
  __syncthreads();
  const bool more = pass + 1 < p.passes;
  uint32_t* next = counts + (size_t)(pass + 1) * p.tiles * DIGITS;
  for (int i0 = w_lo; i0 < w_hi; i0 += 32) {
    const int i = i0 + lane;
    const bool live = i < w_hi;
    const uint2 kv = live ? load(i) : make_uint2(0u, 0u);
    const uint32_t dgt = live ? ((kv.x >> shift) & mask) : DIGITS;   // lanes past the end match only each other
    const uint32_t same = __match_any_sync(0xffffffffu, dgt);
    const uint32_t rank = __popc(same & ((1u << lane) - 1u));
    const uint32_t at = live ? off[warp][dgt] + rank : 0u;
    __syncwarp();
    if (live && rank == 0u) off[warp][dgt] += __popc(same);
    __syncwarp();
    if (live) {
      out[at] = kv;
      if (more) atomicAdd(next + (size_t)(at / (uint32_t)p.tile) * DIGITS + ((kv.x >> (shift + p.bits)) & mask), 1u);
      if (FIRST && kv.x < (uint32_t)vocab) touched[kv.x] = 1;
    }
  }
}

// ---- gradient ----
// LG lanes (a power of two up to GRAD_THREADS) work on one chunk and one slice of LG * V columns.
template <typename T, int V>
__global__ void __launch_bounds__(GRAD_THREADS)
embed_grad_kernel(SortPlan p, int vocab, int d, int nvec, int lanes, int slices, unsigned int grad_blocks, const uint2* __restrict__ sorted,
                  const T* __restrict__ dout, float scale, int accumulate, float* __restrict__ dtable,
                  float* __restrict__ partial, const uint8_t* __restrict__ touched) {
  typedef typename Vec<T, V>::type vec;
  fax_grid_dependency_wait();
  if (blockIdx.x >= grad_blocks) {
    // rows that no token touches: a warp per row
    const unsigned int zb = blockIdx.x - grad_blocks, zblocks = gridDim.x - grad_blocks;
    const int lane = threadIdx.x & 31;
    for (long long v = (long long)zb * (GRAD_THREADS / 32) + (threadIdx.x >> 5); v < vocab; v += (long long)zblocks * (GRAD_THREADS / 32)) {
      if (touched[v]) continue;
      float* row = dtable + (size_t)v * d;
      if (V > 1) for (int c = lane; c < d / 4; c += 32) reinterpret_cast<float4*>(row)[c] = make_float4(0.f, 0.f, 0.f, 0.f);
      else for (int c = lane; c < d; c += 32) row[c] = 0.f;
    }
    return;
  }
  const int groups = GRAD_THREADS / lanes;
  const long long item = (long long)blockIdx.x * groups + threadIdx.x / lanes;
  const int chunk = (int)(item / slices), slice = (int)(item - (long long)chunk * slices);
  const int c = slice * lanes + (threadIdx.x & (lanes - 1));
  if (chunk >= p.chunks || c >= nvec) return;
  const int lo = chunk * p.chunk, hi = min(p.n, lo + p.chunk);
  const uint32_t prev = lo > 0 ? sorted[lo - 1].x : 0xffffffffu, after = hi < p.n ? sorted[hi].x : 0xffffffffu;
  const vec* src = reinterpret_cast<const vec*>(dout);
  float acc[V];
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] = 0.f;
  auto flush = [&](uint32_t key, bool first_run, bool last_run) {
    if (key >= (uint32_t)vocab) return;
    const bool from_before = first_run && prev == key, goes_on = last_run && after == key;
    if (from_before || goes_on) {
      // a run that crosses an edge: partial sums, slot 0 where it came from before, else slot 1
      float* o = partial + ((size_t)chunk * 2 + (from_before ? 0 : 1)) * d + (size_t)c * V;
#pragma unroll
      for (int j = 0; j < V; ++j) o[j] = acc[j];
    } else {
      float* o = dtable + (size_t)key * d + (size_t)c * V;
#pragma unroll
      for (int j = 0; j < V; j += (V > 1 ? 4 : 1)) {
        if (V > 1) {
          float4 y = make_float4(scale * acc[j], scale * acc[j + 1], scale * acc[j + 2], scale * acc[j + 3]);
          if (accumulate) {
            const float4 z = *reinterpret_cast<const float4*>(o + j);
            y.x += z.x; y.y += z.y; y.z += z.z; y.w += z.w;
          }
          *reinterpret_cast<float4*>(o + j) = y;
        } else {
          o[j] = accumulate ? o[j] + scale * acc[j] : scale * acc[j];
        }
      }
    }
  };
  constexpr int U = 4;
  uint32_t cur = sorted[lo].x;
  bool first_run = true;
  for (int i0 = lo; i0 < hi; i0 += U) {
    uint2 kv[U];
    vec x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) kv[u] = i0 + u < hi ? sorted[i0 + u] : make_uint2((uint32_t)vocab, 0u);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (kv[u].x < (uint32_t)vocab) x[u] = src[(size_t)kv[u].y * nvec + c];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u >= hi) break;
      if (kv[u].x != cur) {
        flush(cur, first_run, false);
        first_run = false;
        cur = kv[u].x;
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = 0.f;
      }
      if (cur < (uint32_t)vocab) {
        float f[V];
        widen<T, V>(x[u], f);
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += f[j];
      }
    }
  }
  flush(cur, first_run, true);
}

// The runs that crossed a chunk's edge: block (chunk, slice of 32 columns); nothing to do unless a run begins
// in this chunk and goes on.  JOIN_GROUPS warps take the following chunks in turn; their sums are added in order.
__global__ void __launch_bounds__(32 * JOIN_GROUPS)
embed_join_kernel(SortPlan p, int vocab, int d, int slices, const uint2* __restrict__ sorted, const float* __restrict__ partial, float scale,
                  int accumulate, float* __restrict__ dtable) {
  __shared__ float part[JOIN_GROUPS][32];
  fax_grid_dependency_wait();
  const int chunk = blockIdx.x / slices, slice = blockIdx.x - chunk * slices;
  const int lo = chunk * p.chunk, hi = lo + p.chunk;
  if (hi >= p.n) return;                                             // the last chunk: nothing follows
  const uint32_t key = sorted[hi - 1].x;
  if (key >= (uint32_t)vocab || sorted[hi].x != key) return;         // its last run ends here
  if (lo > 0 && sorted[lo - 1].x == key && sorted[lo].x == key) return;   // the run began before this chunk
  // the run's last chunk: chunks after this one whose first token still has the key (binary search, sorted)
  int a = chunk + 1, b = p.chunks - 1;
  while (a < b) {
    const int m = (a + b + 1) >> 1;
    if (sorted[(size_t)m * p.chunk].x == key) a = m; else b = m - 1;
  }
  const int last = a;
  const int col = slice * 32 + (threadIdx.x & 31), grp = threadIdx.x >> 5;
  const int count = last - chunk, per = (count + JOIN_GROUPS - 1) / JOIN_GROUPS;
  const int c0 = chunk + 1 + grp * per, c1 = min(last + 1, c0 + per);
  float s = 0.f;
  if (col < d) {
#pragma unroll 8
    for (int c = c0; c < c1; ++c) s += partial[(size_t)c * 2 * d + col];
  }
  part[grp][threadIdx.x & 31] = s;
  __syncthreads();
  if (grp == 0 && col < d) {
    float t = partial[((size_t)chunk * 2 + 1) * d + col];
#pragma unroll
    for (int w = 0; w < JOIN_GROUPS; ++w) t += part[w][threadIdx.x];
    float* o = dtable + (size_t)key * d + col;
    *o = accumulate ? *o + scale * t : scale * t;
  }
}

template <typename T, int V>
fax_status launch_grad(fax_ctx* ctx, const SortPlan& p, int vocab, int d, const uint2* sorted, const void* dout, float scale,
                       int accumulate, float* dtable, const EmbedScratch& s) {
  const int nvec = d / V;
  int lanes = 1;
  while (lanes < nvec && lanes < GRAD_THREADS) lanes *= 2;
  const int slices = (nvec + lanes - 1) / lanes, groups = GRAD_THREADS / lanes;
  const long long items = (long long)p.chunks * slices, gb = (items + groups - 1) / groups;
  long long zb = 0;
  if (!accumulate) {
    zb = ((long long)vocab + GRAD_THREADS / 32 - 1) / (GRAD_THREADS / 32);
    if (zb > (long long)ctx->sm_count * 16) zb = (long long)ctx->sm_count * 16;
  }
  if (gb + zb > 0x7fffffffLL) return FAX_ERR_UNSUPPORTED_SHAPE;
  fax_launch(ctx, embed_grad_kernel<T, V>, dim3((unsigned int)(gb + zb)), dim3(GRAD_THREADS), 0, p, vocab, d, nvec, lanes, slices,
             (unsigned int)gb, sorted, (const T*)dout, scale, accumulate, dtable, s.partial, (const uint8_t*)s.touched);
  return fax_after_launch(ctx);
}

template <typename T, int V>
fax_status launch_lookup(fax_ctx* ctx, int n, int vocab, int d, const int32_t* ids, const void* table, float scale, void* out) {
  const int nvec = d / V, parts = (nvec + 127) / 128;
  const long long blocks = ((long long)n * parts + 7) / 8;
  if (blocks > 0x7fffffffLL) return FAX_ERR_UNSUPPORTED_SHAPE;
  fax_launch(ctx, embed_lookup_kernel<T, V>, dim3((unsigned int)blocks), dim3(256), 0, n, vocab, nvec, parts, ids, (const T*)table, scale, (T*)out);
  return fax_after_launch(ctx);
}

fax_status embed_args(int32_t prec, int32_t n, int32_t vocab, int32_t d) {
  if (prec != FAX_PREC_BF16 && prec != FAX_PREC_FP32_VALIDATE) return FAX_ERR_INVALID_ARG;
  if (n < 0 || vocab <= 0 || d <= 0) return FAX_ERR_INVALID_ARG;
  if (n > MAX_TOKENS) return FAX_ERR_UNSUPPORTED_SHAPE;
  return FAX_OK;
}

}  // namespace

fax_status fax_embedding_lookup(fax_ctx* ctx, int prec, int n, int vocab, int d, const int32_t* ids, const void* table, float scale, void* out) {
  FaxProfScope prof(ctx, KC_EMBED, 0.0, 2.0 * n * (double)d * fax_elem_size(prec));
  const bool wide = fax_aligned(table, 16) && fax_aligned(out, 16);
  if (prec == FAX_PREC_BF16)
    return wide && d % 8 == 0 ? launch_lookup<bf16, 8>(ctx, n, vocab, d, ids, table, scale, out) : launch_lookup<bf16, 1>(ctx, n, vocab, d, ids, table, scale, out);
  return wide && d % 4 == 0 ? launch_lookup<float, 4>(ctx, n, vocab, d, ids, table, scale, out) : launch_lookup<float, 1>(ctx, n, vocab, d, ids, table, scale, out);
}

size_t fax_embedding_grad_scratch_bytes(int n, int vocab, int d) {
  FaxArena ar(nullptr, 0);
  EmbedScratch s;
  carve(ar, plan_for(n > 0 ? n : 1, vocab), vocab, d, &s);
  return ar.used();
}

fax_status fax_embedding_grad(fax_ctx* ctx, int prec, int n, int vocab, int d, const int32_t* ids, const void* dout, float scale,
                              bool accumulate, float* dtable, void* scratch, size_t scratch_bytes) {
  if (scratch_bytes < fax_embedding_grad_scratch_bytes(n, vocab, d)) return FAX_ERR_WORKSPACE_TOO_SMALL;
  if (n == 0) {
    if (!accumulate) FAX_CUDA_TRY(ctx, cudaMemsetAsync(dtable, 0, (size_t)vocab * d * sizeof(float), ctx->stream));
    return FAX_OK;
  }
  FaxProfScope prof(ctx, KC_EMBED, 0.0, (double)n * d * fax_elem_size(prec) + (accumulate ? 0.0 : 4.0 * vocab * (double)d));
  const SortPlan p = plan_for(n, vocab);
  FaxArena ar(scratch, scratch_bytes);
  EmbedScratch s;
  carve(ar, p, vocab, d, &s);
  const unsigned long long later = s.count_words - (size_t)p.tiles * DIGITS, tv = fax_round_up((size_t)vocab, 16) / 16;
  fax_launch(ctx, embed_sort_count_kernel, dim3(p.tiles > ctx->sm_count ? p.tiles : ctx->sm_count), dim3(SORT_THREADS), 0, p, vocab, ids, s.counts, later,
             (uint4*)s.touched, tv);
  FAX_TRY(fax_after_launch(ctx));
  for (int pass = 0; pass < p.passes; ++pass) {
    uint2* out = (pass & 1) ? s.b : s.a;
    const uint2* in = (pass & 1) ? s.a : s.b;
    if (pass == 0)
      fax_launch(ctx, embed_sort_scatter_kernel<true>, dim3(p.tiles), dim3(SORT_THREADS), 0, p, pass, vocab, ids, in, out, s.counts, s.touched);
    else
      fax_launch(ctx, embed_sort_scatter_kernel<false>, dim3(p.tiles), dim3(SORT_THREADS), 0, p, pass, vocab, ids, in, out, s.counts, s.touched);
    FAX_TRY(fax_after_launch(ctx));
  }
  const uint2* sorted = ((p.passes - 1) & 1) ? s.b : s.a;
  const bool wide = fax_aligned(dout, 16) && fax_aligned(dtable, 16);
  const int acc = accumulate ? 1 : 0;
  if (prec == FAX_PREC_BF16)
    FAX_TRY((wide && d % 8 == 0 ? launch_grad<bf16, 8>(ctx, p, vocab, d, sorted, dout, scale, acc, dtable, s)
                                : launch_grad<bf16, 1>(ctx, p, vocab, d, sorted, dout, scale, acc, dtable, s)));
  else
    FAX_TRY((wide && d % 4 == 0 ? launch_grad<float, 4>(ctx, p, vocab, d, sorted, dout, scale, acc, dtable, s)
                                : launch_grad<float, 1>(ctx, p, vocab, d, sorted, dout, scale, acc, dtable, s)));
  if (p.chunks > 1) {
    const int slices = (d + 31) / 32;
    if ((long long)p.chunks * slices > 0x7fffffffLL) return FAX_ERR_UNSUPPORTED_SHAPE;
    fax_launch(ctx, embed_join_kernel, dim3((unsigned int)((long long)p.chunks * slices)), dim3(32 * JOIN_GROUPS), 0, p, vocab, d, slices, sorted,
               (const float*)s.partial, scale, acc, dtable);
    FAX_TRY(fax_after_launch(ctx));
  }
  return FAX_OK;
}

extern "C" fax_status fax_op_embedding_forward(fax_ctx* ctx, int32_t prec, int32_t n_tokens, int32_t vocab, int32_t d, const int32_t* ids,
                                               const void* table, float scale, void* out) {
  if (!ctx) return FAX_ERR_INVALID_ARG;
  FAX_TRY(embed_args(prec, n_tokens, vocab, d));
  if (n_tokens == 0) return FAX_OK;
  if (!ids || !table || !out) return FAX_ERR_INVALID_ARG;
  if (!fax_aligned(ids, 4) || !fax_aligned(table, fax_elem_size(prec)) || !fax_aligned(out, fax_elem_size(prec))) return FAX_ERR_INVALID_ARG;
  return fax_embedding_lookup(ctx, prec, n_tokens, vocab, d, ids, table, scale, out);
}

extern "C" fax_status fax_op_embedding_backward_scratch_bytes(int32_t n_tokens, int32_t vocab, int32_t d, size_t* bytes) {
  if (!bytes) return FAX_ERR_INVALID_ARG;
  FAX_TRY(embed_args(FAX_PREC_BF16, n_tokens, vocab, d));
  *bytes = fax_embedding_grad_scratch_bytes(n_tokens, vocab, d);
  return FAX_OK;
}

extern "C" fax_status fax_op_embedding_backward(fax_ctx* ctx, int32_t prec, int32_t n_tokens, int32_t vocab, int32_t d, const int32_t* ids,
                                                const void* dout, float scale, int32_t accumulate, float* dtable, void* scratch,
                                                size_t scratch_bytes) {
  if (!ctx || !dtable || !scratch) return FAX_ERR_INVALID_ARG;
  FAX_TRY(embed_args(prec, n_tokens, vocab, d));
  if (n_tokens > 0 && (!ids || !dout)) return FAX_ERR_INVALID_ARG;
  if (!fax_aligned(ids, 4) || !fax_aligned(dout, fax_elem_size(prec)) || !fax_aligned(dtable, 4) || !fax_aligned(scratch, 256)) return FAX_ERR_INVALID_ARG;
  return fax_embedding_grad(ctx, prec, n_tokens, vocab, d, ids, dout, scale, accumulate != 0, dtable, scratch, scratch_bytes);
}
