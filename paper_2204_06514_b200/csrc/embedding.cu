// Token table lookup with scaling, and its gradient by sorted tokens.
//
//   forward   out[i] = scale * table[ids[i]]                     (a zero row where ids[i] is outside the table)
//   backward  dtable[v] (+)= scale * sum_{i : ids[i] = v} dout[i]
//
// The gradient's sums run over tokens grouped by id, in the order in which the tokens stand: every row of
// the table is written once, nothing is added by float atomics, and the same call gives the same bits.
//
// Small batches (DIRECT_TOKENS) need no sort: a block per token looks through all ids; the first token of its id
// sums the rows of those that are alike.  One launch instead of five, bound by its latency; back to back, accumulated:
// 64 tokens x 256 7.6 us against 15-20 by the sort, 256 x 768 6.4 against 16.  512 tokens of one id x 1,024 (the
// longest list, bf16): 9.4 against 13.2; at 1,024 tokens of one id the sort is ahead (13.2 against 15.9), and so it is
// from about 2,000 blocks (1,000 different ids x 1,024: 16.8 against 18.4), whence the two limits.
//
// Larger ones:
//
//  1. A least-significant-digit radix sort of the ids (8 bits a pass at most, as many passes as the
//     vocabulary needs: two for 50,304 ids).  embed_sort_count zeroes the counters and counts the first
//     digit per tile of tokens; embed_sort_scatter places a tile's tokens behind those of the tiles before
//     it, keeping their order (rank within a warp by match, then warps, then tiles), and counts the next
//     digit of the tile each token lands in (whole-number atomics: the sums do not depend on their order).
//  2. embed_grad: chunks of consecutive sorted tokens.  A run of equal ids inside a chunk is summed in
//     registers and written; a run that crosses a chunk's edge leaves partial sums (at most a first and
//     a last one per chunk), and the chunk it begins in is listed.
//  3. embed_join: adds the partial sums of each listed run in chunk order.
// A row that is accumulated gets its sum by one reduction at L2 (nothing waits for the old value; one addition per
// element and call, so the order is still fixed).
//
// An overwritten table has to be zeroed where no token touches it, most of the bytes of a small batch.
// Where the rows that can be touched are few, further blocks of the sort's launches zero the whole table
// meanwhile (the sort is latency, the zeros are bandwidth; touched rows are written twice); where they are
// many, the sort marks them and further blocks of embed_grad zero the others.
#include "common.cuh"

namespace {

constexpr int SORT_THREADS = 512;
constexpr int SORT_WARPS = SORT_THREADS / 32;
constexpr int DIGITS = 256;
constexpr int TILE_UNIT = 512;         // tokens per tile: a multiple of this
constexpr int MAX_TILES = 256;         // a scatter block reads every tile's counts of its pass
constexpr int MAX_TOKENS = 1 << 30;    // token and tile positions stay within 32 bits
constexpr int MAX_WIDTH = 1 << 30;     // so do columns
constexpr int GRAD_THREADS = 128;
constexpr int DIRECT_THREADS = 512;
constexpr int DIRECT_TOKENS = DIRECT_THREADS;   // one id a thread
constexpr int DIRECT_BLOCKS = 1024;    // tokens times slices of columns: each block looks through all ids
constexpr int DIRECT_LANES = 64;       // of a group: the other groups share a long list
constexpr int DIRECT_ROWS = 32;        // table rows that a zeroing block looks up at a time
constexpr int JOIN_WARPS = 8;
constexpr int JOIN_SHORT = 8;          // a run over at most this many further chunks is joined by one warp per 128 columns
// Rows of a batch that may be written twice for the zeros to run under the sort: at HBM rate about what the sort takes.
constexpr double PREFILL_BYTES = 64e6;

struct SortPlan {
  int n, tile, tiles, passes, bits;    // bits per pass
  int chunk, chunks;                   // sorted tokens per gradient chunk
};
// Chunks of 16 sorted tokens keep the launch wide; longer ones for large batches keep the partial sums few.
constexpr int CHUNK_LEAST = 16, CHUNK_MOST = 1024, CHUNKS = 1024;    // longer chunks are taken from CHUNKS of them on

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
  p.chunk = CHUNK_LEAST;
  while (p.chunk < CHUNK_MOST && (n + p.chunk - 1) / p.chunk > CHUNKS) p.chunk *= 2;
  p.chunks = (n + p.chunk - 1) / p.chunk;
  return p;
}

// Tiles and chunks that no batch of up to n tokens exceeds: a longer tile or chunk makes fewer of them, and scratch sized
// for a batch has to serve every shorter one.
SortPlan most_for(int n, int vocab) {
  SortPlan p = plan_for(n, vocab);
  const int units = (n + TILE_UNIT - 1) / TILE_UNIT, least = (n + CHUNK_LEAST - 1) / CHUNK_LEAST;
  p.tiles = units < MAX_TILES ? units : MAX_TILES;
  const int at_least = least < CHUNKS ? least : CHUNKS;
  if (p.chunks < at_least) p.chunks = at_least;
  return p;
}

struct EmbedScratch {
  uint32_t* counts;                    // [passes][tiles][DIGITS], then the lengths of the two lists
  uint2* lists;                        // [2][chunks]: (chunk, id) of the short / long runs that begin in a chunk and go on
  uint8_t* touched;                    // [vocab]
  uint2* a; uint2* b;                  // (id, token) before and after a pass
  float* partial;                      // [chunks][2][d]: first run's part, last run's part
  size_t count_words;
};

void carve(FaxArena& ar, const SortPlan& p, int vocab, int d, EmbedScratch* s) {
  s->count_words = (size_t)p.passes * p.tiles * DIGITS + 4;
  s->counts = (uint32_t*)ar.take(s->count_words * 4);
  s->lists = (uint2*)ar.take((size_t)p.chunks * 2 * sizeof(uint2));
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
// This launch's share of zeroing the table, done by the blocks behind the sort's.
struct Fill { float4* p; unsigned long long lo, hi; };               // vectors [lo, hi)
__device__ __forceinline__ void fill_zero(const Fill& f, unsigned int first_block) {
  const unsigned long long step = (unsigned long long)(gridDim.x - first_block) * SORT_THREADS;
  for (unsigned long long i = f.lo + (unsigned long long)(blockIdx.x - first_block) * SORT_THREADS + threadIdx.x; i < f.hi; i += step)
    f.p[i] = make_float4(0.f, 0.f, 0.f, 0.f);
}

__global__ void __launch_bounds__(SORT_THREADS)
embed_sort_count_kernel(SortPlan p, int vocab, const int32_t* __restrict__ ids, uint32_t* __restrict__ counts,
                        unsigned long long later_words, uint4* __restrict__ touched, unsigned long long touched_vecs, Fill fill) {
  __shared__ uint32_t hist[DIGITS];
  for (int i = threadIdx.x; i < DIGITS; i += SORT_THREADS) hist[i] = 0u;
  __syncthreads();
  fax_grid_dependency_wait();
  if (blockIdx.x >= p.tiles) { fill_zero(fill, p.tiles); return; }
  const unsigned long long tid = (unsigned long long)blockIdx.x * SORT_THREADS + threadIdx.x, step = (unsigned long long)p.tiles * SORT_THREADS;
  uint32_t* later = counts + (size_t)p.tiles * DIGITS;              // the counts of the passes after the first, and the lists' lengths
  for (unsigned long long i = tid; i < later_words; i += step) later[i] = 0u;
  for (unsigned long long i = tid; i < touched_vecs; i += step) touched[i] = make_uint4(0u, 0u, 0u, 0u);
  const int lo = blockIdx.x * p.tile, hi = min(p.n, lo + p.tile);
  for (int i = lo + threadIdx.x; i < hi; i += SORT_THREADS)
    atomicAdd(&hist[key_of(ids[i], vocab) & ((1u << p.bits) - 1u)], 1u);
  __syncthreads();
  for (int i = threadIdx.x; i < DIGITS; i += SORT_THREADS) counts[(size_t)blockIdx.x * DIGITS + i] = hist[i];
}

// One tile per block.  FIRST: the tokens are read from ids, and the table rows they touch are marked (touched not null).
template <bool FIRST>
__global__ void __launch_bounds__(SORT_THREADS)
embed_sort_scatter_kernel(SortPlan p, int pass, int vocab, const int32_t* __restrict__ ids, const uint2* __restrict__ in,
                          uint2* __restrict__ out, uint32_t* __restrict__ counts, uint8_t* __restrict__ touched, Fill fill) {
  constexpr int QUADS = DIGITS / 4, TILE_GROUPS = SORT_THREADS / QUADS;    // a thread reads four digits of every eighth tile
  __shared__ uint4 before[TILE_GROUPS][QUADS], total[TILE_GROUPS][QUADS];
  __shared__ uint32_t warp_total[8];
  __shared__ uint32_t off[SORT_WARPS][DIGITS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < SORT_WARPS * DIGITS; i += SORT_THREADS) (&off[0][0])[i] = 0u;
  fax_grid_dependency_wait();
  if (blockIdx.x >= p.tiles) { fill_zero(fill, p.tiles); return; }
  const int t = blockIdx.x;
  const int shift = pass * p.bits;
  const uint32_t mask = (1u << p.bits) - 1u;
  const int lo = t * p.tile, hi = min(p.n, lo + p.tile);
  const int per_warp = p.tile / SORT_WARPS;                          // a multiple of 32
  const int w_lo = lo + warp * per_warp, w_hi = min(hi, w_lo + per_warp);

  auto load = [&](int i) { return FIRST ? make_uint2(key_of(ids[i], vocab), (uint32_t)i) : in[i]; };
  const uint2 early = w_lo + lane < w_hi ? load(w_lo + lane) : make_uint2(0u, 0u);      // in flight while the counts are read

  // counts of the tiles before this one, and of all tiles, by digit
  {
    const uint4* c = reinterpret_cast<const uint4*>(counts + (size_t)pass * p.tiles * DIGITS);
    const int quad = threadIdx.x % QUADS, grp = threadIdx.x / QUADS;
    uint4 b = make_uint4(0u, 0u, 0u, 0u), all = b;
#pragma unroll 8
    for (int i = grp; i < p.tiles; i += TILE_GROUPS) {
      const uint4 x = c[(size_t)i * QUADS + quad];
      all.x += x.x; all.y += x.y; all.z += x.z; all.w += x.w;
      if (i < t) { b.x += x.x; b.y += x.y; b.z += x.z; b.w += x.w; }
    }
    before[grp][quad] = b;
    total[grp][quad] = all;
  }
  __syncthreads();
  // this tile's digits, by warp
  for (int i = w_lo + lane; i < w_hi; i += 32) atomicAdd(&off[warp][((i < w_lo + 32 ? early : load(i)).x >> shift) & mask], 1u);
  // exclusive sum of all tiles' totals over the digits
  uint32_t x = 0u, mine = 0u, incl = 0u;
  if (threadIdx.x < DIGITS) {
#pragma unroll
    for (int g = 0; g < TILE_GROUPS; ++g) {
      x += reinterpret_cast<const uint32_t*>(total[g])[threadIdx.x];
      mine += reinterpret_cast<const uint32_t*>(before[g])[threadIdx.x];
    }
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
    uint32_t at = incl - x + mine;
    for (int w = 0; w < warp; ++w) at += warp_total[w];
#pragma unroll
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
    const uint2 kv = i0 == w_lo ? early : (live ? load(i) : make_uint2(0u, 0u));
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
      if (FIRST && touched != nullptr && kv.x < (uint32_t)vocab) touched[kv.x] = 1;
    }
  }
}

// ---- gradient ----
// Four sums of a table row: stored, or added to it by one vector reduction (16-byte aligned).
__device__ __forceinline__ void put4(float* o, float a, float b, float c, float d, int accumulate) {
  if (accumulate) asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(o), "f"(a), "f"(b), "f"(c), "f"(d) : "memory");
  else *reinterpret_cast<float4*>(o) = make_float4(a, b, c, d);
}

// Small batches: blocks (token, slice of lanes * V columns), then blocks that zero the rows no token touches.
template <typename T, int V>
__global__ void __launch_bounds__(DIRECT_THREADS)
embed_direct_kernel(int n, int vocab, int d, int nvec, int lanes, int slices, unsigned int work_blocks, const int32_t* __restrict__ ids,
                    const T* __restrict__ dout, float scale, int accumulate, float* __restrict__ dtable) {
  typedef typename Vec<T, V>::type vec;
  constexpr int WARPS = DIRECT_THREADS / 32;
  __shared__ uint32_t list[DIRECT_TOKENS];
  __shared__ int counts[WARPS];
  __shared__ int hit[DIRECT_ROWS];
  __shared__ float parts[DIRECT_THREADS * V];
  fax_grid_dependency_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int i = threadIdx.x;                                         // this thread's token
  const uint32_t mine = i < n ? key_of(ids[i], vocab) : (uint32_t)vocab;
  if (blockIdx.x >= work_blocks) {
    for (long long v0 = (long long)(blockIdx.x - work_blocks) * DIRECT_ROWS; v0 < vocab; v0 += (long long)(gridDim.x - work_blocks) * DIRECT_ROWS) {
      if (threadIdx.x < DIRECT_ROWS) hit[threadIdx.x] = 0;
      __syncthreads();
      const long long r0 = (long long)mine - v0;
      if (mine < (uint32_t)vocab && r0 >= 0 && r0 < DIRECT_ROWS) hit[r0] = 1;
      __syncthreads();
      for (int r = warp; r < DIRECT_ROWS && v0 + r < vocab; r += WARPS) {
        if (hit[r]) continue;
        float* row = dtable + (size_t)(v0 + r) * d;
        if (V > 1) for (int c = lane; c < d / 4; c += 32) reinterpret_cast<float4*>(row)[c] = make_float4(0.f, 0.f, 0.f, 0.f);
        else for (int c = lane; c < d; c += 32) row[c] = 0.f;
      }
      __syncthreads();
    }
    return;
  }
  const int token = blockIdx.x / slices, slice = blockIdx.x - token * slices;
  const uint32_t key = key_of(ids[token], vocab);
  if (key >= (uint32_t)vocab) return;                                // the whole block
  const bool match = mine == key;
  if (__syncthreads_or(match && i < token)) return;                  // an earlier token has this id
  // the tokens that are alike, in their order
  const uint32_t alike = __ballot_sync(0xffffffffu, match);
  if (lane == 0) counts[warp] = __popc(alike);
  __syncthreads();
  int at = 0, total = 0;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) {
    at += w < warp ? counts[w] : 0;
    total += counts[w];
  }
  if (match) list[at + __popc(alike & ((1u << lane) - 1u))] = (uint32_t)i;
  __syncthreads();
  // one group of lanes sums a short list; a longer one is cut into equal parts, whose sums are added in order
  const int groups = DIRECT_THREADS / lanes, group = threadIdx.x / lanes, c = slice * lanes + (threadIdx.x & (lanes - 1));
  const int used = total > 8 ? groups : 1, share = (total + used - 1) / used;
  const int r0 = group * share, r1 = group < used ? min(total, r0 + share) : r0;
  float acc[V];
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] = 0.f;
  if (c < nvec) {
    const vec* src = reinterpret_cast<const vec*>(dout) + c;
    constexpr int U = 8;
    for (int q = r0; q < r1; q += U) {
      vec x[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (q + u < r1) x[u] = src[(size_t)list[q + u] * nvec];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (q + u < r1) {
          float f[V];
          widen<T, V>(x[u], f);
#pragma unroll
          for (int j = 0; j < V; ++j) acc[j] += f[j];
        }
    }
  }
  if (used > 1) {
#pragma unroll
    for (int j = 0; j < V; ++j) parts[j * DIRECT_THREADS + threadIdx.x] = acc[j];
    __syncthreads();
    if (group == 0)
      for (int g = 1; g < used; ++g)
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += parts[j * DIRECT_THREADS + g * lanes + threadIdx.x];
  }
  if (group == 0 && c < nvec) {
    float* o = dtable + (size_t)key * d + (size_t)c * V;
    if (V > 1) {
#pragma unroll
      for (int j = 0; j < V; j += 4) put4(o + j, scale * acc[j], scale * acc[j + 1], scale * acc[j + 2], scale * acc[j + 3], accumulate);
    } else {
      if (accumulate) atomicAdd(o, scale * acc[0]); else o[0] = scale * acc[0];
    }
  }
}

// `lanes` lanes (32, 64 or 128) work on one chunk and one slice of lanes * V columns.  A warp holds 32 sorted tokens at a
// time, one a lane; where runs begin is one ballot, and rows are loaded U at a time whatever runs they belong to.
template <typename T, int V>
__global__ void __launch_bounds__(GRAD_THREADS)
embed_grad_kernel(SortPlan p, int vocab, int d, int nvec, int lanes, int slices, unsigned int grad_blocks, const uint2* __restrict__ sorted,
                  const T* __restrict__ dout, float scale, int accumulate, float* __restrict__ dtable,
                  float* __restrict__ partial, const uint8_t* __restrict__ touched, uint32_t* __restrict__ list_len,
                  uint2* __restrict__ lists) {
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
  if (chunk >= p.chunks) return;
  const int lo = chunk * p.chunk, hi = min(p.n, lo + p.chunk);
  const uint32_t prev = lo > 0 ? sorted[lo - 1].x : 0xffffffffu, after = hi < p.n ? sorted[hi].x : 0xffffffffu;
  const bool active = c < nvec;
  const vec* src = reinterpret_cast<const vec*>(dout) + (active ? c : 0);
  float acc[V];
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] = 0.f;
  auto flush = [&](uint32_t key, bool first_run, bool last_run) {
    if (key >= (uint32_t)vocab || !active) return;
    const bool from_before = first_run && prev == key, goes_on = last_run && after == key;
    if (from_before || goes_on) {
      // a run that crosses an edge: partial sums, slot 0 where it came from before, else slot 1
      float* o = partial + ((size_t)chunk * 2 + (from_before ? 0 : 1)) * d + (size_t)c * V;
#pragma unroll
      for (int j = 0; j < V; ++j) o[j] = acc[j];
      if (!from_before && c == 0) {
        const size_t far = (size_t)(chunk + 1 + JOIN_SHORT) * p.chunk;
        const int which = far < (size_t)p.n && sorted[far].x == key ? 1 : 0;
        lists[(size_t)which * p.chunks + atomicAdd(list_len + which, 1u)] = make_uint2((uint32_t)chunk, key);
      }
    } else {
      float* o = dtable + (size_t)key * d + (size_t)c * V;
      if (V > 1) {
#pragma unroll
        for (int j = 0; j < V; j += 4) put4(o + j, scale * acc[j], scale * acc[j + 1], scale * acc[j + 2], scale * acc[j + 3], accumulate);
      } else {
        if (accumulate) atomicAdd(o, scale * acc[0]); else o[0] = scale * acc[0];
      }
    }
  };
  constexpr int U = 4;                                               // rows in flight per lane
  const int lane = threadIdx.x & 31;
  uint32_t cur = sorted[lo].x;
  bool first_run = true;
  for (int base = lo; base < hi; base += 32) {
    const uint2 kv = base + lane < hi ? sorted[base + lane] : make_uint2((uint32_t)vocab, 0u);
    uint32_t before = __shfl_up_sync(0xffffffffu, kv.x, 1);
    if (lane == 0) before = cur;
    const uint32_t heads = __ballot_sync(0xffffffffu, kv.x != before);
    const int live = __popc(__ballot_sync(0xffffffffu, kv.x < (uint32_t)vocab));      // ids outside the table come last
    for (int q = 0; q < live; q += U) {
      vec x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t token = __shfl_sync(0xffffffffu, kv.y, (q + u) & 31);
        if (q + u < live) x[u] = src[(size_t)token * nvec];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (q + u >= live) break;
        if ((heads >> (q + u)) & 1u) {
          flush(cur, first_run, false);
          first_run = false;
          cur = __shfl_sync(0xffffffffu, kv.x, q + u);
#pragma unroll
          for (int j = 0; j < V; ++j) acc[j] = 0.f;
        }
        float f[V];
        widen<T, V>(x[u], f);
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += f[j];
      }
    }
    if (live < 32 && base + live < hi) {                             // what follows is outside the table: the last run ends here
      flush(cur, first_run, false);
      return;
    }
  }
  flush(cur, first_run, true);
}

// The runs that crossed a chunk's edge.  Items: a listed short run and 1024 columns of it (a warp for each 128),
// then a listed long run and 128 columns (the warps take its chunks in equal parts, whose sums are added in order).
template <bool WIDE>
__global__ void __launch_bounds__(32 * JOIN_WARPS)
embed_join_kernel(SortPlan p, int d, const uint2* __restrict__ sorted, const float* __restrict__ partial, const uint32_t* __restrict__ list_len,
                  const uint2* __restrict__ lists, float scale, int accumulate, float* __restrict__ dtable) {
  __shared__ float4 part[JOIN_WARPS][32];
  fax_grid_dependency_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long slices = (d + 127) / 128, groups = (slices + JOIN_WARPS - 1) / JOIN_WARPS;
  const long long n_short = list_len[0] * groups, n_items = n_short + list_len[1] * slices;
  auto load = [&](const float* row, int col) {
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (WIDE) { if (col < d) v = *reinterpret_cast<const float4*>(row + col); }
    else {
      if (col < d) v.x = row[col];
      if (col + 1 < d) v.y = row[col + 1];
      if (col + 2 < d) v.z = row[col + 2];
      if (col + 3 < d) v.w = row[col + 3];
    }
    return v;
  };
  auto add = [](float4& a, const float4& b) { a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w; };
  auto finish = [&](uint32_t key, int col, const float4& t) {
    float* o = dtable + (size_t)key * d + col;
    if (WIDE) {
      if (col < d) put4(o, scale * t.x, scale * t.y, scale * t.z, scale * t.w, accumulate);
    } else {
      const float f[4] = {scale * t.x, scale * t.y, scale * t.z, scale * t.w};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (col + j < d) { if (accumulate) atomicAdd(o + j, f[j]); else o[j] = f[j]; }
    }
  };
  for (long long item = blockIdx.x; item < n_items; item += gridDim.x) {
    const bool is_long = item >= n_short;
    const long long k = is_long ? item - n_short : item, per = is_long ? slices : groups;
    const uint2 run = lists[(is_long ? (size_t)p.chunks : 0) + (size_t)(k / per)];
    const int chunk = (int)run.x;
    const uint32_t key = run.y;
    const int slice = is_long ? (int)(k % per) : (int)(k % per) * JOIN_WARPS + warp;
    const int col = slice < slices ? slice * 128 + 4 * lane : d;
    const float* rest = partial + (size_t)(chunk + 1) * 2 * d;       // slot 0 of the next chunk
    // the run's first part and the one after it, and the chunks after this one that begin with the id, in one go
    const float4 first = load(partial + ((size_t)chunk * 2 + 1) * d, col), second = load(rest, col);
    int count = 0;
    for (int c = chunk + 1;; c += 32) {
      const bool same = c + lane < p.chunks && sorted[(size_t)(c + lane) * p.chunk].x == key;
      const uint32_t m = __ballot_sync(0xffffffffu, same);
      count += __popc(m);
      if (m != 0xffffffffu) break;
    }
    if (!is_long) {
      float4 t = first;
      add(t, second);
#pragma unroll 8
      for (int c = 1; c < count; ++c) add(t, load(rest + (size_t)c * 2 * d, col));
      finish(key, col, t);
    } else {
      const int share = (count + JOIN_WARPS - 1) / JOIN_WARPS, c1 = min(count, (warp + 1) * share);
      float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 16
      for (int c = warp * share; c < c1; ++c) add(t, load(rest + (size_t)c * 2 * d, col));
      part[warp][lane] = t;
      __syncthreads();
      if (warp == 0) {
        float4 u = first;
#pragma unroll
        for (int w = 0; w < JOIN_WARPS; ++w) add(u, part[w][lane]);
        finish(key, col, u);
      }
      __syncthreads();
    }
  }
}

// Lanes of a group and slices of columns: one vector a lane, 32 to `most` lanes.
void lanes_for(int nvec, int most, int* lanes, int* slices) {
  *lanes = 32;
  while (*lanes < nvec && *lanes < most) *lanes *= 2;
  *slices = (nvec + *lanes - 1) / *lanes;
}

template <typename T, int V>
fax_status launch_direct(fax_ctx* ctx, int n, int vocab, int d, int lanes, const int32_t* ids, const void* dout, float scale, int accumulate, float* dtable) {
  const int nvec = d / V, slices = (nvec + lanes - 1) / lanes;
  long long zb = 0;
  if (!accumulate) {
    zb = ((long long)vocab + DIRECT_ROWS - 1) / DIRECT_ROWS;
    if (zb > (long long)ctx->sm_count * 4) zb = (long long)ctx->sm_count * 4;
  }
  fax_launch(ctx, embed_direct_kernel<T, V>, dim3((unsigned int)(n * slices + zb)), dim3(DIRECT_THREADS), 0, n, vocab, d, nvec, lanes, slices,
             (unsigned int)(n * slices), ids, (const T*)dout, scale, accumulate, dtable);
  return fax_after_launch(ctx);
}

template <typename T, int V>
fax_status launch_grad(fax_ctx* ctx, const SortPlan& p, int vocab, int d, const uint2* sorted, const void* dout, float scale,
                       int accumulate, bool fill_here, float* dtable, const EmbedScratch& s) {
  const int nvec = d / V;
  int lanes, slices;
  lanes_for(nvec, GRAD_THREADS, &lanes, &slices);
  const int groups = GRAD_THREADS / lanes;
  const long long items = (long long)p.chunks * slices, gb = (items + groups - 1) / groups;
  long long zb = 0;
  if (fill_here) {
    zb = ((long long)vocab + GRAD_THREADS / 32 - 1) / (GRAD_THREADS / 32);
    if (zb > (long long)ctx->sm_count * 16) zb = (long long)ctx->sm_count * 16;
  }
  if (gb + zb > 0x7fffffffLL) return FAX_ERR_UNSUPPORTED_SHAPE;
  fax_launch(ctx, embed_grad_kernel<T, V>, dim3((unsigned int)(gb + zb)), dim3(GRAD_THREADS), 0, p, vocab, d, nvec, lanes, slices,
             (unsigned int)gb, sorted, (const T*)dout, scale, accumulate, dtable, s.partial, (const uint8_t*)s.touched, s.counts + s.count_words - 4, s.lists);
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
  if (n > MAX_TOKENS || d > MAX_WIDTH) return FAX_ERR_UNSUPPORTED_SHAPE;
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
  carve(ar, most_for(n > 0 ? n : 1, vocab), vocab, d, &s);
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
  const bool wide = fax_aligned(dout, 16) && fax_aligned(dtable, 16);
  {
    // The route and the cut of a list into parts follow d and the type, never the alignment: the sums' order, and so
    // their bits, are those of aligned buffers.
    const int v = prec == FAX_PREC_BF16 ? (d % 8 == 0 ? 8 : 1) : (d % 4 == 0 ? 4 : 1);
    int lanes, slices;
    lanes_for(d / v, DIRECT_LANES, &lanes, &slices);
    if (n <= DIRECT_TOKENS && (long long)n * slices <= DIRECT_BLOCKS) {
      const int acc = accumulate ? 1 : 0;
      const bool vec = wide && v > 1;
      if (prec == FAX_PREC_BF16)
        return vec ? launch_direct<bf16, 8>(ctx, n, vocab, d, lanes, ids, dout, scale, acc, dtable)
                   : launch_direct<bf16, 1>(ctx, n, vocab, d, lanes, ids, dout, scale, acc, dtable);
      return vec ? launch_direct<float, 4>(ctx, n, vocab, d, lanes, ids, dout, scale, acc, dtable)
                 : launch_direct<float, 1>(ctx, n, vocab, d, lanes, ids, dout, scale, acc, dtable);
    }
  }
  const SortPlan p = plan_for(n, vocab);
  FaxArena ar(scratch, scratch_bytes);
  EmbedScratch s;
  carve(ar, p, vocab, d, &s);
  const double rows = n < vocab ? n : vocab;
  const bool prefill = !accumulate && fax_aligned(dtable, 16) && ((size_t)vocab * d) % 4 == 0 && rows * d * 4.0 <= PREFILL_BYTES;
  const bool mark = !accumulate && !prefill;
  const unsigned long long later = s.count_words - (size_t)p.tiles * DIGITS, tv = mark ? fax_round_up((size_t)vocab, 16) / 16 : 0;
  // the zeros in equal shares under the counting and each pass
  const unsigned long long vecs = prefill ? (unsigned long long)vocab * d / 4 : 0, shares = p.passes + 1;
  const unsigned long long share = (vecs + shares - 1) / shares;
  auto part = [&](unsigned long long k) {
    Fill f;
    f.p = (float4*)dtable;
    f.lo = k * share < vecs ? k * share : vecs;
    f.hi = f.lo + share < vecs ? f.lo + share : vecs;
    return f;
  };
  auto fill_blocks = [&](const Fill& f) {
    const unsigned long long want = (f.hi - f.lo + 4 * SORT_THREADS - 1) / (4 * SORT_THREADS), cap = (unsigned long long)ctx->sm_count * 4;
    return (unsigned int)(want < cap ? want : cap);
  };
  Fill f = part(0);
  fax_launch(ctx, embed_sort_count_kernel, dim3(p.tiles + fill_blocks(f)), dim3(SORT_THREADS), 0, p, vocab, ids, s.counts, later, (uint4*)s.touched, tv, f);
  FAX_TRY(fax_after_launch(ctx));
  for (int pass = 0; pass < p.passes; ++pass) {
    uint2* out = (pass & 1) ? s.b : s.a;
    const uint2* in = (pass & 1) ? s.a : s.b;
    f = part(pass + 1);
    const dim3 grid(p.tiles + fill_blocks(f));
    if (pass == 0)
      fax_launch(ctx, embed_sort_scatter_kernel<true>, grid, dim3(SORT_THREADS), 0, p, pass, vocab, ids, in, out, s.counts, mark ? s.touched : (uint8_t*)nullptr, f);
    else
      fax_launch(ctx, embed_sort_scatter_kernel<false>, grid, dim3(SORT_THREADS), 0, p, pass, vocab, ids, in, out, s.counts, (uint8_t*)nullptr, f);
    FAX_TRY(fax_after_launch(ctx));
  }
  const uint2* sorted = ((p.passes - 1) & 1) ? s.b : s.a;
  const int acc = accumulate ? 1 : 0;
  if (prec == FAX_PREC_BF16)
    FAX_TRY((wide && d % 8 == 0 ? launch_grad<bf16, 8>(ctx, p, vocab, d, sorted, dout, scale, acc, mark, dtable, s)
                                : launch_grad<bf16, 1>(ctx, p, vocab, d, sorted, dout, scale, acc, mark, dtable, s)));
  else
    FAX_TRY((wide && d % 4 == 0 ? launch_grad<float, 4>(ctx, p, vocab, d, sorted, dout, scale, acc, mark, dtable, s)
                                : launch_grad<float, 1>(ctx, p, vocab, d, sorted, dout, scale, acc, mark, dtable, s)));
  if (p.chunks > 1) {
    const long long items = (long long)p.chunks * ((d + 1023) / 1024), cap = (long long)ctx->sm_count * 8;
    const dim3 grid((unsigned int)(items < cap ? items : cap));
    const uint32_t* len = s.counts + s.count_words - 4;
    if (d % 4 == 0 && fax_aligned(dtable, 16))
      fax_launch(ctx, embed_join_kernel<true>, grid, dim3(32 * JOIN_WARPS), 0, p, d, sorted, (const float*)s.partial, len, (const uint2*)s.lists, scale, acc, dtable);
    else
      fax_launch(ctx, embed_join_kernel<false>, grid, dim3(32 * JOIN_WARPS), 0, p, d, sorted, (const float*)s.partial, len, (const uint2*)s.lists, scale, acc, dtable);
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
