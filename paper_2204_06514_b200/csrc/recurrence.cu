// Gated linear recurrence over sequences, forward and backward (see fax_ops.h): h_t = a_t h_{t-1} + b_t for each channel.
//
// A stretch of tokens maps the state before it to the state behind it as h -> A h + B, and two stretches join as
// (A2 A1, A2 B1 + B2), so that time can be split: a thread folds 16 tokens of its channels into (A, B), the (A, B) of
// the stretches before it are joined in their order, and with the state that gives it goes over its 16 tokens again.
// Backward the same runs from the end: e_t = a_t (u_t + e_{t+1}) with u_t = dy_t gate_t is what token t hands to the one
// before it, dh_t = u_t + e_{t+1}; h itself is worked out again from the state the forward pass kept for every 16th token.
// Inputs are read once and outputs written once, which is the floor of both passes (memory); next to it stand the
// instructions, so that two channels share one wherever the hardware has it (f32x2).
//
// A warp has 64 channels, two a lane, and 16 tokens at a time.  Where sequences are few, a cluster of CTAs shares one:
// each CTA has 4 to 8 warps, one after the other in time, and the CTAs of a cluster follow one another; (A, B) of a CTA goes to
// the others through distributed shared memory, once a round of (CTAs * warps * 16) tokens.  Where channels and sequences
// alone fill the GPU, or sequences are one stretch, each warp takes a whole sequence by itself.
// The order of joining is fixed by the sizes: the same inputs give the same bits.
#include <type_traits>

#include "gemm_common.cuh"
#include "stream_common.cuh"
#include "../../include/fax_ops.h"

namespace {

constexpr int MAX_WARPS = 16;                    // of a CTA: 128 registers a thread
constexpr int STEPS = FAX_RECURRENCE_BLOCK;      // tokens of a stretch
constexpr int CHANNELS = 64;                     // of a warp
constexpr int MAX_CLUSTER = 16;
constexpr int MAX_STAGES = 2;
constexpr int SMEM_MAX = 226 * 1024;

// How rows come in and go out.  TILES: 16 x 64 boxes by TMA through shared memory, the next round's under the current
// one's work (the backward pass, which has no room for its outputs, and a sequence's last rows, fewer than 16, are
// stored row by row).  PAIRS: the same boxes filled by the lanes, a lane's two channels side by side in one access.
// SINGLES: a lane has channels c and c + 32, an access each, for widths, pitches and addresses of any kind.
enum Rows { TILES, PAIRS, SINGLES };

struct RecurrenceParams {
  int32_t rows, d, n_seq, seq, tiles;
  const int32_t* offsets;
  const void *f, *x, *g, *dy;
  void *y, *df, *dx, *dg;
  int64_t ldf, ldx, ldg, lddy, ldy, lddf, lddx, lddg;
  const float *h0, *dh_last;
  float *h_last, *states, *dh0;
  int32_t units;                                 // sequences * tiles of channels
  int32_t warps;                                 // of a CTA
  int32_t stages;                                // buffers of a warp (TILES: up to MAX_STAGES; else 1)
  int32_t* status;
};
struct Maps { CUtensorMap in[4], out; };          // f, x, (g), (dy); y

// ---- two channels at once ----

typedef unsigned long long two;
__device__ __forceinline__ two pack2(float a, float b) { two r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float2 unpack2(two v) { float2 r; asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v)); return r; }
__device__ __forceinline__ two mul2(two a, two b) { two r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ two add2(two a, two b) { two r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ two fma2(two a, two b, two c) { two r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }

// Two elements as they are stored.
template <typename T> struct Raw;
template <> struct Raw<bf16> {
  uint32_t v;
  __device__ __forceinline__ two wide() const { return pack2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
  static __device__ __forceinline__ Raw of(two x) {
    const float2 f = unpack2(x);
    const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
    return {*reinterpret_cast<const uint32_t*>(&h)};
  }
  static __device__ __forceinline__ Raw of(bf16 a, bf16 b) { return {(uint32_t)__bfloat16_as_ushort(a) | (uint32_t)__bfloat16_as_ushort(b) << 16}; }
  __device__ __forceinline__ bf16 first() const { return __ushort_as_bfloat16((unsigned short)v); }
  __device__ __forceinline__ bf16 second() const { return __ushort_as_bfloat16((unsigned short)(v >> 16)); }
};
template <> struct Raw<float> {
  two v;
  __device__ __forceinline__ two wide() const { return v; }
  static __device__ __forceinline__ Raw of(two x) { return {x}; }
  static __device__ __forceinline__ Raw of(float a, float b) { return {pack2(a, b)}; }
  __device__ __forceinline__ float first() const { return unpack2(v).x; }
  __device__ __forceinline__ float second() const { return unpack2(v).y; }
};

// sigmoid(f) and sigmoid(-f), both with a small relative error (where a is close to 1, 1 - a is what a channel forgets): with
// e = exp(-f) they are 1 / (1 + e) and e / (1 + e).  bf16 inputs take the hardware's exponential and reciprocal (within 2^-21 + |f| 2^-23
// of their values, against the 2^-8 of f's and the outputs' own rounding) and cut e at 2^126, whose reciprocal is still normal, so that
// the second one is 1 from there on.  The first one would stay at 2^-126, which times the lowest bf16 as a gate is -4: it is taken 2^-126 lower,
// 0 from there on and elsewhere off by no more than what a float flushes.  min keeps a NaN.  Float inputs take the library's functions of |f|.
template <typename T>
__device__ __forceinline__ void gates(two f, two* a, two* rest) {
  if constexpr (sizeof(T) == 2) {
    const float2 t = unpack2(mul2(f, pack2(-1.4426950408889634f, -1.4426950408889634f)));
    float e0, e1, r0, r1;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(t.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(t.y));
    asm("min.NaN.f32 %0, %0, 0f7E800000;" : "+f"(e0));                          // 2^126
    asm("min.NaN.f32 %0, %0, 0f7E800000;" : "+f"(e1));
    const two e = pack2(e0, e1);
    const float2 s = unpack2(add2(e, pack2(1.f, 1.f)));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r0) : "f"(s.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r1) : "f"(s.y));
    const two r = pack2(r0, r1);
    *a = add2(r, pack2(-0x1p-126f, -0x1p-126f));
    *rest = mul2(e, r);
  } else {
    const float2 v = unpack2(f);
    float big[2], small[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float e = expf(-fabsf(i ? v.y : v.x));
      big[i] = 1.f / (1.f + e);
      small[i] = e * big[i];
    }
    *a = pack2(v.x < 0.f ? small[0] : big[0], v.y < 0.f ? small[1] : big[1]);
    *rest = pack2(v.x < 0.f ? big[0] : small[0], v.y < 0.f ? big[1] : small[1]);
  }
}

// ---- clusters ----

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cluster_size() { uint32_t r; asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Where a state is written in the place of the one it began with: no CTA writes it before all have read theirs.
__device__ __forceinline__ void cluster_has_read() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait_read() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
// The CTAs of a cluster go together: none leaves while another one may still send to it.  (Where no wait ran out everything sent has been
// received by then, so that nothing has to be ordered.)
__device__ __forceinline__ void cluster_arrive_end() { asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait_end() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
// Where a wait ran out, rows asked for and other CTAs' links may still be on their way into this CTA's memory: they get as long again as the wait had.
__device__ __forceinline__ void let_arrive(volatile int* gave_up) {
  if (!*gave_up) return;
  const long long t0 = clock64();
  while (clock64() - t0 < tc::WAIT_CYCLES) {}
}

// (A, B) of a lane's two channels.
struct alignas(16) Link { two a, b; };
// To the same place of CTA `rank`, whose barrier at the place of `bar` counts the bytes: nothing else is waited for or flushed.
__device__ __forceinline__ void send(const Link* here, uint32_t bar, uint32_t rank, const Link& v) {
  uint32_t at, remote_bar;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(tc::smem_u32(here)), "r"(rank));
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote_bar) : "r"(bar), "r"(rank));
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.b64 [%0], {%1, %2}, [%3];" ::"r"(at), "l"(v.a), "l"(v.b), "r"(remote_bar) : "memory");
}
// Bounded wait for what other CTAs sent; false where it ran out.
__device__ __forceinline__ bool wait_sent(uint32_t bar, uint32_t parity, volatile int* gave_up, int32_t* status) {
  const long long t0 = clock64();
  for (int spins = 0;; ++spins) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    if (ok) return true;
    if ((spins & 255) == 255) {
      if (*gave_up) return false;
      if (clock64() - t0 > tc::WAIT_CYCLES) {
        *gave_up = 1;
        if (atomicCAS(status, 0, 1) == 0) status[1] = 602;
        return false;
      }
    }
  }
}

constexpr uint32_t RAN_OUT = 1u << 31;            // a wait of this warp has run out: it asks and waits for nothing any more

// What warps and CTAs tell one another, in the order of joining.  The CTAs' links have two places that take turns: one is written again two rounds
// later, by a CTA that has received this CTA's link of the round between, which was sent after the reading of it.
struct Exchange {
  Link* links;                                   // [warps][32] of the CTA's warps
  Link* ctas;                                    // [2][CTAs][32]
  two* starts;                                   // [warps][32]: the states before the warps' stretches
  int n_warps, n_ctas;
  uint32_t bars;                                 // two barriers, of what the CTAs send
  volatile int* gave_up;
  int32_t* status;
  __device__ __forceinline__ Exchange(uint8_t* mem, int warps, int n, volatile int* flag, int32_t* s)
      : links(reinterpret_cast<Link*>(mem)), ctas(links + warps * 32), starts(reinterpret_cast<two*>(ctas + 2 * n * 32)), n_warps(warps), n_ctas(n),
        bars(tc::smem_u32(starts + warps * 32)), gave_up(flag), status(s) {}
  static __host__ __device__ constexpr int bytes(int warps, int n) { return (warps + 2 * n) * 32 * (int)sizeof(Link) + warps * 32 * (int)sizeof(two); }      // then the barriers
};

// Which stretches of which sequence a warp works on.
template <int ROWS, bool CLUSTER>
struct Place {
  int warp, lane, seq, tile, slot, n;            // slot: place in time among the warps that share the sequence
  uint32_t rank, ctas;
  int64_t lo, block0;                            // first row, first kept state
  int c0;                                        // first of the lane's channels
  bool live0, live1, whole;                      // channels there are; all of the warp's
  int span, rounds;                              // tokens of a round
  static constexpr int STEP = ROWS == SINGLES ? 32 : 1;          // from the first channel to the second
  __device__ __forceinline__ bool set(const RecurrenceParams& p) {
    warp = __shfl_sync(0xffffffffu, (int)threadIdx.x / 32, 0);
    lane = threadIdx.x % 32;
    int unit;
    if (CLUSTER) {
      rank = cluster_rank(); ctas = cluster_size();
      unit = blockIdx.x / ctas;
      slot = rank * p.warps + warp;
      span = ctas * p.warps * STEPS;
    } else {
      rank = 0; ctas = 1;
      unit = blockIdx.x * p.warps + warp;
      slot = 0;
      span = STEPS;
      if (unit >= p.units) return false;
    }
    seq = unit / p.tiles;
    tile = unit - seq * p.tiles;
    c0 = tile * CHANNELS + (ROWS == SINGLES ? lane : 2 * lane);
    live0 = c0 < p.d;
    live1 = c0 + STEP < p.d;
    whole = (tile + 1) * CHANNELS <= p.d;
    if (p.offsets) {
      const int a = min(max(p.offsets[seq], 0), p.rows), b = min(max(p.offsets[seq + 1], a), p.rows);
      lo = a; n = b - a;
    } else {
      lo = (int64_t)seq * p.seq; n = p.seq;
    }
    block0 = lo / STEPS + seq;
    rounds = (n + span - 1) / span;
    return true;
  }
  __device__ __forceinline__ two load_state(const float* row) const {
    return pack2(live0 ? row[c0] : 0.f, live1 ? row[c0 + STEP] : 0.f);
  }
  __device__ __forceinline__ void store_state(float* row, two v) const {
    const float2 f = unpack2(v);
    if (ROWS != SINGLES) { if (live0) *reinterpret_cast<float2*>(row + c0) = f; }
    else { if (live0) row[c0] = f.x; if (live1) row[c0 + STEP] = f.y; }
  }
  // ALL: rows and channels are all there.
  template <bool ALL, typename T>
  __device__ __forceinline__ Raw<T> load(const T* at, bool row) const {      // at: the lane's first channel
    if (ALL) {
      if (ROWS != SINGLES) return *reinterpret_cast<const Raw<T>*>(at);
      return Raw<T>::of(at[0], at[STEP]);
    }
    if (ROWS != SINGLES) {
      Raw<T> r = Raw<T>::of(0ull);
      if (live0 && row) r = *reinterpret_cast<const Raw<T>*>(at);
      return r;
    }
    return Raw<T>::of(live0 && row ? at[0] : from_f32<T>(0.f), live1 && row ? at[STEP] : from_f32<T>(0.f));
  }
  template <typename T>
  __device__ __forceinline__ void store(T* at, Raw<T> v) const {
    if (ROWS != SINGLES) { if (live0) *reinterpret_cast<Raw<T>*>(at) = v; }
    else { if (live0) at[0] = v.first(); if (live1) at[STEP] = v.second(); }
  }
};

// Joins the stretches of a round: mine is this warp's; carry (of the first warp): the state before the round, afterwards the one behind
// it; waits: RAN_OUT in it when a wait of the first warp has run out; returns the state before this warp's stretch.  The first warp does it for all: every warp reading every link is bound by shared
// memory (16 CTAs of 8 warps: 2400 of a round's 5200 cycles that way).  FORWARD: earlier slots come first; else later ones.
template <bool FORWARD, typename P>
__device__ __forceinline__ two join(const Exchange& ex, const P& at, int round, const Link& mine, two& carry, uint32_t& waits) {
  const int me = FORWARD ? at.warp : ex.n_warps - 1 - at.warp;
  Link* const links = ex.links + at.lane;
  links[me * 32] = mine;
  tc::named_barrier_sync(1, ex.n_warps * 32);     // (warps with whole and with short stretches come here from different places)
  if (at.warp == 0) {
    two state = carry;
    if (at.ctas > 1) {
      Link all{pack2(1.f, 1.f), 0ull};
#pragma unroll 4
      for (int i = 0; i < ex.n_warps; ++i) {
        const Link s = links[i * 32];
        all.a = mul2(all.a, s.a);
        all.b = fma2(s.a, all.b, s.b);
      }
      const int my_cta = FORWARD ? at.rank : at.ctas - 1 - at.rank;
      const uint32_t bar = ex.bars + 8 * (round & 1);
      Link* const ctas = ex.ctas + ((round & 1) * ex.n_ctas) * 32 + at.lane;
      // (where a wait ran out this CTA takes no further part, its barriers may be behind; the others' waits run out in their turn)
      if (waits < RAN_OUT) {
        if (at.lane == 0) tc::mbar_expect_tx(bar, at.ctas * 32 * sizeof(Link));
#pragma unroll 4
        for (uint32_t r = 0; r < at.ctas; ++r) send(ctas + my_cta * 32, bar, r, all);
        if (!wait_sent(bar, (round >> 1) & 1, ex.gave_up, ex.status)) waits |= RAN_OUT;
      }
#pragma unroll 4
      for (int c = 0; c < my_cta; ++c) {
        const Link s = ctas[c * 32];
        carry = fma2(s.a, carry, s.b);
      }
      state = carry;
#pragma unroll 4
      for (int c = my_cta; c < (int)at.ctas; ++c) {
        const Link s = ctas[c * 32];
        carry = fma2(s.a, carry, s.b);
      }
    }
#pragma unroll 4
    for (int i = 0; i < ex.n_warps; ++i) {
      const Link s = links[i * 32];
      ex.starts[i * 32 + at.lane] = state;
      state = fma2(s.a, state, s.b);
    }
    if (at.ctas == 1) carry = state;
    else if (__any_sync(0xffffffffu, waits >= RAN_OUT)) waits |= RAN_OUT;                  // (one lane for all, not right behind the wait: 93.2 -> 91.1 us at 1 x 65536 x 768)
  }
  tc::named_barrier_sync(1, ex.n_warps * 32);
  return ex.starts[me * 32 + at.lane];
}

// ---- rows coming in ----

template <typename T> constexpr int box_bytes() { return STEPS * CHANNELS * (int)sizeof(T); }

// N tensors' rows of one stretch, in a warp's buffer of N boxes of STEPS x CHANNELS elements, a lane's two side by side.
template <typename T, int N>
struct Inputs {
  uint8_t* at;                                   // this lane's pair of row 0
  template <int K>
  __device__ __forceinline__ Raw<T>* place(int i) const { return reinterpret_cast<Raw<T>*>(at + K * box_bytes<T>() + i * CHANNELS * (int)sizeof(T)); }
  __device__ __forceinline__ two get(int k, int i) const { return reinterpret_cast<const Raw<T>*>(at + k * box_bytes<T>() + i * CHANNELS * (int)sizeof(T))->wide(); }
  // PAIRS and SINGLES: through registers, R rows' loads on their way together.
  template <int R, bool ALL, typename P>
  __device__ __forceinline__ void fetch(const P& pl, const T* const (&src)[N], const int64_t (&ld)[N], int64_t row, int count) const {
    Raw<T> r[N][R];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const T* q = src[k] + row * ld[k] + pl.c0;
#pragma unroll
      for (int i = 0; i < R; ++i) {
        r[k][i] = pl.template load<ALL>(q, i < count);
        q += ld[k];
      }
    }
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int i = 0; i < R; ++i) *reinterpret_cast<Raw<T>*>(at + k * box_bytes<T>() + i * CHANNELS * (int)sizeof(T)) = r[k][i];
  }
  template <typename P>
  __device__ __forceinline__ void fetch(const P& pl, const T* const (&src)[N], const int64_t (&ld)[N], int64_t row, int count) const {
    if (count == STEPS && pl.whole) fetch<STEPS, true>(pl, src, ld, row, count);
    else if (count > 4) fetch<STEPS, false>(pl, src, ld, row, count);
    else if (count > 1) fetch<4, false>(pl, src, ld, row, count);
    else if (count == 1) fetch<1, false>(pl, src, ld, row, count);
  }
};

// A warp's buffers, in turn, and the barriers that say they are full.  With two, rows are asked for a round ahead; a buffer
// is asked for again when every lane has read it and what was stored from it has left.
template <typename T, int N>
struct Tiles {
  uint32_t bar, phase = 0;                       // barriers, their phases and RAN_OUT
  uint8_t* buf;
  int stages, now;                               // buffers, the current round's one
  __device__ __forceinline__ void init(uint8_t* buffers, uint64_t* bars, int n, int lane) {
    buf = buffers; bar = tc::smem_u32(bars); stages = n; now = 0;
    if (lane == 0) {
#pragma unroll
      for (int i = 0; i < MAX_STAGES; ++i) tc::mbar_init(bar + 8 * i, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
  }
  __device__ __forceinline__ uint8_t* current() const { return buf + now * N * box_bytes<T>(); }
  // The rows of `ahead` rounds from now, when lane 0's stores have left their buffers.
  // (None when a wait has run out: the buffer may be one that is still waited for.)
  __device__ __forceinline__ void ask(const Maps& maps, int ahead, int col, int64_t row, int lane) {
    int s = now + ahead;
    s = s >= stages ? s - stages : s;
    __syncwarp();
    if (lane == 0 && phase < RAN_OUT) {
      tc::bulk_wait_read_all();
      tc::mbar_expect_tx(bar + 8 * s, N * box_bytes<T>());
#pragma unroll
      for (int k = 0; k < N; ++k) tc::tma_load_2d(tc::smem_u32(buf + (s * N + k) * box_bytes<T>()), &maps.in[k], bar + 8 * s, col, (int)row);
    }
  }
  // Bounded; a wait that runs out sets the context's status, and the work goes on with what is there, without further waits, so that nobody waits for this warp.
  __device__ __forceinline__ void wait(volatile int* gave_up, int32_t* status) {
    if (phase < RAN_OUT && !tc::mbar_wait_warp(bar + 8 * now, (phase >> now) & 1, gave_up, status, 601)) phase |= RAN_OUT;
    phase ^= 1u << now;
  }
  __device__ __forceinline__ void next() { now = now + 1 == stages ? 0 : now + 1; }
};
// Before what the lanes wrote to shared memory is stored by lane 0.
__device__ __forceinline__ void written() { tc::fence_proxy_async(); __syncwarp(); }

__host__ __device__ constexpr int align128(int n) { return (n + 127) / 128 * 128; }
// Shared memory: the exchange of a cluster (its bytes), its two barriers and each warp's, then the warps' buffers (their place).
template <bool CLUSTER> __host__ __device__ constexpr int exchange_bytes(int warps, int ctas) { return CLUSTER ? Exchange::bytes(warps, ctas) : 0; }
template <bool CLUSTER> __host__ __device__ constexpr int buffers_at(int warps, int ctas) { return align128(exchange_bytes<CLUSTER>(warps, ctas) + 16 + warps * 8 * MAX_STAGES); }

template <typename T, int ROWS, bool GATE, bool COMPLEMENT, bool CLUSTER>
__global__ void __launch_bounds__(MAX_WARPS * 32, 1) recurrence_forward_kernel(const __grid_constant__ Maps maps, const RecurrenceParams p) {
  constexpr int N = 2 + GATE;
  extern __shared__ __align__(128) uint8_t mem[];
  __shared__ int gave_up;
  const int ctas = CLUSTER ? (int)cluster_size() : 1;
  const Exchange ex(mem, p.warps, ctas, &gave_up, p.status);
  const int warp_buffer = p.stages * N * box_bytes<T>();
  if (threadIdx.x == 0) {
    gave_up = 0;
    if (CLUSTER) {
      tc::mbar_init(ex.bars, 1);
      tc::mbar_init(ex.bars + 8, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
  }
  Tiles<T, N> tiles;
  uint8_t* const buffer = mem + buffers_at<CLUSTER>(p.warps, ctas) + (threadIdx.x / 32) * warp_buffer;
  if (ROWS == TILES)
    tiles.init(buffer, reinterpret_cast<uint64_t*>(mem + exchange_bytes<CLUSTER>(p.warps, ctas) + 16) + threadIdx.x / 32 * MAX_STAGES,
               p.stages, threadIdx.x % 32);
  __syncthreads();
  if (CLUSTER && ctas > 1) cluster_sync();             // the others run: their shared memory can be written
  fax_grid_dependency_wait();
  Place<ROWS, CLUSTER> at;
  if (!at.set(p)) return;
  const int64_t seq_row = (int64_t)at.seq * p.d;
  two carry = p.h0 ? at.load_state(p.h0 + seq_row) : 0ull;
  const bool in_place = CLUSTER && p.h_last && p.h_last == p.h0;
  if (in_place) cluster_has_read();
  const T* src[N]; int64_t ld[N];
  src[0] = (const T*)p.f; ld[0] = p.ldf; src[1] = (const T*)p.x; ld[1] = p.ldx;
  if constexpr (GATE) { src[2] = (const T*)p.g; ld[2] = p.ldg; }

  const int first = at.slot * STEPS;
  auto tokens = [&](int round) { return round < at.rounds ? min(max(at.n - (round * at.span + first), 0), STEPS) : 0; };
  const int ahead = p.stages - 1;
  auto ask = [&](int round, int by) {
    if (tokens(round) > 0) tiles.ask(maps, by, at.tile * CHANNELS, at.lo + (int64_t)round * at.span + first, at.lane);
  };
  if (ROWS == TILES)
    for (int i = 0; i < max(ahead, 1); ++i) ask(i, i);
  for (int round = 0; round < at.rounds; ++round) {
    const int count = tokens(round);
    const int64_t row = at.lo + (int64_t)round * at.span + first;
    Inputs<T, N> in;
    if constexpr (ROWS == TILES) {
      if (count > 0) tiles.wait(&gave_up, p.status);
      in.at = tiles.current() + at.lane * 2 * sizeof(T);
    } else {
      in.at = buffer + at.lane * 2 * sizeof(T);
      in.fetch(at, src, ld, row, count);
    }
    T* out = (T*)p.y + row * p.ldy + at.c0;
    float* kept = p.states && count > 0 ? p.states + (at.block0 + (row - at.lo) / STEPS) * p.d : nullptr;
    // FULL: a whole stretch, nothing to look at token by token
    auto work = [&](auto full) {
      constexpr bool FULL = decltype(full)::value, BOX = FULL && ROWS == TILES;
      // y goes out in the place of f
      auto put = [&](int i, two h) {
        two y = h;
        if constexpr (GATE) {
          const two g = in.get(2, i);
          two s, r;
          gates<T>(g, &s, &r);
          y = mul2(h, mul2(g, s));
        }
        if constexpr (BOX) *in.template place<0>(i) = Raw<T>::of(y);
        else at.store(out + i * p.ldy, Raw<T>::of(y));
      };
      if constexpr (CLUSTER) {
        two a[STEPS], b[STEPS];
        Link mine{pack2(1.f, 1.f), pack2(0.f, 0.f)};
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
          a[i] = pack2(1.f, 1.f); b[i] = 0ull;
          if (FULL || i < count) {
            two rest;
            gates<T>(in.get(0, i), &a[i], &rest);
            b[i] = COMPLEMENT ? mul2(rest, in.get(1, i)) : in.get(1, i);
            mine.a = mul2(mine.a, a[i]);
            mine.b = fma2(a[i], mine.b, b[i]);
          }
        }
        if (ROWS == TILES && ahead > 0) ask(round + ahead, ahead);
        two h = join<true>(ex, at, round, mine, carry, tiles.phase);
        if (kept) at.store_state(kept, h);
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
          if (FULL || i < count) {
            h = fma2(a[i], h, b[i]);
            put(i, h);
          }
      } else {
        if (kept) at.store_state(kept, carry);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
          if (FULL || i < count) {
            two a, rest;
            gates<T>(in.get(0, i), &a, &rest);
            carry = fma2(a, carry, COMPLEMENT ? mul2(rest, in.get(1, i)) : in.get(1, i));
            put(i, carry);
          }
          if (ROWS == TILES && i == STEPS / 2 && ahead > 0) ask(round + ahead, ahead);
        }
      }
      if constexpr (BOX) {
        written();
        if (at.lane == 0) {
          tc::tma_store_2d(&maps.out, tc::smem_u32(tiles.current()), at.tile * CHANNELS, (int)row);
          tc::bulk_commit_group();
        }
      }
    };
    if (count == STEPS) work(std::true_type{}); else work(std::false_type{});
    if constexpr (ROWS == TILES) {
      if (ahead == 0) ask(round + 1, 0);
      tiles.next();
    }
  }
  if (in_place) cluster_wait_read();
  if (CLUSTER) cluster_arrive_end();
  if (ROWS == TILES && at.lane == 0) tc::bulk_wait_all();
  if (CLUSTER) cluster_wait_end();
  let_arrive(&gave_up);
  if (p.h_last && at.slot == 0) at.store_state(p.h_last + seq_row, carry);
}

// What the backward pass keeps of a token between its walks over a stretch, in the buffer its inputs were in: w, what h_{t-1} (and x) make of dh in df, and with a gate u.  A lane's own places throughout.
template <typename T>
struct Kept {
  uint8_t* at;                                   // this lane's pair of row 0
  static constexpr bool WIDE = sizeof(T) == 4;   // a pair's place holds two floats; else it takes two boxes' places
  static constexpr int ROW = CHANNELS * (int)sizeof(T), BOX = box_bytes<T>();
  __device__ __forceinline__ void put(int box, int i, two v) const {
    if constexpr (WIDE) {
      *reinterpret_cast<two*>(at + box / 2 * BOX + i * ROW) = v;
    } else {
      const float2 f = unpack2(v);
      *reinterpret_cast<float*>(at + box * BOX + i * ROW) = f.x;
      *reinterpret_cast<float*>(at + (box + 1) * BOX + i * ROW) = f.y;
    }
  }
  __device__ __forceinline__ two get(int box, int i) const {
    if constexpr (WIDE) return *reinterpret_cast<const two*>(at + box / 2 * BOX + i * ROW);
    else return pack2(*reinterpret_cast<const float*>(at + box * BOX + i * ROW), *reinterpret_cast<const float*>(at + (box + 1) * BOX + i * ROW));
  }
  __device__ __forceinline__ void put_w(int i, two v) const { put(0, i, v); }
  __device__ __forceinline__ two get_w(int i) const { return get(0, i); }
  __device__ __forceinline__ void put_u(int i, two v) const { put(2, i, v); }
  __device__ __forceinline__ two get_u(int i) const { return get(2, i); }
};

template <typename T, int ROWS, bool GATE, bool COMPLEMENT, bool CLUSTER>
__global__ void __launch_bounds__(MAX_WARPS * 32, 1) recurrence_backward_kernel(const __grid_constant__ Maps maps, const RecurrenceParams p) {
  constexpr int N = 3 + GATE, DY = 2 + GATE;
  extern __shared__ __align__(128) uint8_t mem[];
  __shared__ int gave_up;
  const int ctas = CLUSTER ? (int)cluster_size() : 1;
  const Exchange ex(mem, p.warps, ctas, &gave_up, p.status);
  const int warp_buffer = p.stages * N * box_bytes<T>();
  uint8_t* const buffer = mem + buffers_at<CLUSTER>(p.warps, ctas) + (threadIdx.x / 32) * warp_buffer;
  if (threadIdx.x == 0) {
    gave_up = 0;
    if (CLUSTER) {
      tc::mbar_init(ex.bars, 1);
      tc::mbar_init(ex.bars + 8, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
  }
  Tiles<T, N> tiles;
  if (ROWS == TILES) tiles.init(buffer, reinterpret_cast<uint64_t*>(mem + exchange_bytes<CLUSTER>(p.warps, ctas) + 16) + threadIdx.x / 32 * MAX_STAGES, p.stages, threadIdx.x % 32);
  __syncthreads();
  if (CLUSTER && ctas > 1) cluster_sync();
  fax_grid_dependency_wait();
  Place<ROWS, CLUSTER> at;
  if (!at.set(p)) return;
  const int64_t seq_row = (int64_t)at.seq * p.d;
  two carry = p.dh_last ? at.load_state(p.dh_last + seq_row) : 0ull;          // e behind the round: what its last token receives
  const bool in_place = CLUSTER && p.dh0 && p.dh0 == p.dh_last;
  if (in_place) cluster_has_read();
  const T* src[N]; int64_t ld[N];
  src[0] = (const T*)p.f; ld[0] = p.ldf; src[1] = (const T*)p.x; ld[1] = p.ldx;
  if constexpr (GATE) { src[2] = (const T*)p.g; ld[2] = p.ldg; }
  src[DY] = (const T*)p.dy; ld[DY] = p.lddy;

  // round 0 is the sequence's last one
  const int first = at.slot * STEPS;
  auto begin = [&](int round) { return (at.rounds - 1 - round) * at.span + first; };
  auto tokens = [&](int round) { return round < at.rounds ? min(max(at.n - begin(round), 0), STEPS) : 0; };
  const int ahead = p.stages - 1;
  auto ask = [&](int round, int by) {
    if (tokens(round) > 0) tiles.ask(maps, by, at.tile * CHANNELS, at.lo + begin(round), at.lane);
  };
  if (ROWS == TILES)
    for (int i = 0; i < max(ahead, 1); ++i) ask(i, i);
  for (int round = 0; round < at.rounds; ++round) {
    const int count = tokens(round);
    const int64_t row = at.lo + begin(round);
    Inputs<T, N> in;
    Kept<T> kept;
    two before = count > 0 ? at.load_state(p.states + (at.block0 + begin(round) / STEPS) * p.d) : 0ull;
    if constexpr (ROWS == TILES) {
      if (ahead > 0) ask(round + ahead, ahead);
      if (count > 0) tiles.wait(&gave_up, p.status);
      in.at = tiles.current() + at.lane * 2 * sizeof(T);
    } else {
      in.at = buffer + at.lane * 2 * sizeof(T);
      in.fetch(at, src, ld, row, count);
    }
    kept.at = in.at;
    // rows are stored a pitch apart; the last walk goes from the end
    auto row_of = [&](void* base, int64_t pitch, int i) { return (T*)base + (row + i) * pitch + at.c0; };
    auto work = [&](auto full) {
      constexpr bool FULL = decltype(full)::value;
      two a[STEPS], rest[STEPS];
      [[maybe_unused]] T* dg = GATE ? row_of(p.dg, p.lddg, 0) : nullptr;
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        a[i] = pack2(1.f, 1.f); rest[i] = 0ull;
        if (FULL || i < count) {
          gates<T>(in.get(0, i), &a[i], &rest[i]);
          const two x = in.get(1, i);
          const two h = fma2(a[i], before, COMPLEMENT ? mul2(rest[i], x) : x);
          const two w = COMPLEMENT ? fma2(x, pack2(-1.f, -1.f), before) : before;
          kept.put_w(i, mul2(w, mul2(a[i], rest[i])));              // (before dh: dh times a state may pass float's range where a shut gate leaves nothing of it)
          if constexpr (GATE) {
            const two g = in.get(2, i), dy = in.get(DY, i);
            two s, r;
            gates<T>(g, &s, &r);
            const two gs = mul2(g, s);
            at.store(dg, Raw<T>::of(mul2(mul2(dy, fma2(gs, r, s)), h)));         // (in this order: see w)
            dg += p.lddg;
            kept.put_u(i, mul2(dy, gs));
          }
          before = h;
        }
      }
      auto u_of = [&](int i) { if constexpr (GATE) return kept.get_u(i); else return in.get(DY, i); };
      two e = carry;
      if constexpr (CLUSTER) {
        Link mine{pack2(1.f, 1.f), pack2(0.f, 0.f)};               // the stretch's, from its end
#pragma unroll
        for (int i = STEPS - 1; i >= 0; --i)
          if (FULL || i < count) {
            mine.a = mul2(mine.a, a[i]);
            mine.b = mul2(a[i], add2(u_of(i), mine.b));
          }
        e = join<false>(ex, at, round, mine, carry, tiles.phase);
      }
      const int last = (FULL ? STEPS : count) - 1;
      T* df = row_of(p.df, p.lddf, last);
      T* dx = row_of(p.dx, p.lddx, last);
#pragma unroll
      for (int i = STEPS - 1; i >= 0; --i)
        if (FULL || i < count) {
          const two dh = add2(u_of(i), e);
          at.store(df, Raw<T>::of(mul2(dh, kept.get_w(i))));
          at.store(dx, Raw<T>::of(COMPLEMENT ? mul2(dh, rest[i]) : dh));
          df -= p.lddf;
          dx -= p.lddx;
          e = mul2(a[i], dh);
        }
      if (ROWS == TILES) tc::fence_proxy_async();                  // this lane wrote to the buffer, which is TMA's again
      if constexpr (!CLUSTER) carry = e;
    };
    if (count == STEPS) work(std::true_type{}); else work(std::false_type{});
    if constexpr (ROWS == TILES) {
      if (ahead == 0) ask(round + 1, 0);
      tiles.next();
    }
  }
  if (in_place) cluster_wait_read();
  if (CLUSTER) cluster_arrive_end();
  if (CLUSTER) cluster_wait_end();
  let_arrive(&gave_up);
  if (p.dh0 && at.slot == 0) at.store_state(p.dh0 + seq_row, carry);
}

// A token or two a sequence (a step of generation): a thread has N neighbouring channels, 16 bytes of them, and walks them through
// its sequence; short code, nothing to set up (256 x 1 x 1024: 7.0 us on the device by the kernels above, 3.7 us by this one).
constexpr int FEW = 2;
constexpr int FEW_THREADS = 128;
template <typename T, int N, bool GATE, bool COMPLEMENT>
__global__ void __launch_bounds__(FEW_THREADS) recurrence_few_kernel(const RecurrenceParams p, const FastDiv vectors) {
  fax_grid_dependency_wait();
  const uint32_t id = blockIdx.x * FEW_THREADS + threadIdx.x;
  const int seq = (int)vectors.div(id), c0 = (int)vectors.mod(id, seq) * N;
  if (seq >= p.n_seq) return;
  int64_t lo = (int64_t)seq * p.seq, n = p.seq;
  if (p.offsets) {
    const int a = min(max(p.offsets[seq], 0), p.rows);
    lo = a; n = min(max(p.offsets[seq + 1], a), p.rows) - a;
  }
  const int64_t sc = (int64_t)seq * p.d + c0;
  Pack<float, N> h;
  if (p.h0) h = load_pack<float, N>(p.h0 + sc);
  else {
#pragma unroll
    for (int i = 0; i < N; ++i) h.e[i] = 0.f;
  }
#pragma unroll 1
  for (int64_t t = 0; t < n; ++t) {
    const int64_t row = lo + t;
    const Pack<T, N> f = load_pack<T, N>((const T*)p.f + row * p.ldf + c0), x = load_pack<T, N>((const T*)p.x + row * p.ldx + c0);
    Pack<T, N> g, y;
    if constexpr (GATE) g = load_pack<T, N>((const T*)p.g + row * p.ldg + c0);
    if (p.states && t % STEPS == 0) store_pack<float, N>(p.states + (lo / STEPS + seq + t / STEPS) * p.d + c0, h);
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      two a, rest;
      gates<T>(pack2(to_f32(f.e[i]), to_f32(f.e[i + 1])), &a, &rest);
      const two xv = pack2(to_f32(x.e[i]), to_f32(x.e[i + 1]));
      two v = fma2(a, pack2(h.e[i], h.e[i + 1]), COMPLEMENT ? mul2(rest, xv) : xv);
      const float2 s = unpack2(v);
      h.e[i] = s.x; h.e[i + 1] = s.y;
      if constexpr (GATE) {
        const two gv = pack2(to_f32(g.e[i]), to_f32(g.e[i + 1]));
        gates<T>(gv, &a, &rest);
        v = mul2(v, mul2(gv, a));
      }
      const Raw<T> o = Raw<T>::of(v);
      y.e[i] = o.first(); y.e[i + 1] = o.second();
    }
    store_pack<T, N>((T*)p.y + row * p.ldy + c0, y);
  }
  if (p.h_last) store_pack<float, N>(p.h_last + sc, h);
}

template <bool BACKWARD, typename T, int ROWS, bool GATE, bool COMPLEMENT, bool CLUSTER>
fax_status launch(fax_ctx* ctx, int64_t grid, int cluster, const Maps& maps, RecurrenceParams p) {
  constexpr int N = 2 + GATE + BACKWARD;
  auto kernel = [] {
    if constexpr (BACKWARD) return recurrence_backward_kernel<T, ROWS, GATE, COMPLEMENT, CLUSTER>;
    else return recurrence_forward_kernel<T, ROWS, GATE, COMPLEMENT, CLUSTER>;
  }();
  auto smem = [&](int stages) { return buffers_at<CLUSTER>(p.warps, cluster) + p.warps * stages * N * box_bytes<T>(); };
  if (ROWS != TILES) p.stages = 1;
  while (p.stages > 1 && smem(p.stages) > SMEM_MAX) --p.stages;
  static bool done[FAX_MAX_DEVICES] = {}, wide[FAX_MAX_DEVICES] = {};
  FAX_TRY(fax_opt_in_shared_memory(ctx, kernel, SMEM_MAX, done));
  if (CLUSTER && cluster > 8 && !(ctx->device < FAX_MAX_DEVICES && wide[ctx->device])) {
    FAX_CUDA_TRY(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    if (ctx->device < FAX_MAX_DEVICES) wide[ctx->device] = true;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid); cfg.blockDim = dim3(p.warps * 32); cfg.dynamicSmemBytes = smem(p.stages); cfg.stream = ctx->stream;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = ctx->use_pdl ? 2 : 1;
  (void)cudaLaunchKernelEx(&cfg, kernel, maps, p);          // errors surface in fax_after_launch
  return fax_after_launch(ctx);
}

template <bool BACKWARD, typename T, int ROWS, bool CLUSTER>
fax_status launch(fax_ctx* ctx, bool complement, int64_t grid, int cluster, const Maps& maps, const RecurrenceParams& p) {
  if (p.g) return complement ? launch<BACKWARD, T, ROWS, true, true, CLUSTER>(ctx, grid, cluster, maps, p) : launch<BACKWARD, T, ROWS, true, false, CLUSTER>(ctx, grid, cluster, maps, p);
  return complement ? launch<BACKWARD, T, ROWS, false, true, CLUSTER>(ctx, grid, cluster, maps, p) : launch<BACKWARD, T, ROWS, false, false, CLUSTER>(ctx, grid, cluster, maps, p);
}

// Boxes of 16 rows x 64 columns, as they are in memory.
bool make_map_rows(fax_ctx* ctx, CUtensorMap* map, const void* base, int64_t cols, int64_t rows, int64_t ld, bool f32) {
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)ld * (f32 ? 4 : 2)};
  cuuint32_t box[2] = {CHANNELS, STEPS};
  cuuint32_t estr[2] = {1, 1};
  return ((tc::EncodeTiledFn)ctx->encode_tiled)(map, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, (void*)base, dims, strides, box, estr,
                                            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// How warps share the work.  warp_bytes: one of a warp's buffers.
struct Shape { bool alone; int warps, cluster; };
template <bool BACKWARD>
Shape shape_for(const fax_ctx* ctx, int64_t units, int seq, int warp_bytes) {
  const int64_t sms = ctx->sm_count;
  // A warp a sequence and tile: sequences of one stretch, or 12 warps an SM and more of them.
  if (seq <= STEPS || units >= 12 * sms) {
    // (backward, CTAs of 4 warps: 12 warps an SM; of 16, with one buffer each: 16, where shared memory holds them: floats with a gate are 4 boxes of
    // 4 KB a warp, 16 of which would be 256 KB)
    auto rounds = [&](int64_t an_sm) { return (units + an_sm * sms - 1) / (an_sm * sms) * an_sm; };
    const bool fits = buffers_at<false>(MAX_WARPS, 1) + MAX_WARPS * warp_bytes <= SMEM_MAX;
    return {true, BACKWARD && fits && seq > 2 * STEPS && rounds(16) * 20 < rounds(12) * 19 ? MAX_WARPS : 4, 1};
  }
  // Else CTAs of `warps`, a cluster of them a sequence and tile: as many warps as the SMs hold at once, and no more than the
  // longest sequence has stretches for.  By its registers an SM holds 16 warps of the forward pass, 12 of the backward pass; where shared memory holds fewer (float
  // boxes, a gate in a cluster of 16 CTAs) some CTAs come in a second wave, which the rule does not weigh.
  Shape best{false, 4, 1};
  int64_t most = 0;
  for (const int warps : {4, BACKWARD ? 6 : 8}) {
    const int an_sm = BACKWARD ? 12 / warps : 16 / warps;
    for (int cluster = 1; cluster <= MAX_CLUSTER; cluster *= 2) {
      if (cluster > 1 && (cluster / 2) * warps * STEPS >= seq) break;
      if (cluster > 1 && units * cluster > (cluster == 16 ? 112 : sms) * an_sm) break;                // (seven GPCs have 16 SMs for a cluster of 16)
      const int64_t held = units * cluster > sms * an_sm ? sms * an_sm * warps : units * cluster * warps;
      if (held > most || (held == most && best.cluster > 2 && cluster < best.cluster)) { best = {false, warps, cluster}; most = held; }
    }
  }
  return best;
}

template <bool BACKWARD, typename T>
fax_status run(fax_ctx* ctx, RecurrenceParams p, bool complement) {
  if constexpr (!BACKWARD) {
    constexpr int n = 16 / (int)sizeof(T);
    auto fits = [&](const void* q, int64_t ld) { return !q || fax_rows_aligned(q, ld, sizeof(T), 16); };
    const int64_t threads = (int64_t)p.n_seq * (p.d / n);
    if (p.seq <= FEW && p.d % n == 0 && fits(p.f, p.ldf) && fits(p.x, p.ldx) && fits(p.g, p.ldg) && fits(p.y, p.ldy) && fax_aligned(p.h0, 16) && fax_aligned(p.h_last, 16) &&
        fax_aligned(p.states, 16) && threads <= 0x7fffffff - FEW_THREADS) {
      void (*kernel)(RecurrenceParams, FastDiv) = p.g ? (complement ? recurrence_few_kernel<T, n, true, true> : recurrence_few_kernel<T, n, true, false>)
                                                      : (complement ? recurrence_few_kernel<T, n, false, true> : recurrence_few_kernel<T, n, false, false>);
      fax_launch(ctx, kernel, dim3((unsigned)((threads + FEW_THREADS - 1) / FEW_THREADS)), dim3(FEW_THREADS), 0, p, FastDiv((uint32_t)(p.d / n)));
      return fax_after_launch(ctx);
    }
  }
  p.tiles = (p.d + CHANNELS - 1) / CHANNELS;
  const int64_t units = (int64_t)p.n_seq * p.tiles;
  if (units > 0x7fffffff / MAX_CLUSTER) return FAX_ERR_UNSUPPORTED_SHAPE;
  p.units = (int32_t)units;
  p.status = ctx->dev_status;
  const Shape shape = shape_for<BACKWARD>(ctx, units, p.seq, (2 + (p.g != nullptr) + BACKWARD) * box_bytes<T>());
  const bool alone = shape.alone;
  const int cluster = shape.cluster;
  p.warps = shape.warps;
  const int span = (alone ? 1 : cluster * p.warps) * STEPS;
  p.stages = p.seq > span ? 2 : 1;
  const int64_t grid = alone ? (units + p.warps - 1) / p.warps : units * cluster;

  // Pairs of channels: addresses and pitches of whole pairs (states: of 8 bytes).  Boxes: of 16 bytes.
  const size_t es = sizeof(T);
  const void* const ins[4] = {p.f, p.x, p.g, p.dy};
  const int64_t in_ld[4] = {p.ldf, p.ldx, p.ldg, p.lddy};
  const void* const outs[4] = {p.y, p.df, p.dx, p.dg};
  const int64_t out_ld[4] = {p.ldy, p.lddf, p.lddx, p.lddg};
  bool pairs = p.d % 2 == 0, boxes = p.rows > 0;
  for (int i = 0; i < 4; ++i) {
    pairs = pairs && (!ins[i] || fax_rows_aligned(ins[i], in_ld[i], es, 2 * es)) && (!outs[i] || fax_rows_aligned(outs[i], out_ld[i], es, 2 * es));
    boxes = boxes && (!ins[i] || (fax_rows_aligned(ins[i], in_ld[i], es, 16) && in_ld[i] * (int64_t)es < (1ll << 40))) ;
  }
  boxes = boxes && (BACKWARD || (fax_rows_aligned(p.y, p.ldy, es, 16) && p.ldy * (int64_t)es < (1ll << 40)));
  pairs = pairs && fax_aligned(p.h0, 8) && fax_aligned(p.dh_last, 8) && fax_aligned(p.h_last, 8) && fax_aligned(p.dh0, 8) && fax_aligned(p.states, 8);
  Maps maps = {};
  if (p.seq > STEPS && pairs && boxes) {
    int n = 0;
    for (int i = 0; i < 4; ++i)
      if (ins[i] && !make_map_rows(ctx, &maps.in[n++], ins[i], p.d, p.rows, in_ld[i], es == 4)) return FAX_ERR_INVALID_ARG;
    if (!BACKWARD && !make_map_rows(ctx, &maps.out, p.y, p.d, p.rows, p.ldy, es == 4)) return FAX_ERR_INVALID_ARG;
    return alone ? launch<BACKWARD, T, TILES, false>(ctx, complement, grid, 1, maps, p) : launch<BACKWARD, T, TILES, true>(ctx, complement, grid, cluster, maps, p);
  }
  if (!alone) return launch<BACKWARD, T, SINGLES, true>(ctx, complement, grid, cluster, maps, p);
  return pairs ? launch<BACKWARD, T, PAIRS, false>(ctx, complement, grid, 1, maps, p) : launch<BACKWARD, T, SINGLES, false>(ctx, complement, grid, 1, maps, p);
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
  const bool complement = d->input == FAX_RECURRENCE_COMPLEMENT;
  return prec == FAX_PREC_BF16 ? run<false, bf16>(ctx, p, complement) : run<false, float>(ctx, p, complement);
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
  const bool complement = d->input == FAX_RECURRENCE_COMPLEMENT;
  return prec == FAX_PREC_BF16 ? run<true, bf16>(ctx, p, complement) : run<true, float>(ctx, p, complement);
}
