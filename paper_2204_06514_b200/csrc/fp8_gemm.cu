// Product of two matrices in 8-bit floating point with a power-of-two scale for each block of 128 along K:
//
//   C[m, n] = sum_b sa[b, m] sb[b, n] sum_{k in block b} A[m, k] B[n, k]   (+ bias[n])  (+ C[m, n])
//
// The scales differ from row to row and block to block, so they cannot be applied after the sum over all of
// K.  Applied to each block's accumulator by the row warps, they cost a hand-over of the accumulator per 128
// k: two accumulators in flight leave 512 cycles for it and it takes about 770 (8192 x 16384 x 4096: 654 us).
// Powers of two are the tensor core's own scale type (ue8m0, one byte): kind::mxf8f6f4 multiplies each
// row's 32 k by the row's scale on the way in, the accumulator is handed over once a tile, and
// a scale of 128 k is the same byte for four MMAs.
//
// Scales travel like this: float32 in global memory -> exponent bytes, four blocks of K in one word per row,
// packed by the scale warps into shared memory -> tensor memory (tcgen05.cp, 32 x 128 bits, copied to the four
// lane quarters) -> named by the MMA, which picks the byte of its block of K.
//
//   warp 0      : TMA producer
//   warp 1      : tensor-memory allocation, scale copies and MMA issue (even CTA of a pair)
//   warps 2, 3  : scales of every other group of four K blocks; warps 12, 13: of the groups between
//   warps 4..11 : epilogue; warp w reads lanes 32 (w % 4) .. and every other 32 columns
//   warps 14, 15: none (registers are split by groups of four warps)
//
// CG = 2: a pair of SMs works on one 256 x BN tile (each CTA 128 rows of A and half of B's rows); CG = 1: one
// SM on 128 x BN.  BN and the pipeline's depth are run-time parameters: the launcher picks them by size.
//
// SPLIT: few tiles and a long K (one token's product with a large weight).  A cluster of CTAs shares one tile, each over a
// slice of K; all but the first send their float sums to the first one's shared memory, which adds them in
// order (16 x 4096 x 4096: 12.5 us unsplit, 10.4 us on clusters of four with eight K blocks a CTA; 128 x 1024 x 8192:
// 21.9 and 16.1 us).
//
// Edges: TMA fills what lies outside a matrix with zeros (scales outside are 1), and the stores are
// limited to C.  Every wait is bounded.
#include "gemm_common.cuh"
#include "../../include/fax_ops.h"

namespace {

using namespace tc;

constexpr int BM = 128;            // rows of A per CTA
constexpr int MAX_BN = 256;
constexpr int BK = FAX_FP8_BLOCK;  // bytes = elements
constexpr int GROUP = 4;           // K blocks per scale word
// Float outputs: the tensor core cuts off what falls below its accumulator's last digit, a bias that grows with the
// number of MMAs (2.4e-6 of the result's norm at K = 5000, where float32 sums are off by 4e-7), so the sums of
// 512 k are handed over and added in registers (128 sums a lane at 256 columns, for which the other warps
// give up registers).  A bf16 output is rounded far more coarsely: one sum over all of K.
constexpr int SEGMENT = 4;         // K blocks
constexpr int SUM_CHUNKS = MAX_BN / 64;
static_assert(SEGMENT % GROUP == 0, "scales are grouped by four blocks within a segment");
constexpr int NUM_EPI_WARPS = 8;
constexpr int NUM_THREADS = 512;
// 128 registers a thread at launch; 256 x 64 + 256 x 192 = 512 x 128
constexpr int REGS_OTHER = 64, REGS_SUMS = 192;
static_assert(256 * REGS_OTHER + 256 * REGS_SUMS <= NUM_THREADS * 128, "register split");
constexpr int SPLIT_CHUNKS = 2;    // SPLIT: tiles of 128 columns at most
constexpr int TEAM = 64;           // threads of a scale team
constexpr int MAX_STAGES = 12;
constexpr int SC_SLOTS = 4;        // groups of scales in flight
constexpr int SC_A_BYTES = 512, SC_B_BYTES = 1024, SC_BYTES = SC_A_BYTES + SC_B_BYTES;
constexpr int BAR_BYTES = 512;
constexpr int SMEM_MAX = 227 * 1024;
constexpr int TMEM_SCALE_COLS = 32;                  // two sets of 4 (A) + 8 (B) columns
static_assert(8 * (2 * MAX_STAGES + 4 + 2 * SC_SLOTS) + 8 <= BAR_BYTES, "barrier area");

struct Fp8Params {
  int M, N, K;
  uint32_t a_fmt, b_fmt;
  const float* sa; long long ldsa;
  const float* sb; long long ldsb; int sb_shift;                    // 7: one scale per 128 rows of B
  void* C; long long ldc; int c_f32, accumulate;
  int bulk;                                                         // C can be described by a tensor map
  const bf16* bias;
  int bn, stages, tmem_cols, acc1, scale_col;                       // tile width, pipeline depth, tensor-memory columns
  int tiles_m, tiles_n, group_m, group_along_n;
  int splits, kb_per, rows_q;                                       // SPLIT: CTAs per tile, K blocks of each, groups of 32 rows in a tile
  int32_t* status;
};

__device__ __forceinline__ uint32_t cluster_ctarank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The same shared-memory offset in the even CTA of the pair, as a shared::cluster address.
__device__ __forceinline__ uint32_t leader_addr(uint32_t a) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(0u));
  return r;
}
template <int CG>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1) {
  if (CG == 1)
    tma_load_2d(dst, map, bar, c0, c1);
  else
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
// Arrivals on a barrier of the even CTA.  Relaxed: what it orders (tensor-memory reads) has been completed;
// release: what the warp has written to shared memory (and fenced for the asynchronous proxy) is seen first.
template <int CG>
__device__ __forceinline__ void arrive_leader_relaxed(uint32_t bar) {
  if (CG == 1) mbar_arrive_relaxed(bar);
  else asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(leader_addr(bar)) : "memory");
}
template <int CG>
__device__ __forceinline__ void arrive_leader(uint32_t bar) {
  if (CG == 1) mbar_arrive(bar);
  else asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(leader_addr(bar)) : "memory");
}
template <int CG>
__device__ __forceinline__ void commit(uint32_t bar) {
  if (CG == 1)
    tc_commit(bar);
  else
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)3) : "memory");
}
// Bounded wait that also orders the other CTA's writes (acquire at cluster scope).
__device__ __forceinline__ bool mbar_wait_cluster(uint32_t bar, uint32_t parity, volatile int* abort_flag, int32_t* status, int code) {
  auto test = [&]() {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
  };
  if (test()) return true;
  const long long t0 = clock64();
  int spins = 0;
  while (!test()) {
    if ((++spins & 255) == 0) {
      if (*abort_flag) return false;
      if (clock64() - t0 > WAIT_CYCLES) {
        *abort_flag = 1;
        if (atomicCAS(status, 0, 1) == 0) status[1] = code;
        return false;
      }
    }
  }
  return true;
}
template <int CG>
__device__ __forceinline__ void mma_scaled(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
  if (CG == 1)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate) : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate) : "memory");
}
// 128 scale words (32 rows of 16 bytes in shared memory) to four columns of tensor memory, in each lane quarter.
template <int CG>
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint64_t desc) {
  if (CG == 1) asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
  else asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
// Descriptor of those 32 rows: no swizzle, groups of eight rows 128 bytes apart.
__device__ __forceinline__ uint64_t scale_desc(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFF) >> 4) | ((uint64_t)(128u >> 4) << 32) | ((uint64_t)1 << 46);
}

// A warp's 32 x 32 sums (a row a lane) of rows row0 .. and columns col .., to C, through the warp's staging buffer.
// Where a tensor map can describe C, one bulk store (or, for a product that is added, one bulk reduction at L2: nothing
// waits for C) takes the buffer, swizzled as the map says, and cuts it off at C's edges (float 4096 x 4096 x 4096: 78 us,
// 81 us by rows; bf16 4096 x 4096 x 128: 11 and 18 us).  Other pitches: the lanes write along a row.
constexpr int STG_BYTES = 5120;        // per warp: 32 x 33 floats, or the 4096 bytes of a swizzled box; a multiple of 1024
__device__ __forceinline__ void store_chunk(const Fp8Params& p, const CUtensorMap* mc, const uint32_t (&r)[32], long long row0, int col, float* stg,
                                            uint32_t stg_addr, int lane) {
  if (col >= p.N || row0 >= p.M) return;
  const float bias = p.bias && col + lane < p.N ? __bfloat162float(p.bias[col + lane]) : 0.f;
  if (p.bulk) {
    float v[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
    if (p.bias) {
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] += __shfl_sync(0xffffffffu, bias, j);
    }
    if (lane == 0) bulk_wait_read_all();                             // the previous chunk has left the buffer
    __syncwarp();
    if (p.c_f32) {
#pragma unroll
      for (int u = 0; u < 8; ++u)
        st_shared_v4(stg_addr + epi_sw128(lane, u), __float_as_uint(v[4 * u]), __float_as_uint(v[4 * u + 1]), __float_as_uint(v[4 * u + 2]),
                     __float_as_uint(v[4 * u + 3]));
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u) {                                  // 64-byte rows, 64-byte swizzle
        uint32_t h[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const __nv_bfloat162 x = __floats2bfloat162_rn(v[8 * u + 2 * e], v[8 * u + 2 * e + 1]);
          h[e] = *reinterpret_cast<const uint32_t*>(&x);
        }
        st_shared_v4(stg_addr + (uint32_t)(lane * 64 + ((u ^ ((lane >> 1) & 3)) << 4)), h[0], h[1], h[2], h[3]);
      }
    }
    fence_proxy_async();
    __syncwarp();
    if (lane == 0) {
      if (p.accumulate) tma_reduce_add_2d(mc, stg_addr, col, (int)row0);
      else tma_store_2d(mc, stg_addr, col, (int)row0);
      bulk_commit_group();
    }
    return;
  }
  __syncwarp();                                                      // the previous chunk has been read
#pragma unroll
  for (int j = 0; j < 32; ++j) stg[lane * 33 + j] = __uint_as_float(r[j]);
  __syncwarp();
  const int rows = (int)(p.M - row0 < 32 ? p.M - row0 : 32);
  if (col + lane < p.N) {
    // Eight rows at a time: their words leave shared memory together.  A product that is added is added at L2 too, one
    // addition an element (1891 x 7069 x 1283: 37 us; 65 us where each lane read C, added and wrote; with N = 7072,
    // through the tensor map, 36 us).
    auto each = [&](auto put) {
      const float* src = stg + lane;
      for (int i0 = 0; i0 < rows; i0 += 8, src += 8 * 33) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = src[i * 33];
        if (rows - i0 >= 8) {
#pragma unroll
          for (int i = 0; i < 8; ++i) put(v[i] + bias);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (i0 + i < rows) put(v[i] + bias);
        }
      }
    };
    if (p.c_f32) {
      float* o = (float*)p.C + row0 * p.ldc + col + lane;
      if (p.accumulate) each([&](float x) { atomicAdd(o, x); o += p.ldc; });
      else each([&](float x) { *o = x; o += p.ldc; });
    } else {
      bf16* o = (bf16*)p.C + row0 * p.ldc + col + lane;
      each([&](float x) { *o = __float2bfloat16_rn(x); o += p.ldc; });
    }
  }
}

// Words to the same place of the first CTA of the cluster.
__device__ __forceinline__ void st_cluster(uint32_t addr, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

template <int CG, bool SUMS, bool SPLIT>
__global__ void __launch_bounds__(NUM_THREADS, 1)
fp8_gemm_kernel(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_b, const __grid_constant__ CUtensorMap tmap_c,
                const __grid_constant__ Fp8Params p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t tiles_base = (raw + 1023u) & ~1023u;
  uint8_t* gen_base = smem_raw + (tiles_base - raw);
  const uint32_t b_bytes = (uint32_t)(p.bn / CG) * BK, stage_bytes = BM * BK + b_bytes;
  const int stages = p.stages;
  const uint32_t sc_off = (uint32_t)stages * stage_bytes, bar_off = sc_off + SC_SLOTS * SC_BYTES + NUM_EPI_WARPS * STG_BYTES;
  const uint32_t bars = tiles_base + bar_off;
  auto full_bar = [&](int s) { return bars + 8u * s; };                              // used in the even CTA
  auto empty_bar = [&](int s) { return bars + 8u * (MAX_STAGES + s); };              // one per CTA
  auto tfull_bar = [&](int a) { return bars + 8u * (2 * MAX_STAGES + a); };          // one per CTA
  auto tempty_bar = [&](int a) { return bars + 8u * (2 * MAX_STAGES + 2 + a); };     // used in the even CTA
  auto sfull_bar = [&](int s) { return bars + 8u * (2 * MAX_STAGES + 4 + s); };      // used in the even CTA
  auto sempty_bar = [&](int s) { return bars + 8u * (2 * MAX_STAGES + 4 + SC_SLOTS + s); };   // one per CTA
  volatile uint32_t* tmem_base_slot = (volatile uint32_t*)(gen_base + bar_off + 8 * (2 * MAX_STAGES + 4 + 2 * SC_SLOTS));
  volatile int* abort_flag = (volatile int*)(tmem_base_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CG == 1 ? 0u : cluster_ctarank();
  const bool leader = (rank == 0);
  static_assert(!SPLIT || (CG == 1 && SUMS), "slices of K are joined as float sums");
  const int slice = SPLIT ? (int)cluster_ctarank() : 0;
  const int num_tiles = p.tiles_m * p.tiles_n;
  const int unit = SPLIT ? blockIdx.x / p.splits : blockIdx.x / CG, num_units = SPLIT ? num_tiles : gridDim.x / CG;
  const int kb_all = (p.K + BK - 1) / BK;
  const int kb_off = SPLIT ? slice * p.kb_per : 0, kb_total = SPLIT ? min(p.kb_per, kb_all - kb_off) : kb_all;      // this CTA's K blocks
  const int seg_len = SUMS ? SEGMENT : kb_total, segments = (kb_total + seg_len - 1) / seg_len;

  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(tfull_bar(a), 1); mbar_init(tempty_bar(a), CG * NUM_EPI_WARPS); }
    for (int s = 0; s < SC_SLOTS; ++s) { mbar_init(sfull_bar(s), CG * (TEAM / 32)); mbar_init(sempty_bar(s), 1); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_a) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_b) : "memory");
    if (p.bulk) asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_c) : "memory");
  }
  if (warp == 1) {
    if (CG == 1) {
      tmem_alloc(smem_u32((const void*)tmem_base_slot), (uint32_t)p.tmem_cols);
    } else {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                   ::"r"(smem_u32((const void*)tmem_base_slot)), "r"((uint32_t)p.tmem_cols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  __syncthreads();
  if (CG == 2 || SPLIT) cluster_sync_all();   // the other CTAs run, their barriers exist
  tc_fence_after();
  const uint32_t tmem_base = *tmem_base_slot;
  fax_grid_dependency_wait();        // global memory only from here

  if (warp < 4 || warp >= 12) {
  if (SUMS) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_OTHER));
  if (warp == 0) {
    // ---------------- TMA producer ----------------
    if (lane == 0) {
      int stage = 0; uint32_t phase = 0;
      bool ok = true;
      for (int tile = unit; tile < num_tiles && ok; tile += num_units) {
        int tm, tn;
        tile_coords(tile, p.tiles_m, p.tiles_n, p.group_m, p.group_along_n, tm, tn);
        const int m0 = tm * CG * BM + (int)rank * BM, n0 = tn * p.bn + (int)rank * (p.bn / CG);
        for (int kb = 0; kb < kb_total; ++kb) {
          if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag, p.status, 501)) { ok = false; break; }
          const uint32_t a_dst = tiles_base + (uint32_t)stage * stage_bytes;
          const uint32_t fbar = CG == 1 ? full_bar(stage) : leader_addr(full_bar(stage));
          if (leader) mbar_expect_tx(full_bar(stage), CG * stage_bytes);             // both CTAs' bytes
          tma_load<CG>(a_dst, &tmap_a, fbar, (kb_off + kb) * BK, m0);
          tma_load<CG>(a_dst + BM * BK, &tmap_b, fbar, (kb_off + kb) * BK, n0);
          if (++stage == stages) { stage = 0; phase ^= 1u; }
        }
      }
      if (!ok) { const long long t0 = clock64(); while (clock64() - t0 < 2000000LL) { } }     // copies in flight land first
    }
  } else if (warp == 1) {
    // ---------------- scale copies and MMA issue (even CTA) ----------------
    if (leader && lane == 0) {
      // D = f32, the two formats, both K-major, N, ue8m0 scales, M over the unit; the scale bytes are named per block
      const uint32_t idesc0 = (p.a_fmt << 7) | (p.b_fmt << 10) | ((uint32_t)(p.bn >> 3) << 17) | (1u << 23) | ((uint32_t)((CG * BM) >> 4) << 24);
      // operand descriptors: 128-byte swizzle, eight-row groups 1024 bytes apart; the low word holds the address
      const uint32_t desc_lo0 = (uint32_t)smem_desc(tiles_base, 16u, 1024u), desc_hi = (uint32_t)(smem_desc(tiles_base, 16u, 1024u) >> 32);
      auto desc_word = [&](uint32_t lo) { return ((uint64_t)desc_hi << 32) | lo; };
      const bool overlap = p.acc1 < p.bn;      // the two accumulators share columns
      int stage = 0; uint32_t phase = 0;
      int group = 0;                           // groups of four K blocks, over all tiles
      const int num_groups = unit < num_tiles ? ((num_tiles - unit + num_units - 1) / num_units) * ((kb_total + GROUP - 1) / GROUP) : 0;
      auto scale_cols = [&](int g) { return tmem_base + (uint32_t)p.scale_col + (uint32_t)(g & 1) * 16u; };
      // copies the scales of group g to tensor memory, once the MMAs of group g - 2 have read what they replace
      auto scales_of = [&](int g) {
        const int slot = g & (SC_SLOTS - 1), old = g - 2;
        if (old >= 0 && !mbar_wait(sempty_bar(old & (SC_SLOTS - 1)), (uint32_t)(old / SC_SLOTS) & 1u, abort_flag, p.status, 507)) return false;
        if (!mbar_wait_cluster(sfull_bar(slot), (uint32_t)(g / SC_SLOTS) & 1u, abort_flag, p.status, 505)) return false;
        tc_fence_after();
        const uint32_t src = tiles_base + sc_off + (uint32_t)slot * SC_BYTES, t = scale_cols(g);
        copy_scales<CG>(t, scale_desc(src));
        copy_scales<CG>(t + 8u, scale_desc(src + SC_A_BYTES));
        if (p.bn > 128) copy_scales<CG>(t + 12u, scale_desc(src + SC_A_BYTES + 512u));
        return true;
      };
      bool ready = false;                      // the stage at hand has been seen full
      int j = 0;                               // accumulators handed over
      bool ok = true;
      for (int tile = unit; tile < num_tiles && ok; tile += num_units) {
        for (int seg = 0; seg < segments && ok; ++seg, ++j) {
          const int acc = j & 1;
          // the accumulator before the last has been read; where the two share columns, the last one's shared ones too
          if (!overlap) { if (!mbar_wait(tempty_bar(acc), (uint32_t)((j >> 1) & 1) ^ 1u, abort_flag, p.status, 502)) { ok = false; break; } }
          else if (j > 0) { if (!mbar_wait(tempty_bar(acc ^ 1), (uint32_t)((j - 1) >> 1) & 1u, abort_flag, p.status, 502)) { ok = false; break; } }
          tc_fence_after();
          const uint32_t d_tmem = tmem_base + (acc ? (uint32_t)p.acc1 : 0u);
          const int first = seg * seg_len, end = min(kb_total, first + seg_len);
          for (int kb0 = first; kb0 < end && ok; kb0 += GROUP, ++group) {
            if (group == 0 && !scales_of(0)) { ok = false; break; }
            const uint32_t sa_t = scale_cols(group), sb_t = sa_t + 8u;
#pragma unroll
            for (int b = 0; b < GROUP; ++b) {
              if (kb0 + b >= end) break;
              if (!ready && !mbar_wait(full_bar(stage), phase, abort_flag, p.status, 503)) { ok = false; break; }
              tc_fence_after();
              const uint32_t idesc = idesc0 + (uint32_t)b * ((1u << 4) | (1u << 29));
              const uint32_t a_lo = desc_lo0 + (uint32_t)stage * (stage_bytes >> 4), b_lo = a_lo + (BM * BK >> 4);
              const uint32_t ebar = empty_bar(stage);
              if (++stage == stages) { stage = 0; phase ^= 1u; }
              ready = mbar_try_wait(full_bar(stage), phase);         // the next stage is looked at while this one is issued
#pragma unroll
              for (int k = 0; k < BK / 32; ++k)                      // 32 k = two 16-byte units on
                mma_scaled<CG>(d_tmem, desc_word(a_lo + 2u * k), desc_word(b_lo + 2u * k), idesc, sa_t, sb_t, ((kb0 - first) | b | k) ? 1u : 0u);
              commit<CG>(ebar);                    // frees this stage (in both CTAs)
              // the next group's scales, under the MMAs of this one
              if (b == 0 && group + 1 < num_groups && !scales_of(group + 1)) { ok = false; break; }
            }
            commit<CG>(sempty_bar(group & (SC_SLOTS - 1)));
          }
          if (!ok) break;
          commit<CG>(tfull_bar(acc));              // accumulator complete (both halves)
        }
      }
    }
  } else if (warp < 14) {
    // ---------------- scales ----------------
    const int team = warp < 4 ? 0 : 1, t = threadIdx.x & (TEAM - 1);
    const int rows_b = (p.bn + TEAM - 1) / TEAM;                     // of B per thread, 1 .. 4
    const int groups_k = (kb_total + GROUP - 1) / GROUP;
    int group = 0;
    bool ok = true;
    for (int tile = unit; tile < num_tiles && ok; tile += num_units) {
      int tm, tn;
      tile_coords(tile, p.tiles_m, p.tiles_n, p.group_m, p.group_along_n, tm, tn);
      const int m0 = tm * CG * BM + (int)rank * BM, n0 = tn * p.bn;
      for (int g = 0; g < groups_k; ++g, ++group) {
        if ((group & 1) != team) continue;
        // exponent bytes of four K blocks; 127 (a scale of 1) outside the matrices.  Every load is issued, from a
        // place inside, so that none waits for another
        uint32_t wa[BM / TEAM], wb[MAX_BN / TEAM];
        long long at[GROUP];
#pragma unroll
        for (int b = 0; b < GROUP; ++b) at[b] = kb_off + min(g * GROUP + b, kb_total - 1);
        float fa[BM / TEAM][GROUP], fb[MAX_BN / TEAM][GROUP];
#pragma unroll
        for (int i = 0; i < BM / TEAM; ++i)
#pragma unroll
          for (int b = 0; b < GROUP; ++b) fa[i][b] = __ldg(p.sa + at[b] * p.ldsa + min(m0 + t + TEAM * i, p.M - 1));
#pragma unroll
        for (int i = 0; i < MAX_BN / TEAM; ++i)
          if (i < rows_b) {
#pragma unroll
            for (int b = 0; b < GROUP; ++b) fb[i][b] = __ldg(p.sb + at[b] * p.ldsb + (min(n0 + t + TEAM * i, p.N - 1) >> p.sb_shift));
          }
        auto word = [](const float (&f)[GROUP], bool in) {
          uint32_t w = 0u;
#pragma unroll
          for (int b = 0; b < GROUP; ++b) w |= ((__float_as_uint(f[b]) >> 23) & 0xffu) << (8 * b);
          return in ? w : 0x7f7f7f7fu;
        };
#pragma unroll
        for (int i = 0; i < BM / TEAM; ++i) wa[i] = word(fa[i], m0 + t + TEAM * i < p.M);
#pragma unroll
        for (int i = 0; i < MAX_BN / TEAM; ++i) wb[i] = word(fb[i], n0 + t + TEAM * i < p.N);
        const int slot = group & (SC_SLOTS - 1);
        if (!mbar_wait(sempty_bar(slot), ((uint32_t)(group / SC_SLOTS) & 1u) ^ 1u, abort_flag, p.status, 506)) { ok = false; break; }
        uint8_t* dst = gen_base + sc_off + slot * SC_BYTES;
        auto place = [](int r) { return (r >> 7) * 512 + (r & 31) * 16 + ((r >> 5) & 3) * 4; };
#pragma unroll
        for (int i = 0; i < BM / TEAM; ++i) *reinterpret_cast<uint32_t*>(dst + place(t + TEAM * i)) = wa[i];
#pragma unroll
        for (int i = 0; i < MAX_BN / TEAM; ++i)
          if (i < rows_b) *reinterpret_cast<uint32_t*>(dst + SC_A_BYTES + place(t + TEAM * i)) = wb[i];
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) arrive_leader<CG>(sfull_bar(slot));
      }
    }
  }
  if (SPLIT) { __syncwarp(); cluster_sync_all(); }                   // the row warps' exchange below
  } else {
    // ---------------- epilogue: this CTA's 128 rows of the tile ----------------
    if (SUMS) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_SUMS));
    const int q = warp & 3, half = (warp - 4) >> 2;
    const uint32_t stg_off = sc_off + SC_SLOTS * SC_BYTES + (uint32_t)(warp - 4) * STG_BYTES;
    float* stg = reinterpret_cast<float*>(gen_base + stg_off);
    const uint32_t stg_addr = tiles_base + stg_off;
    const bool overlap = p.acc1 < p.bn;
    const int chunks = (p.bn / 32 - half + 1) / 2;                   // this warp's 32-column chunks: half, half + 2, ...
    int j = 0;
    bool ok = true;
    for (int tile = unit; tile < num_tiles && ok; tile += num_units) {
      int tm, tn;
      tile_coords(tile, p.tiles_m, p.tiles_n, p.group_m, p.group_along_n, tm, tn);
      const long long row0 = (long long)tm * CG * BM + (int)rank * BM + 32 * q;
      const int n0 = tn * p.bn;
      uint32_t sum[SUMS ? SUM_CHUNKS : 1][32];
      if (SUMS) {
#pragma unroll
        for (int i = 0; i < SUM_CHUNKS; ++i)
#pragma unroll
          for (int e = 0; e < 32; ++e) sum[SUMS ? i : 0][e] = 0u;
      }
      for (int seg = 0; seg < segments; ++seg, ++j) {
        const int acc = j & 1;
        if (!mbar_wait_warp(tfull_bar(acc), (uint32_t)(j >> 1) & 1u, abort_flag, p.status, 504)) { ok = false; break; }
        tc_fence_after();
        const uint32_t t = tmem_base + ((uint32_t)(32 * q) << 16) + (acc ? (uint32_t)p.acc1 : 0u);
        auto release = [&]() {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_leader_relaxed<CG>(tempty_bar(acc));
        };
        if (chunks == 0) release();
        // where the accumulators share columns (the first one's last chunk, the second one's first), those are read first
        if (SUMS) {
          auto add = [&](int i, bool last) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint32_t r[16];
              tc_ld16(t + 32 * (half + 2 * i) + 16 * h, r);
              tc_wait_ld();
              if (h == 1 && last) release();
#pragma unroll
              for (int e = 0; e < 16; ++e)
                sum[SUMS ? i : 0][16 * h + e] = __float_as_uint(__uint_as_float(sum[SUMS ? i : 0][16 * h + e]) + __uint_as_float(r[e]));
            }
          };
          if (acc) {
#pragma unroll
            for (int i = 0; i < SUM_CHUNKS; ++i)
              if (i < chunks) add(i, overlap ? i == 0 : i == chunks - 1);
          } else {
#pragma unroll
            for (int i = SUM_CHUNKS - 1; i >= 0; --i)
              if (i < chunks) add(i, overlap ? i == chunks - 1 : i == 0);
          }
        } else {
          for (int i = 0; i < chunks; ++i) {
            const int c = 32 * (half + 2 * (acc ? i : chunks - 1 - i));
            uint32_t r[32];
            tc_ld32(t + c, r);
            tc_wait_ld();
            if (i == (overlap ? 0 : chunks - 1)) release();
            store_chunk(p, &tmap_c, r, row0, n0 + c, stg, stg_addr, lane);
          }
        }
      }
      if (SPLIT) {
        // a unit has one tile: every warp passes this exchange once.  Slot of (slice, row group, half, chunk): 32 columns x 32 rows
        const uint32_t recv = tiles_base + bar_off + BAR_BYTES;
        auto slot = [&](int sl, int i) { return (uint32_t)((((sl - 1) * p.rows_q + q) * 2 + half) * chunks + i) * 4096u + (uint32_t)lane * 4u; };
        if (slice != 0 && q < p.rows_q) {
#pragma unroll
          for (int i = 0; i < SPLIT_CHUNKS; ++i)
            if (i < chunks) {
              const uint32_t dst = leader_addr(recv + slot(slice, i));
#pragma unroll
              for (int e = 0; e < 32; ++e) st_cluster(dst + 128u * e, sum[SUMS ? i : 0][e]);
            }
        }
        __syncwarp();
        cluster_sync_all();                        // release of the sums, acquire by the first CTA
        if (slice == 0 && q < p.rows_q) {
          const uint8_t* src = gen_base + bar_off + BAR_BYTES;
#pragma unroll
          for (int i = 0; i < SPLIT_CHUNKS; ++i)
            if (i < chunks)
              for (int sl = 1; sl < p.splits; ++sl) {
                const float* f = reinterpret_cast<const float*>(src + slot(sl, i));
#pragma unroll
                for (int e = 0; e < 32; ++e) sum[SUMS ? i : 0][e] = __float_as_uint(__uint_as_float(sum[SUMS ? i : 0][e]) + f[32 * e]);
              }
        }
      }
      if (SUMS && ok && slice == 0) {
#pragma unroll
        for (int i = 0; i < SUM_CHUNKS; ++i)
          if (i < chunks) store_chunk(p, &tmap_c, sum[SUMS ? i : 0], row0, n0 + 32 * (half + 2 * i), stg, stg_addr, lane);
      }
    }
    if (p.bulk && lane == 0) bulk_wait_all();                        // the stores are complete
  }

  tc_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync_all();   // neither CTA leaves (or frees tensor memory) while the other may still signal it
  if (warp == 1) {
    tc_fence_after();
    if (CG == 1) tmem_dealloc(tmem_base, (uint32_t)p.tmem_cols);
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)p.tmem_cols) : "memory");
  }
}

bool make_map_u8(fax_ctx* ctx, CUtensorMap* map, const void* base, uint64_t inner, uint64_t outer, uint64_t ld, uint32_t box_outer) {
  cuuint64_t dims[2] = {inner, outer};
  cuuint64_t strides[1] = {ld};
  cuuint32_t box[2] = {(cuuint32_t)BK, box_outer};
  cuuint32_t estr[2] = {1, 1};
  return ((EncodeTiledFn)ctx->encode_tiled)(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, (void*)base, dims, strides, box, estr,
                                            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// C in boxes of 32 x 32: rows of 128 bytes (float) or 64 bytes (bf16), swizzled over their own width.
bool make_map_c(fax_ctx* ctx, CUtensorMap* map, const void* base, uint64_t inner, uint64_t outer, uint64_t ld, bool f32) {
  if (f32) return make_map_f32(ctx, map, base, inner, outer, ld, 32, 32);
  cuuint64_t dims[2] = {inner, outer};
  cuuint64_t strides[1] = {ld * 2};
  cuuint32_t box[2] = {32, 32};
  cuuint32_t estr[2] = {1, 1};
  return ((EncodeTiledFn)ctx->encode_tiled)(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, (void*)base, dims, strides, box, estr,
                                            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B,
                                            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// fax_launch, with clusters of `cluster` CTAs.
template <int CG, bool SUMS, bool SPLIT>
fax_status launch(fax_ctx* ctx, int grid, int cluster, int smem, const CUtensorMap& ma, const CUtensorMap& mb, const CUtensorMap& mc, const Fp8Params& p) {
  static bool done[FAX_MAX_DEVICES] = {};
  FAX_TRY(fax_opt_in_shared_memory(ctx, fp8_gemm_kernel<CG, SUMS, SPLIT>, SMEM_MAX, done));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid); cfg.blockDim = dim3(NUM_THREADS); cfg.dynamicSmemBytes = smem; cfg.stream = ctx->stream;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = ctx->use_pdl ? 2 : 1;
  (void)cudaLaunchKernelEx(&cfg, fp8_gemm_kernel<CG, SUMS, SPLIT>, ma, mb, mc, p);      // errors surface in fax_after_launch
  return fax_after_launch(ctx);
}

// Shared memory beside the stages; `split_bytes`: the sums that the first CTA of a cluster receives.
constexpr int FIXED_SMEM = SC_SLOTS * SC_BYTES + 1024 + BAR_BYTES + NUM_EPI_WARPS * STG_BYTES;
int split_bytes(int splits, int M, int bn) { return (splits - 1) * (M < 128 ? (M + 31) / 32 : 4) * (bn / 32) * 4096; }

// What tile shapes are compared by, in microseconds: waves of tiles times (K blocks times the pace of one, plus the tile's
// end), the paces as measured with all SMs busy, with one sum over K and with sums of 512 k.  It orders the shapes and is no
// forecast of a call, which also pays for the launch, the first loads and the last stores (4096 x 1000 x 5000 added to float:
// 23.6 here, for pairs and single SMs alike, of which the first in the table is taken; 30 us measured in a graph).  A pair of SMs loads each operand byte for twice the work and runs best
// where there are tiles for all pairs; a narrower tile has about the pace of the 128-column one (the issue of
// its MMAs bounds it), so it pays only where it brings more SMs to work.  Where the tiles leave SMs idle, slices of K
// bring them in, for the price of the exchange.
struct TileChoice { int cg, bn, splits; };
TileChoice choose_tile(const fax_ctx* ctx, int M, int N, int K, bool sums) {
  struct Shape { int cg, bn; double pace, pace_sums, end; };
  static const Shape shapes[] = {{2, 256, 0.41, 0.54, 1.5}, {2, 192, 0.38, 0.45, 1.3}, {1, 256, 0.45, 0.56, 1.2}, {1, 128, 0.31, 0.40, 0.8}, {1, 64, 0.29, 0.36, 0.6}};
  constexpr double EXCHANGE = 1.5;
  const int kb = (K + BK - 1) / BK;
  TileChoice best = {1, 256, 1};
  double least = 1e30;
  for (const Shape& s : shapes) {
    if (s.cg == 2 && !ctx->use_2cta) continue;
    const double tiles = (double)((M + s.cg * BM - 1) / (s.cg * BM)) * ((N + s.bn - 1) / s.bn);
    const double waves = (double)(long long)((tiles + ctx->sm_count / s.cg - 1) / (ctx->sm_count / s.cg));
    const double pace = sums ? s.pace_sums : s.pace;
    const double t = waves * (kb * pace + s.end) + (s.cg == 2 ? 0.5 : 0.0);
    if (t < least) { least = t; best = {s.cg, s.bn, 1}; }
    if (s.cg != 1 || s.bn > 32 * 2 * SPLIT_CHUNKS) continue;
    for (int splits = 2; splits <= 8; splits *= 2) {
      const int per = (kb + splits - 1) / splits;
      if (per < 2 || (kb + per - 1) / per != splits || tiles * splits > ctx->sm_count) continue;
      if (SMEM_MAX - FIXED_SMEM - split_bytes(splits, M, s.bn) < 4 * (BM + s.bn) * BK) continue;
      const double ts = per * s.pace_sums + s.end + EXCHANGE;
      if (ts < least) { least = ts; best = {1, s.bn, splits}; }
    }
  }
  return best;
}
// A float output longer than one segment is summed in registers; otherwise one accumulator holds all of K.
TileChoice tile_for(const fax_ctx* ctx, int M, int N, int K, bool c_f32) { return choose_tile(ctx, M, N, K, c_f32 && K > SEGMENT * BK); }

fax_status check_sizes(int M, int N, int K) {
  if (M <= 0 || N <= 0 || K <= 0) return FAX_ERR_INVALID_ARG;
  return M > 0x7ffffe00 || N > 0x7ffffe00 || K > 0x7ffffe00 ? FAX_ERR_UNSUPPORTED_SHAPE : FAX_OK;
}

}  // namespace

extern "C" fax_status fax_op_fp8_gemm_tile(const fax_ctx* ctx, int32_t M, int32_t N, int32_t K, int32_t c_f32, int32_t* sms, int32_t* columns, int32_t* slices) {
  if (!ctx || !sms || !columns || !slices) return FAX_ERR_INVALID_ARG;
  FAX_TRY(check_sizes(M, N, K));
  const TileChoice t = tile_for(ctx, M, N, K, c_f32 != 0);
  *sms = t.cg; *columns = t.bn; *slices = t.splits;
  return FAX_OK;
}

extern "C" fax_status fax_op_fp8_gemm(fax_ctx* ctx, const fax_fp8_gemm_desc* d) {
  if (!ctx || !d || !d->A || !d->B || !d->C || !d->a_scale || !d->b_scale) return FAX_ERR_INVALID_ARG;
  if (d->M <= 0 || d->N <= 0 || d->K <= 0) return FAX_ERR_INVALID_ARG;
  if ((d->a_format != FAX_FP8_E4M3 && d->a_format != FAX_FP8_E5M2) || (d->b_format != FAX_FP8_E4M3 && d->b_format != FAX_FP8_E5M2)) return FAX_ERR_INVALID_ARG;
  if (d->b_tile != 1 && d->b_tile != FAX_FP8_BLOCK) return FAX_ERR_INVALID_ARG;
  if (d->accumulate && !d->c_f32) return FAX_ERR_INVALID_ARG;
  if (d->lda < d->K || d->ldb < d->K || d->lda % 16 || d->ldb % 16 || d->ldc < d->N) return FAX_ERR_INVALID_ARG;
  if (d->a_scale_ld < d->M || d->b_scale_ld < (d->b_tile == 1 ? (int64_t)d->N : ((int64_t)d->N + 127) / 128)) return FAX_ERR_INVALID_ARG;
  const size_t es = d->c_f32 ? 4 : 2;
  if (!fax_aligned(d->A, 16) || !fax_aligned(d->B, 16) || !fax_aligned(d->C, es) || !fax_aligned(d->a_scale, 4) || !fax_aligned(d->b_scale, 4) ||
      !fax_aligned(d->bias, 2))
    return FAX_ERR_INVALID_ARG;
  if (d->lda >= (1LL << 40) || d->ldb >= (1LL << 40)) return FAX_ERR_UNSUPPORTED_SHAPE;        // the pitch a tensor map can hold
  FAX_TRY(check_sizes(d->M, d->N, d->K));
  const TileChoice t = tile_for(ctx, d->M, d->N, d->K, d->c_f32 != 0);
  const bool sums = t.splits > 1 || (d->c_f32 && d->K > SEGMENT * BK);
  CUtensorMap ma, mb;
  if (!make_map_u8(ctx, &ma, d->A, d->K, d->M, d->lda, BM) || !make_map_u8(ctx, &mb, d->B, d->K, d->N, d->ldb, (uint32_t)(t.bn / t.cg))) return FAX_ERR_INVALID_ARG;
  Fp8Params p;
  p.M = d->M; p.N = d->N; p.K = d->K;
  p.a_fmt = (uint32_t)d->a_format; p.b_fmt = (uint32_t)d->b_format;
  p.sa = d->a_scale; p.ldsa = d->a_scale_ld; p.sb = d->b_scale; p.ldsb = d->b_scale_ld; p.sb_shift = d->b_tile == 1 ? 0 : 7;
  p.C = d->C; p.ldc = d->ldc; p.c_f32 = d->c_f32 != 0; p.accumulate = d->accumulate != 0;
  // whole 16-byte units only: a bulk store does not cut off within one, it would write behind column N
  p.bulk = fax_aligned(d->C, 16) && ((size_t)d->ldc * es) % 16 == 0 && ((size_t)d->N * es) % 16 == 0 && d->ldc < (1LL << 36);
  CUtensorMap mc = ma;
  if (p.bulk && !make_map_c(ctx, &mc, d->C, d->N, d->M, d->ldc, d->c_f32 != 0)) return FAX_ERR_INVALID_ARG;
  p.bias = (const bf16*)d->bias;
  p.bn = t.bn;
  const int stage_bytes = BM * BK + t.bn / t.cg * BK, fixed = FIXED_SMEM + (t.splits > 1 ? split_bytes(t.splits, d->M, t.bn) : 0);
  p.stages = (SMEM_MAX - fixed) / stage_bytes;
  if (p.stages > MAX_STAGES) p.stages = MAX_STAGES;
  const int smem = p.stages * stage_bytes + fixed;
  p.splits = t.splits;
  p.kb_per = ((d->K + BK - 1) / BK + t.splits - 1) / t.splits;
  p.rows_q = d->M < 128 ? (d->M + 31) / 32 : 4;
  // two accumulators and the scales; at 256 columns the accumulators share the columns that the scales take
  p.tmem_cols = 64;
  while (p.tmem_cols < 2 * t.bn + TMEM_SCALE_COLS && p.tmem_cols < 512) p.tmem_cols *= 2;
  p.scale_col = p.tmem_cols - TMEM_SCALE_COLS;
  p.acc1 = t.bn < p.scale_col - t.bn ? t.bn : p.scale_col - t.bn;
  p.tiles_m = (int)(((int64_t)d->M + t.cg * BM - 1) / (t.cg * BM)); p.tiles_n = (int)(((int64_t)d->N + t.bn - 1) / t.bn);
  // tile order: as for the bf16 products, with one byte an element (8192 x 16384 x 4096, sustained: 462 us in groups of 8
  // row-tiles, 450 us with all of A's panels kept in L2)
  GemmParams order;
  order.M = p.tiles_m * t.cg * BM; order.N = p.tiles_n * t.bn; order.K = d->K / 2;
  order.group_m = 8; order.group_along_n = 0;
  if (ctx->gemm_l2_budget > 0 && d->K >= 2) gemm_choose_raster(order, t.cg * BM, t.bn, ctx->sm_count / t.cg, ctx->gemm_l2_budget);
  p.group_m = order.group_m; p.group_along_n = order.group_along_n;
  p.status = ctx->dev_status;
  if ((long long)p.tiles_m * p.tiles_n > 0x7fff0000LL) return FAX_ERR_UNSUPPORTED_SHAPE;
  FaxProfScope prof(ctx, KC_FP8_GEMM, 2.0 * d->M * (double)d->N * d->K, 0.0);
  const int tiles = p.tiles_m * p.tiles_n, max_units = ctx->sm_count / t.cg;
  const int units = tiles < max_units ? tiles : max_units;
  if (t.splits > 1) return launch<1, true, true>(ctx, tiles * t.splits, t.splits, smem, ma, mb, mc, p);
  if (t.cg == 2) return sums ? launch<2, true, false>(ctx, 2 * units, 2, smem, ma, mb, mc, p) : launch<2, false, false>(ctx, 2 * units, 2, smem, ma, mb, mc, p);
  return sums ? launch<1, true, false>(ctx, units, 1, smem, ma, mb, mc, p) : launch<1, false, false>(ctx, units, 1, smem, ma, mb, mc, p);
}
