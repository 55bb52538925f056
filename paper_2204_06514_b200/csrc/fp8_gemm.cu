// Product of two matrices in 8-bit floating point with a scale for each block of 128 along K:
//
//   C[m, n] = sum_b sa[b, m] sb[b, n] sum_{k in block b} A[m, k] B[n, k]   (+ bias[n])  (+ C[m, n])
//
// The tensor cores of two SMs work on one 256 x 256 tile (tcgen05.mma.cta_group::2, kind::f8f6f4).  A K
// block is 128 bytes a row, exactly one 128-byte-swizzled operand tile and one block of scales, so the
// pipeline runs block by block: TMA fills a stage, four MMAs (32 k each) multiply it into one of
// two accumulators in tensor memory, and the row warps add the accumulator, times its two scales, into
// float32 registers while the other one fills.  The scales differ from row to row and block to block,
// so they cannot be applied after the sum over all of K.
//
//   warp 0      : TMA producer (both CTAs; each loads its 128 rows of A and its half of B)
//   warp 1      : tensor-memory allocation (both CTAs), MMA issue (even CTA)
//   warps 2, 3  : none (they give their registers to the row warps)
//   warps 4..11 : 128 rows x 256 columns of the CTA: warp w owns 32 rows and 128 columns, 128 sums a lane
//
// Edges: TMA fills what lies outside a matrix with zeros, the scales of rows outside are taken as 0, and
// the stores are limited to C.  Every wait is bounded.
#include "gemm_common.cuh"
#include "../../include/fax_ops.h"

namespace {

using namespace tc;

constexpr int BM = 128;            // rows of A per CTA (256 per pair)
constexpr int BN = 256;            // columns per pair; each CTA stages 128 of B's rows
constexpr int BNH = 128;
constexpr int BK = FAX_FP8_BLOCK;  // bytes = elements
constexpr int NUM_EPI_WARPS = 8;
constexpr int NUM_THREADS = 32 * (4 + NUM_EPI_WARPS);
// 168 registers a thread at launch (65536 / 384); 128 x 40 + 256 x 232 = 384 x 168
constexpr int REGS_LOAD = 40, REGS_ROWS = 232;
static_assert(128 * REGS_LOAD + 256 * REGS_ROWS <= 384 * 168, "register split");
constexpr int A_BYTES = BM * BK, B_BYTES = BNH * BK, STAGE_BYTES = A_BYTES + B_BYTES;
constexpr int STAGES = 6;
constexpr int TMEM_COLS = 512;
constexpr int SCALE_BYTES = NUM_EPI_WARPS * 2 * 128 * 4;            // B's scales of a block, per warp, two blocks
constexpr int BAR_BYTES = 256;
constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + SCALE_BYTES + 1024 + BAR_BYTES;
static_assert(SMEM_BYTES <= 227 * 1024, "shared memory per CTA");
static_assert(8 * (2 * STAGES + 4) + 8 <= BAR_BYTES, "barrier area");

struct Fp8Params {
  int M, N, K;
  uint32_t a_fmt, b_fmt;
  const float* sa; long long ldsa;
  const float* sb; long long ldsb;
  void* C; long long ldc; int c_f32, accumulate, wide;              // wide: rows of C are 32-byte aligned
  const bf16* bias;
  int tiles_m, tiles_n, group_m, group_along_n;
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
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_commit_pair(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
               ::"r"(bar), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void tc_mma_fp8_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}

__device__ __forceinline__ uint64_t pack2(uint32_t lo, uint32_t hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) {
  uint32_t a, b;
  asm("mov.b64 {%0, %1}, %2;" : "=r"(a), "=r"(b) : "l"(v));
  lo = __uint_as_float(a); hi = __uint_as_float(b);
}
// Two float32 products or fused multiply-adds in one instruction.
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// 32 columns of the accumulator, scaled, into the sums.  s: sa twice (times sb where a block of B has one scale).
template <bool B_ROWS>
__device__ __forceinline__ void add_scaled(const uint32_t (&r)[32], uint64_t s, const ulonglong2* sb, uint64_t* sum) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (B_ROWS) {
      const ulonglong2 b = sb[j];
      sum[2 * j] = fma2(pack2(r[4 * j], r[4 * j + 1]), mul2(s, b.x), sum[2 * j]);
      sum[2 * j + 1] = fma2(pack2(r[4 * j + 2], r[4 * j + 3]), mul2(s, b.y), sum[2 * j + 1]);
    } else {
      sum[2 * j] = fma2(pack2(r[4 * j], r[4 * j + 1]), s, sum[2 * j]);
      sum[2 * j + 1] = fma2(pack2(r[4 * j + 2], r[4 * j + 3]), s, sum[2 * j + 1]);
    }
  }
}

// One lane's 128 sums of row `row`, columns col0 .. col0 + 127.
__device__ __forceinline__ void store_row(const Fp8Params& p, const uint64_t (&sum)[64], long long row, int col0) {
  float acc[128];
#pragma unroll
  for (int j = 0; j < 64; ++j) unpack2(sum[j], acc[2 * j], acc[2 * j + 1]);
  if (row >= p.M || col0 >= p.N) return;
  if (p.wide && col0 + 128 <= p.N) {
#pragma unroll
    for (int c = 0; c < 128; c += 16) {
      float v[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] = acc[c + j] + (p.bias ? __bfloat162float(p.bias[col0 + c + j]) : 0.f);
      if (p.c_f32) {
        float* o = (float*)p.C + row * p.ldc + col0 + c;
#pragma unroll
        for (int j8 = 0; j8 < 2; ++j8) {
          U8 u;
          if (p.accumulate) {
            const U8 old = ld_global_v8(o + 8 * j8);
#pragma unroll
            for (int e = 0; e < 8; ++e) u.w[e] = __float_as_uint(v[8 * j8 + e] + __uint_as_float(old.w[e]));
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) u.w[e] = __float_as_uint(v[8 * j8 + e]);
          }
          st_global_v8(o + 8 * j8, u);
        }
      } else {
        U8 u;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
          u.w[e] = *reinterpret_cast<const uint32_t*>(&h);
        }
        st_global_v8((bf16*)p.C + row * p.ldc + col0 + c, u);
      }
    }
    return;
  }
#pragma unroll
  for (int c = 0; c < 128; ++c) {
    if (col0 + c < p.N) {
      const float v = acc[c] + (p.bias ? __bfloat162float(p.bias[col0 + c]) : 0.f);
      if (p.c_f32) {
        float* o = (float*)p.C + row * p.ldc + col0 + c;
        *o = p.accumulate ? *o + v : v;
      } else {
        ((bf16*)p.C)[row * p.ldc + col0 + c] = __float2bfloat16_rn(v);
      }
    }
  }
}

template <bool B_ROWS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(NUM_THREADS, 1)
fp8_gemm_pair_kernel(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_b, const __grid_constant__ Fp8Params p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t tiles_base = (raw + 1023u) & ~1023u;
  uint8_t* gen_base = smem_raw + (tiles_base - raw);
  float* scales = reinterpret_cast<float*>(gen_base + STAGES * STAGE_BYTES);
  uint8_t* bar_mem = gen_base + STAGES * STAGE_BYTES + SCALE_BYTES;
  const uint32_t bars = tiles_base + STAGES * STAGE_BYTES + SCALE_BYTES;
  auto full_bar = [&](int s) { return bars + 8u * s; };                         // used in the even CTA
  auto empty_bar = [&](int s) { return bars + 8u * (STAGES + s); };             // one per CTA
  auto tfull_bar = [&](int a) { return bars + 8u * (2 * STAGES + a); };         // one per CTA
  auto tempty_bar = [&](int a) { return bars + 8u * (2 * STAGES + 2 + a); };    // used in the even CTA
  volatile uint32_t* tmem_base_slot = (volatile uint32_t*)(bar_mem + 8 * (2 * STAGES + 4));
  volatile int* abort_flag = (volatile int*)(bar_mem + 8 * (2 * STAGES + 4) + 4);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const bool leader = (rank == 0);
  const int pair = blockIdx.x >> 1, num_pairs = gridDim.x >> 1;
  const int num_tiles = p.tiles_m * p.tiles_n;
  const int kb_total = (p.K + BK - 1) / BK;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(tfull_bar(a), 1); mbar_init(tempty_bar(a), 2 * NUM_EPI_WARPS); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_a) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_b) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32((const void*)tmem_base_slot)), "r"((uint32_t)TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();            // both CTAs' barriers exist before either signals the other
  tc_fence_after();
  const uint32_t tmem_base = *tmem_base_slot;
  fax_grid_dependency_wait();    // global memory only from here

  if (warp < 4) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_LOAD));
  if (warp == 0) {
    // ---------------- TMA producer ----------------
    if (lane == 0) {
      int stage = 0; uint32_t phase = 0;
      bool ok = true;
      for (int tile = pair; tile < num_tiles && ok; tile += num_pairs) {
        int tm, tn;
        tile_coords(tile, p.tiles_m, p.tiles_n, p.group_m, p.group_along_n, tm, tn);
        const int m0 = tm * 2 * BM + (int)rank * BM, n0 = tn * BN + (int)rank * BNH;
        for (int kb = 0; kb < kb_total; ++kb) {
          if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag, p.status, 501)) { ok = false; break; }
          const uint32_t a_dst = tiles_base + stage * STAGE_BYTES;
          const uint32_t fbar = leader_addr(full_bar(stage));
          if (leader) mbar_expect_tx(full_bar(stage), 2 * STAGE_BYTES);       // both CTAs' bytes
          tma_load_2d_pair(a_dst, &tmap_a, fbar, kb * BK, m0);
          tma_load_2d_pair(a_dst + A_BYTES, &tmap_b, fbar, kb * BK, n0);
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
      }
      if (!ok) { const long long t0 = clock64(); while (clock64() - t0 < 2000000LL) { } }     // copies in flight land first
    }
  } else if (warp == 1) {
    // ---------------- MMA issuer (even CTA of the pair) ----------------
    if (leader && lane == 0) {
      // D = f32, the two formats, both operands K-major, N = 256, M = 256 over the pair
      const uint32_t idesc = (1u << 4) | (p.a_fmt << 7) | (p.b_fmt << 10) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)((2 * BM) >> 4) << 24);
      int stage = 0; uint32_t phase = 0;
      int acc = 0; uint32_t acc_phase = 0;
      bool ok = true;
      for (int tile = pair; tile < num_tiles && ok; tile += num_pairs) {
        for (int kb = 0; kb < kb_total; ++kb) {
          if (!mbar_wait(tempty_bar(acc), acc_phase ^ 1u, abort_flag, p.status, 502)) { ok = false; break; }
          if (!mbar_wait(full_bar(stage), phase, abort_flag, p.status, 503)) { ok = false; break; }
          tc_fence_after();
          const uint32_t a_src = tiles_base + stage * STAGE_BYTES, b_src = a_src + A_BYTES;
          const uint32_t d_tmem = tmem_base + (uint32_t)(acc * BN);
#pragma unroll
          for (int k = 0; k < BK / 32; ++k)
            tc_mma_fp8_pair(d_tmem, smem_desc(a_src + 32u * k, 16u, 1024u), smem_desc(b_src + 32u * k, 16u, 1024u), idesc, k ? 1u : 0u);
          tc_commit_pair(empty_bar(stage));      // frees this stage in both CTAs
          tc_commit_pair(tfull_bar(acc));        // this block's accumulator is complete, both halves
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
          if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
        }
      }
    }
  }
  } else {
    // ---------------- row warps ----------------
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_ROWS));
    const int q = warp & 3, half = (warp - 4) >> 2;
    float* my_scales = scales + (warp - 4) * 2 * 128;
    int acc = 0; uint32_t acc_phase = 0;
    bool ok = true;
    for (int tile = pair; tile < num_tiles && ok; tile += num_pairs) {
      int tm, tn;
      tile_coords(tile, p.tiles_m, p.tiles_n, p.group_m, p.group_along_n, tm, tn);
      const long long row = (long long)tm * 2 * BM + (int)rank * BM + 32 * q + lane;
      const int col0 = tn * BN + half * 128;
      const bool row_in = row < p.M;
      auto load_sa = [&](int kb) { return row_in ? __ldg(p.sa + (long long)kb * p.ldsa + row) : 0.f; };
      auto load_sb1 = [&](int kb) { return col0 < p.N ? __ldg(p.sb + (long long)kb * p.ldsb + (col0 >> 7)) : 0.f; };
      auto load_sb = [&](int kb, float (&b)[4]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = col0 + 32 * j + lane < p.N ? __ldg(p.sb + (long long)kb * p.ldsb + col0 + 32 * j + lane) : 0.f;
      };
      uint64_t sum[64];
#pragma unroll
      for (int j = 0; j < 64; ++j) sum[j] = 0ull;
      float sa_next = load_sa(0), sb_next = 0.f, sbv[4];
      if (B_ROWS) load_sb(0, sbv); else sb_next = load_sb1(0);
      for (int kb = 0; kb < kb_total; ++kb) {
        const float s = B_ROWS ? sa_next : sa_next * sb_next;
        float* buf = my_scales + (kb & 1) * 128;
        if (B_ROWS) {
#pragma unroll
          for (int j = 0; j < 4; ++j) buf[32 * j + lane] = sbv[j];
          __syncwarp();                          // the buffer of two blocks ago has been read by every lane before this one's turn
        }
        if (kb + 1 < kb_total) {
          sa_next = load_sa(kb + 1);
          if (B_ROWS) load_sb(kb + 1, sbv); else sb_next = load_sb1(kb + 1);
        }
        if (!mbar_wait_warp(tfull_bar(acc), acc_phase, abort_flag, p.status, 504)) { ok = false; break; }
        tc_fence_after();
        const uint32_t t = tmem_base + ((uint32_t)(32 * q) << 16) + (uint32_t)(acc * BN + half * 128);
        const uint64_t s2 = pack2(__float_as_uint(s), __float_as_uint(s));
        const ulonglong2* b2 = reinterpret_cast<const ulonglong2*>(buf);
        uint32_t ra[32], rb[32];
        tc_ld32(t, ra);
        tc_ld32(t + 32, rb);
        tc_wait_ld();
        add_scaled<B_ROWS>(ra, s2, b2, sum);
        tc_ld32(t + 64, ra);
        add_scaled<B_ROWS>(rb, s2, b2 + 8, sum + 16);
        tc_ld32(t + 96, rb);
        tc_wait_ld();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(leader_addr(tempty_bar(acc)));
        add_scaled<B_ROWS>(ra, s2, b2 + 16, sum + 32);
        add_scaled<B_ROWS>(rb, s2, b2 + 24, sum + 48);
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      }
      if (ok) store_row(p, sum, row, col0);
    }
  }

  tc_fence_before();
  __syncthreads();
  cluster_sync_all();            // neither CTA leaves (or frees tensor memory) while the other may still signal it
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)TMEM_COLS) : "memory");
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

}  // namespace

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
  if (d->M > 0x7fffff00 || d->N > 0x7fffff00 || d->K > 0x7fffff00) return FAX_ERR_UNSUPPORTED_SHAPE;
  CUtensorMap ma, mb;
  if (!make_map_u8(ctx, &ma, d->A, d->K, d->M, d->lda, BM) || !make_map_u8(ctx, &mb, d->B, d->K, d->N, d->ldb, BNH)) return FAX_ERR_INVALID_ARG;
  Fp8Params p;
  p.M = d->M; p.N = d->N; p.K = d->K;
  p.a_fmt = (uint32_t)d->a_format; p.b_fmt = (uint32_t)d->b_format;
  p.sa = d->a_scale; p.ldsa = d->a_scale_ld; p.sb = d->b_scale; p.ldsb = d->b_scale_ld;
  p.C = d->C; p.ldc = d->ldc; p.c_f32 = d->c_f32 != 0; p.accumulate = d->accumulate != 0;
  p.wide = fax_aligned(d->C, 32) && ((size_t)d->ldc * es) % 32 == 0;
  p.bias = (const bf16*)d->bias;
  p.tiles_m = (d->M + 2 * BM - 1) / (2 * BM); p.tiles_n = (d->N + BN - 1) / BN;
  p.group_m = 8; p.group_along_n = 0;
  p.status = ctx->dev_status;
  if ((long long)p.tiles_m * p.tiles_n > 0x7fff0000LL) return FAX_ERR_UNSUPPORTED_SHAPE;
  FaxProfScope prof(ctx, KC_FP8_GEMM, 2.0 * d->M * (double)d->N * d->K, 0.0);
  static bool done[2][FAX_MAX_DEVICES] = {};
  FAX_TRY(fax_opt_in_shared_memory(ctx, fp8_gemm_pair_kernel<false>, SMEM_BYTES, done[0]));
  FAX_TRY(fax_opt_in_shared_memory(ctx, fp8_gemm_pair_kernel<true>, SMEM_BYTES, done[1]));
  const int tiles = p.tiles_m * p.tiles_n, max_pairs = ctx->sm_count / 2;
  const int pairs = tiles < max_pairs ? tiles : max_pairs;
  if (d->b_tile == 1) fax_launch(ctx, fp8_gemm_pair_kernel<true>, dim3(2 * pairs), dim3(NUM_THREADS), SMEM_BYTES, ma, mb, p);
  else fax_launch(ctx, fp8_gemm_pair_kernel<false>, dim3(2 * pairs), dim3(NUM_THREADS), SMEM_BYTES, ma, mb, p);
  return fax_after_launch(ctx);
}
