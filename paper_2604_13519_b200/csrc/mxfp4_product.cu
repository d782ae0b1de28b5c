// y[m][n] = sum_k x[m][k] * W[n][k] with W in MXFP4.  The block-scaled form of the tensor cores' instruction (kind::mxf8f6f4) takes the
// weights' four-bit elements and scale bytes as they are, so a CTA only moves them.  (Widening them to bf16 in registers on the
// way into tensor memory, the first form of this kernel, took 1600 warp instructions for a block of 128 x 128 elements, more than
// the SM issues in the block's share of the memory's time: LM head of 151936 x 4096 at 32 rows 92 us.)
//
// The instruction's other operand has eight bits at most: the activations come as planes of e4m3 numbers with a scale byte per 32
// columns and plane, each plane holding what the ones before it left over (mx_planes8_kernel).  Planes are stacked along the
// instruction's N dimension, as the bf16 planes of gemm_tcgen05.cu are, and the epilogue adds their columns.
//
// Shared memory holds a block's elements in eight-bit containers: TMA puts them there from packed memory (16U4_ALIGN16B).  Scales go from
// shared into tensor memory (tcgen05.cp: 32 lanes x 16 bytes, repeated in all four lane quarters): word j of lane l = the four scales
// of row 32 j + l along a block's 128 columns.
//
// Two ways to deal the work out; which one a product takes depends on its tiles alone (128 features x a chunk of rows).
//
// kStream, for more tiles than CTAs fit: in k-blocks.  (tile, k-block) pairs in order, an equal run of them to each of two CTAs per SM, so
// that all SMs stream the same bytes whatever the matrix's shape and a launch has one start and one end.  A CTA walks its run from the
// end to the start.  A tile that it has without its last k-block (the first that it walks) it leaves as partial sums for the CTAs
// behind it; a tile that it has without its first k-block (its last) it finishes, adding the partial sums of the CTAs before it, in
// order of k.  Those were written at the start of their runs, so there is hardly a wait, and no CTA ever waits for one behind it.
// Two accumulators where the tensor memory holds them: the epilogue of one tile runs under the products of the next.
//
// Otherwise one tile to a CTA, or, where that leaves places empty, to a cluster of CTAs along K, whose sums meet through
// distributed shared memory: less of an exchange than through L2, which counts where a CTA has few k-blocks.
//
// Up to two rows, four or eight where a CTA has few blocks (mx_plan), CTAs that have a tile each make the planes themselves (kTile with
// kOwn): four more warps turn a stage's 128 columns into e4m3 on the way into shared memory, which saves a launch; for more rows a kernel
// ahead does it once for all CTAs (launch_mx_input).
//
// Roles: warp 0 = copies, warp 1 = tensor memory, scales and products, warps 2..5 = epilogue, warps 6.. = planes (kOwn).
// Every wait on a barrier or a flag is bounded; on expiry the CTA records an error word and leaves through the normal exit.  Waits that have
// no bounded form: tcgen05.alloc (an SM holds two of these CTAs by their shared memory, each with half of the tensor memory at most), the
// cluster barriers (every thread reaches them through bounded waits) and the dependency wait.
#include <cuda_fp16.h>

#include <algorithm>

#include "mxfp4.h"

namespace ts {

static constexpr int kProdMaxStages = 12;
static constexpr int kProdW = kMxTileN * kMxTileK;   // a block's elements in shared memory
static constexpr int kProdStaging = 2 * 8 * kMxTileN * 4;   // eight rows of sums, twice
static constexpr int kProdAcc = 224;                  // most columns of an accumulator: with 24 of scales (two stages) half of the tensor memory
static constexpr int kProdCtas = 2;                   // per SM

enum : int { kTile = 0, kStream = 1 };

struct __align__(16) ProdSmemCtl {
  uint64_t full[kProdMaxStages];
  uint64_t empty[kProdMaxStages];
  uint64_t acc_full[2];
  uint64_t acc_empty[2];
  uint32_t tmem_base;
  uint32_t abort_flag;
};

__device__ __forceinline__ void prod_error(const MxArgs &g, int code) { if (g.err) atomicExch(g.err, code); }

// D[tmem] (+)= (A x scales) * (B x scales), A e2m1 and B e4m3 in shared memory, K = 32
__device__ __forceinline__ void umma_mx(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                        uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(sfa), "r"(sfb)
      : "memory");
}
// Instruction descriptor: A e2m1, B e4m3, both K-major, scales ue8m0, D fp32, M x N; the scales' byte within their words is added (see
// mx_scale_byte)
__device__ __forceinline__ uint32_t umma_idesc_mx(uint32_t M, uint32_t N) {
  return (5u << 7) | (0u << 10) | ((N >> 3) << 17) | (1u << 23) | ((M >> 4) << 24);
}
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t i) { return (i << 4) | (i << 29); }

// 32 x 16 bytes of shared memory -> four columns of all four lane quarters
__device__ __forceinline__ void tmem_cp_scales(uint32_t taddr, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
// no swizzle, 8 rows x 16 bytes contiguous, the next 8 rows 128 bytes further on
__device__ __forceinline__ uint64_t scales_desc(uint32_t saddr) {
  return (uint64_t)((saddr >> 4) & 0x3FFF) | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}

// The run of CTA c out of G in units (tile x chunk) * n_kb + k-block
__device__ __forceinline__ long long prod_start(const MxArgs &g, int c, int G) { return (long long)c * g.units / G; }

// One tile of a run: item = tile * chunks + chunk, k-blocks [kb0, kb1)
struct ProdSeg {
  int item, kb0, kb1;
};
// the segment that ends at unit `hi` of a run that starts at `lo`
__device__ __forceinline__ ProdSeg prod_seg(const MxArgs &g, long long lo, long long hi) {
  ProdSeg t;
  t.item = (int)((hi - 1) / g.n_kb);
  const long long first = (long long)t.item * g.n_kb;
  t.kb0 = (int)(max(lo, first) - first);
  t.kb1 = (int)(hi - first);
  return t;
}

__device__ __forceinline__ int ld_acquire(const int *p) {
  int v;
  asm volatile("ld.acquire.gpu.global.b32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
// until the flag is set, or about two seconds
__device__ __forceinline__ bool wait_flag(const int *p) {
  uint64_t t0 = 0;
  for (uint32_t it = 0;; ++it) {
    if (ld_acquire(p)) return true;
    if ((it & 63u) == 63u) {
      const uint64_t now = global_timer_ns();
      if (t0 == 0) t0 = now;
      else if (now - t0 > 2000000000ull) return false;
    }
  }
}

// A block's scales into tensor memory (at `sf`) and its products.  A copy waits for nothing that was issued before it, so a stage of the
// ring has columns of its own for its scales: by the time that its barrier says full again, the products that read them are done.
__device__ __forceinline__ void prod_block(uint32_t sa, uint32_t sf, uint32_t d, uint32_t idesc, int act_bytes, int sb_words, bool accumulate) {
  const uint32_t sx = sa + kProdW, sfx = sx + act_bytes, sfw = sfx + 512 * sb_words;
  tmem_cp_scales(sf, scales_desc(sfw));
  tmem_cp_scales(sf + 4, scales_desc(sfx));
  if (sb_words > 1) tmem_cp_scales(sf + 8, scales_desc(sfx + 512));
  const uint64_t da = umma_desc_sw128(sa), db = umma_desc_sw128(sx);
#pragma unroll
  for (int kk = 0; kk < kMxTileK / 32; ++kk)   // 32 elements along K are 32 bytes of a row
    umma_mx(d, da + 2 * kk, db + 2 * kk, idesc | mx_scale_byte(kk), sf, sf + 4, accumulate || kk != 0);
}

// eight rows' sums of this thread's feature, planes added
__device__ __forceinline__ void prod_sums(const MxArgs &g, uint32_t taddr, float (&v)[8]) {
  constexpr int kMostPlanes = 5;
  uint32_t r[kMostPlanes][8];
#pragma unroll
  for (int p = 0; p < kMostPlanes; ++p)
    if (p < g.planes) tmem_ld8(taddr + p * g.Mc, r[p]);
  tmem_wait_ld();
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[0][i]);
#pragma unroll
  for (int p = 1; p < kMostPlanes; ++p)
    if (p < g.planes) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += __uint_as_float(r[p][i]);
    }
}

// kOwn: pairs of rows whose planes the CTA makes, 0: none
__host__ __device__ constexpr int own_warps(int own) { return own == 0 ? 0 : 4; }
template <int kOwn> __host__ __device__ constexpr int prod_threads() { return 192 + 32 * own_warps(kOwn); }

template <int EPI, int MODE, int kOwn, int TYPE>
__global__ void __launch_bounds__(prod_threads<kOwn>(), kProdCtas)
mx_product_kernel(const __grid_constant__ CUtensorMap tw, const MxArgs g) {
  extern __shared__ __align__(1024) uint8_t smem[];
  constexpr bool kRuns = MODE == kStream;
  const int ncols = g.planes * g.Mc, sb_words = (ncols + 127) / 128;   // (512 bytes of scales for 128 columns)
  const int act_bytes = ncols * kMxTileK, scale_bytes = 512 * (1 + sb_words);
  const int stage_bytes = kProdW + ((act_bytes + scale_bytes + 1023) & ~1023);
  uint8_t *staging = smem + (size_t)g.stages * stage_bytes;
  ProdSmemCtl *ctl = reinterpret_cast<ProdSmemCtl *>(staging + kProdStaging);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int cta = blockIdx.x, G = gridDim.x;
  const int split = blockIdx.y, C = kRuns ? 1 : (int)gridDim.y;   // the CTA's rank in its cluster, which spans the K slices of a tile
  const long long first = (long long)cta * g.n_kb;   // (one tile: cta is the item)
  const long long u0 = kRuns ? prod_start(g, cta, G) : first + (long long)split * g.n_kb / C;
  const long long u1 = kRuns ? prod_start(g, cta + 1, G) : first + (long long)(split + 1) * g.n_kb / C;
  const uint32_t acc_cols = (ncols + 31) & ~31u, n_acc = g.n_acc, scales_at = n_acc * acc_cols, set_cols = 4 + 4 * sb_words;
  uint32_t alloc_cols = 64;
  while (alloc_cols < scales_at + g.stages * set_cols) alloc_cols <<= 1;

  if (warp == 0 && lane == 0) {
    tma_prefetch_desc(&tw);
    for (int s = 0; s < g.stages; ++s) {
      mbar_init(smem_u32(&ctl->full[s]), kOwn ? 2 : 1);   // the copies (and a warp of planes)
      mbar_init(smem_u32(&ctl->empty[s]), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(smem_u32(&ctl->acc_full[b]), 1);
      mbar_init(smem_u32(&ctl->acc_empty[b]), 4);   // (epilogue warps)
    }
    ctl->abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&ctl->tmem_base), alloc_cols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = ctl->tmem_base, scales = tmem_base + scales_at;
  if (threadIdx.x == 0) stamp_min(g.stamp);
  // (placed after this CTA holds its resources, so a waiting dependent can never starve an earlier kernel)
  pdl_launch_dependents();

  if (warp == 0) {
    // ------------------------------------------------------------------ copies
    // The whole warp walks the loop; one elected lane issues a stage's copies (from a lane in a branch of its own each takes twice as
    // long, and this warp's time per stage is what bounds a CTA).
    // (weights that every chunk reads again stay in L2, us a call: 301 x 4096 x 12288 of fp16 64.4 -> 60.0, 57 x 5003 x 4100 of fp32 14.9 -> 14.0,
    // but 1024 x 24576 x 4096 224.7 -> 226.5)
    const uint64_t pol_w = g.chunks > 1 ? policy_evict_normal() : policy_evict_first(), pol_a = policy_evict_last();
    const int n = (int)(u1 - u0), x_block = act_bytes + 512 * sb_words;
    auto load_w = [&](uint32_t dst, uint32_t bar, int blk) {
      mbar_expect_tx(bar, kMxCodeBytes + (kOwn ? 512 : act_bytes + scale_bytes));   // (a copy that widens counts the bytes it reads)
      tma_load_3d(dst, &tw, 0, 0, blk, bar, pol_w);
      bulk_load(dst + kProdW + act_bytes + 512 * sb_words, g.w + (size_t)blk * kMxTileBytes + kMxCodeBytes, 512, bar, pol_w);
    };
    auto load_x = [&](uint32_t dst, uint32_t bar, int blk) { bulk_load(dst + kProdW, (const uint8_t *)g.x + (size_t)blk * x_block, x_block, bar, pol_a); };
    // weights do not depend on the previous kernel, unless it laid them out: they are on their way before the programmatic-dependency wait
    if (!g.early) pdl_wait();
    const int pre = min(g.stages, n);
    for (int pass = 0; pass < 2; ++pass) {
      long long hi = u1;
      for (int i = 0; i < pre;) {
        const ProdSeg t = prod_seg(g, u0, hi);
        const int tile = t.item / g.chunks, z = t.item % g.chunks;
        for (int kb = t.kb0; kb < t.kb1 && i < pre; ++kb, ++i) {
          const uint32_t dst = smem_u32(smem) + i * stage_bytes, bar = smem_u32(&ctl->full[i]);
          if (elect_one()) {
            if (pass == 0) load_w(dst, bar, mx_block(tile, kb, g.n_kb));
            if (pass == 1 && !kOwn) load_x(dst, bar, z * g.n_kb + kb);
          }
          __syncwarp();
        }
        hi -= t.kb1 - t.kb0;
      }
      if (pass == 0) {
        pdl_wait();
        if (threadIdx.x == 0) stamp_waited(g.stamp);
      }
    }
    int s = 0, it = 0;
    uint32_t ph = 0, dst = smem_u32(smem);
    bool ok = true;
    for (long long hi = u1; ok && hi > u0;) {
      const ProdSeg t = prod_seg(g, u0, hi);
      const int tile = t.item / g.chunks, z = t.item % g.chunks;
      for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
        if (it >= pre) {
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl->empty[s]), ph ^ 1));
          if (!ok) {
            if (lane == 0) prod_error(g, DEV_TIMEOUT_EMPTY);
            break;
          }
          const uint32_t bar = smem_u32(&ctl->full[s]);
          if (elect_one()) {
            load_w(dst, bar, mx_block(tile, kb, g.n_kb));
            if (!kOwn) load_x(dst, bar, z * g.n_kb + kb);
          }
          __syncwarp();
        }
        dst += stage_bytes;
        if (++s == g.stages) { s = 0; ph ^= 1; dst = smem_u32(smem); }
      }
      hi -= t.kb1 - t.kb0;
    }
    // whatever becomes of the other roles, this CTA's shared memory stays until its last copies have arrived
    for (int i = max(0, it - g.stages); i < it; ++i)
      if (!mbar_wait(smem_u32(&ctl->full[i % g.stages]), (i / g.stages) & 1)) break;
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------------ products
    const uint32_t idesc = umma_idesc_mx(kMxTileN, ncols);
    bool ok = true;
    int s = 0, j = 0;
    uint32_t ph = 0;
    for (long long hi = u1; ok && hi > u0; ++j) {
      const ProdSeg t = prod_seg(g, u0, hi);
      const int b = n_acc == 2 ? j & 1 : 0, use = n_acc == 2 ? j >> 1 : j;
      const uint32_t d = tmem_base + b * acc_cols;
      // the accumulator's previous tile has been read out
      if (use > 0 && !__all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl->acc_empty[b]), (use - 1) & 1))) {
        if (lane == 0) prod_error(g, DEV_TIMEOUT_TMEM);
        ok = false;
      }
      // Two blocks per round of the loop: of the 600 cycles that a block took by itself, longer than its share of the memory's time, 230 went
      // into its six instructions, the others into waiting, electing and walking.
      for (int kb = t.kb0; ok && kb < t.kb1;) {
        const bool pair = g.stages >= 4 && kb + 1 < t.kb1, wrap = s + 1 == g.stages;   // (a short ring would wait for two copies)
        const int s1 = wrap ? 0 : s + 1;
        const uint32_t ph1 = wrap ? ph ^ 1 : ph;
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl->full[s]), ph) && (!pair || mbar_wait(smem_u32(&ctl->full[s1]), ph1)));
        if (!ok) {
          if (lane == 0) prod_error(g, DEV_TIMEOUT_FULL);
          break;
        }
        tc_fence_after();
        const uint32_t a0 = smem_u32(smem) + s * stage_bytes, a1 = smem_u32(smem) + s1 * stage_bytes;
        if (elect_one()) {
          prod_block(a0, scales + s * set_cols, d, idesc, act_bytes, sb_words, kb != t.kb0);
          umma_commit(smem_u32(&ctl->empty[s]));
          if (pair) {
            prod_block(a1, scales + s1 * set_cols, d, idesc, act_bytes, sb_words, true);
            umma_commit(smem_u32(&ctl->empty[s1]));
          }
        }
        __syncwarp();
        kb += 1 + pair;
        if (pair) {
          s = s1;
          ph = ph1;
        }
        if (++s == g.stages) { s = 0; ph ^= 1; }
      }
      if (elect_one()) {
        if (!ok) *reinterpret_cast<volatile uint32_t *>(&ctl->abort_flag) = 1;
        umma_commit(smem_u32(&ctl->acc_full[b]));
      }
      __syncwarp();
      hi -= t.kb1 - t.kb0;
    }
  } else if (kRuns) {
    // ------------------------------------------------------------------ epilogue of a run
    // Thread <-> feature out of tensor memory, where partial sums go to and come from a slab as they are (a warp's 32 features are a line);
    // finished ones through shared memory, eight rows at a time, to a warp per row with four features per lane.
    const int q = warp & 3;                       // TMEM lane quarter this warp may read
    const int f = q * 32 + lane;                  // this thread's feature of a tile
    const uint32_t stg = smem_u32(staging);
    pdl_wait();   // (flags are cleared by the kernel before; outputs may still be read by its consumers)
    if (EPI == MX_SWIGLU && cta == 0 && warp == 2) mx_clear_flags(g.mo, lane, 32);
    int j = 0, turn = 0;
    bool alive = true;   // (all warps go through the same barriers whatever becomes of a wait; after one has expired none is waited for)
    for (long long hi = u1; hi > u0; ++j) {
      const ProdSeg t = prod_seg(g, u0, hi);
      hi -= t.kb1 - t.kb0;
      const int b = n_acc == 2 ? j & 1 : 0, use = n_acc == 2 ? j >> 1 : j;
      bool ok = alive && __all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl->acc_full[b]), use & 1));
      if (!ok && lane == 0) prod_error(g, DEV_TIMEOUT_TMEM);
      alive = ok;
      tc_fence_after();
      ok = ok && (*reinterpret_cast<volatile uint32_t *>(&ctl->abort_flag) == 0);
      const int tile = t.item / g.chunks, z = t.item - tile * g.chunks, m0 = z * g.Mc, M = min(g.Mc, g.M - m0);
      const uint32_t taddr = tmem_base + b * acc_cols + ((uint32_t)(q * 32) << 16);
      auto emptied = [&]() {   // the sums are out of tensor memory
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ctl->acc_empty[b]));
      };
      if (t.kb1 != g.n_kb) {   // another CTA finishes the tile
        float *slab = g.slabs + (size_t)cta * g.Mc * kMxTileN + f;
        for (int c0 = 0; c0 < M; c0 += 8) {
          float v[8];
          prod_sums(g, taddr + c0, v);
          if (c0 + 8 >= M) emptied();
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (ok) __stcg(slab + (c0 + i) * kMxTileN, v[i]);   // (rows behind the last one too: Mc is a multiple of eight)
        }
        __threadfence();
        asm volatile("bar.sync 1, 128;" ::: "memory");
        if (warp == 2 && lane == 0 && ok) asm volatile("st.release.gpu.global.b32 [%0], %1;" ::"l"(g.flags + cta), "r"(1) : "memory");
        continue;
      }
      int before = cta;   // CTAs [before, cta) have its earlier k-blocks
      if (t.kb0 > 0) {
        const long long first = (long long)t.item * g.n_kb;
        do --before;
        while (prod_start(g, before, G) > first);
        for (int c = before; ok && c < cta; ++c) ok = __all_sync(0xffffffffu, wait_flag(g.flags + c));
        if (!ok && lane == 0) prod_error(g, DEV_TIMEOUT_GRID);
      }
      float part[8];   // the CTAs' partial sums, eight rows ahead of use
      auto fetch = [&](int c0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) part[i] = 0.f;
        for (int c = before; ok && c0 < M && c < cta; ++c) {
          const float *slab = g.slabs + ((size_t)c * g.Mc + c0) * kMxTileN + f;
          float x[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = __ldcg(slab + i * kMxTileN);
#pragma unroll
          for (int i = 0; i < 8; ++i) part[i] += x[i];
        }
      };
      fetch(0);
      const int n = tile * kMxTileN + lane * 4;
      for (int c0 = 0; c0 < M; c0 += 8, turn ^= 1) {
        const uint32_t buf = stg + turn * (kProdStaging / 2);
        float v[8];
        prod_sums(g, taddr + c0, v);
        if (c0 + 8 >= M) emptied();
#pragma unroll
        for (int i = 0; i < 8; ++i) st_shared_f32(buf + (i * kMxTileN + f) * 4, v[i] + part[i]);
        fetch(c0 + 8);
        asm volatile("bar.sync 1, 128;" ::: "memory");
        for (int i = warp - 2; ok && i < 8 && c0 + i < M; i += 4) {
          const uint4 u = ld_shared_v4(buf + (i * kMxTileN + lane * 4) * 4);
          const float w[4] = {__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w)};
          mx_finish<EPI>(g, g.row0 + m0 + c0 + i, n, w, lane);
        }
      }
    }
  } else if (MODE == kTile && warp < 6) {
    // ------------------------------------------------------------------ epilogue of a tile
    // The sums go through the ring's shared memory (free by now: every copy was consumed by a product that has completed) to
    // [row][128 features]; then a warp takes every fourth row with four consecutive features per lane.  The rows are dealt out over the
    // CTAs of a cluster, which add the slices' sums in slice order.
    if (EPI == MX_SWIGLU && cta == 0 && split == 0 && warp == 2) {
      pdl_wait();
      mx_clear_flags(g.mo, lane, 32);
    }
    const int q = warp & 3, item = cta, tile = item / g.chunks, m0 = (item - tile * g.chunks) * g.Mc, M = min(g.Mc, g.M - m0);
    pdl_wait();   // outputs of this kernel may still be read by the previous one's consumers
    const bool done = __all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl->acc_full[0]), 0));
    if (!done && lane == 0) prod_error(g, DEV_TIMEOUT_TMEM);
    tc_fence_after();
    const bool ok = done && (*reinterpret_cast<volatile uint32_t *>(&ctl->abort_flag) == 0);
    const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16), stg = smem_u32(smem);
    for (int c0 = 0; ok && c0 < M; c0 += 8) {
      float v[8];
      prod_sums(g, taddr + c0, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) st_shared_f32(stg + ((c0 + i) * kMxTileN + q * 32 + lane) * 4, v[i]);
    }
    if (C > 1) {
      __syncwarp();
      cluster_arrive();
      cluster_wait();
    } else {
      asm volatile("bar.sync 1, 128;" ::: "memory");
    }
    const int rows_per = (M + C - 1) / C, m_beg = split * rows_per, m_end = min(M, m_beg + rows_per);
    const int n = tile * kMxTileN + lane * 4;
    for (int m = m_beg + warp - 2; ok && m < m_end; m += 4) {
      const uint32_t at = stg + (m * kMxTileN + lane * 4) * 4;
      float v[4] = {0.f, 0.f, 0.f, 0.f};
      if (C == 1) {
        const uint4 u = ld_shared_v4(at);
        v[0] = __uint_as_float(u.x); v[1] = __uint_as_float(u.y); v[2] = __uint_as_float(u.z); v[3] = __uint_as_float(u.w);
      } else {
        float4 p[8];
#pragma unroll
        for (int c = 0; c < 8; ++c)
          if (c < C) p[c] = ld_cluster_v4(at, c);
#pragma unroll
        for (int c = 0; c < 8; ++c)
          if (c < C) { v[0] += p[c].x; v[1] += p[c].y; v[2] += p[c].z; v[3] += p[c].w; }
      }
      mx_finish<EPI>(g, g.row0 + m0 + m, n, v, lane);
    }
  } else if constexpr (kOwn > 0) {
    // ------------------------------------------------------------------ planes
    // A warp to a block, as many blocks at a time as there are warps (one block's chain of conversions takes about a thousand cycles):
    // sixteen threads to a row, eight columns each, two rows at a time.
    typedef typename MxElem<TYPE>::raw raw;
    // (no more warps than stages: a warp that has a block's stage has seen the stage of the block `warps` before emptied, so that the parity
    // it waits for is never that of a phase long past)
    const int warps = min(own_warps(kOwn), g.stages);
    const int col = (lane & 15) * 8, kb0 = (int)(u0 - first), nkb = (int)(u1 - u0);
    MxRaw8<TYPE> x[kOwn];   // the warp's next block
    auto fetch = [&](int i) {
#pragma unroll
      for (int r = 0; r < kOwn; ++r) {
        const int m = 2 * r + (lane >> 4);
        mx_fetch8<TYPE>((const raw *)g.x + (size_t)m * g.ldx, g.pair, m < g.M && i < nkb, (kb0 + i) * kMxTileK + col, g.K, g.vec_x, x[r]);
      }
    };
    pdl_wait();
    if (warp - 6 < warps) fetch(warp - 6);
    for (int i = warp - 6; warp - 6 < warps && i < nkb; i += warps) {
      float v[kOwn][8];
#pragma unroll
      for (int r = 0; r < kOwn; ++r) mx_widen8<TYPE>(x[r], v[r]);
      fetch(i + warps);
      const int s = i % g.stages;
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl->empty[s]), ((i / g.stages) & 1) ^ 1))) {
        if (lane == 0) prod_error(g, DEV_TIMEOUT_EMPTY);
        break;
      }
#pragma unroll
      for (int r = 0; r < kOwn; ++r)
        if (2 * r < g.M) mx_to_planes(v[r], 2 * r + (lane >> 4) < g.M, smem + (size_t)s * stage_bytes + kProdW, act_bytes, g.Mc, g.planes, 2 * r + (lane >> 4), col);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&ctl->full[s]));
    }
  }
  if constexpr (!kRuns) {
    if (C > 1) {
      // (every thread of the cluster takes part in both barriers: the sums are in shared memory, then: nobody reads mine any more)
      __syncwarp();
      if (warp < 2 || warp >= 6) {
        cluster_arrive();
        cluster_wait();
      }
      cluster_arrive();
      cluster_wait();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, alloc_cols);
  }
  if (threadIdx.x == 0 && g.stamp) stamp_max(g.stamp + 3);
}

// (elements of the weights, their scales, the activations' block as it lies in memory: both operands on 1024-byte boundaries)
static size_t prod_stage_bytes(int planes, int Mc) { return kProdW + ((512 + mx_x_block(planes * Mc) + 1023) & ~1023); }

// Rows per chunk: all of them up to 224 instruction columns, else equal chunks of fewer.  Then CTAs, two to an SM: clusters of as many
// along K as there is room for, eight at most, or runs of k-blocks.  Up to 64 rows (fp32: 32, which is a chunk) neither the cut along K nor
// the order of the sums may depend on the number of rows: chunks do not count then, and where runs are dealt out each is a launch of its
// own.
//
// Runs where there are more tiles than places, and where tiles do not come out even over the SMs and the time that costs is worth the
// second exchange at a run's end, 4 to 8 us (device time, tiles and runs): 20480 x 12288, 160 tiles, 1 row 32.8 and 29.1 us, 32 rows 39.7 and 35.1,
// 64 rows 47.3 and 41.5; 20480 x 8192 22.9 and 23.2, 28.3 and 28.1, 34.2 and 35.0; 24576 x 4096, 192 tiles, 13.8 and 18.4, 17.8 and 22.2, 21.3 and 28.2;
// 112 rows x 20480 x 8192 50.1 and 48.0, 301 fp16 rows x 4096 x 12288 65.8 and 50.1, 112 x 24576 x 4096 30.0 and 38.0.  (An SM takes a block in about
// 256 + 2 x columns cycles, the time of its bytes through shared memory: weights 16 KB, columns x 128, all of it written and read, 128 a
// cycle.  Up to 64 rows the rule may not see how many there are and counts 32 columns.)
// Rows whose planes the product makes itself: up to two, and up to four where a CTA has few blocks (its warps make a block of four rows in
// about as long as a block of two takes to be multiplied; 4096 x 4096 at 4 rows 8.4 -> 6.5 us, 24576 x 4096 at 3 rows 15.4 and 17.1).
// Up to eight bf16 rows take as long that way as with a launch for the planes (2048 x 8192 at 8 rows 9.0 and 8.9 us; fp16 9.5 and 8.8, fp32 11.5
// and 8.8), but cost a call of its own one launch less on the host (12.3 -> 9.5 us).
constexpr int kOwnRows = 2, kOwnRowsShort = 4, kOwnRowsAlone = 8, kOwnShort = 8;
constexpr int kRunCycles = 25000;
// Equal chunks of at most kProdAcc instruction columns (planes x rows), of which there are a multiple of 16.
static int mx_step(int planes) { return planes % 2 ? 16 : 8; }
static MxPlan mx_cut(int M, int planes) {
  MxPlan p{};
  const int step = mx_step(planes), most = kProdAcc / planes / step * step;
  p.chunks = (M + most - 1) / most;
  p.Mc = ((M + p.chunks - 1) / p.chunks + step - 1) / step * step;
  p.chunks = (M + p.Mc - 1) / p.Mc;
  return p;
}
MxPlan mx_plan(int M, int tiles, int n_kb, int planes, int n_sms, const int *fits, bool alone) {
  MxPlan p = mx_cut(M, planes);
  n_sms = std::min(n_sms, kMxMostSms);
  const bool same = M <= (planes == 5 ? 32 : 64);
  const long long items = (long long)tiles * (same ? 1 : p.chunks), places = (long long)kProdCtas * n_sms;
  const long long uneven = ((items + n_sms - 1) / n_sms * n_sms - items) * n_kb * (256 + 2 * (same ? 32 : planes * p.Mc)) / n_sms;
  p.apart = same && p.chunks > 1;
  p.stream = items > n_sms && items * n_kb >= 4 * places && ((items > places && (same || p.chunks == 1)) || uneven > kRunCycles);
  // (A tenth more than are needed must fit: how many do depends on how the device's SMs are grouped, and one that finds its place taken runs
  // as a second wave.  6144 x 4096 at 32 rows: 48 clusters of six, of which 45 fit, 15.2 us; of five 9.6.)
  p.cluster = 1;
  for (int c = 2; fits && !p.stream && c <= 8 && c <= n_kb; ++c)
    if (fits[c] * 10ll >= items * 11) p.cluster = c;
  p.ctas = (int)(p.stream ? places : (long long)tiles * p.chunks);
  p.own = !p.stream && M <= (n_kb > kOwnShort * p.cluster ? kOwnRows : alone && planes == 2 ? kOwnRowsAlone : kOwnRowsShort);
  return p;
}

MxScratch mx_scratch(int n_kb, int planes, const MxPlan &p) {
  MxScratch w{};
  if (p.own) return w;
  const uint64_t n_flags = p.stream ? (uint64_t)(p.apart ? p.chunks : 1) * p.ctas : 0;   // (a launch's flags are its own, the slabs are reused)
  w.flags = (uint64_t)p.chunks * n_kb * mx_x_block(planes * p.Mc);
  w.slabs = w.flags + (n_flags * 4 + 127) / 128 * 128;
  w.bytes = w.slabs + (p.stream ? (uint64_t)p.ctas * p.Mc * kMxTileN * 4 : 0);
  return w;
}
uint64_t mx_scratch_most(int rows, int tiles, int n_kb, int planes) {
  if (!rows || !tiles || !n_kb) return 0;
  MxPlan p = mx_cut(rows, planes);
  if (p.chunks > 1) {   // (equal chunks may be larger for fewer rows)
    p.Mc = kProdAcc / planes / mx_step(planes) * mx_step(planes);
    p.chunks = (rows + p.Mc - 1) / p.Mc;
  }
  // (mx_plan deals out in runs where there are more items than SMs, and four k-blocks or more for each of the CTAs, two to an SM)
  const long long items = (long long)tiles * p.chunks;
  p.ctas = (int)std::min({(long long)kProdCtas * kMxMostSms, kProdCtas * (items - 1), items * n_kb / 4});
  p.stream = p.apart = p.ctas > 0;
  return mx_scratch(n_kb, planes, p).bytes;
}

static constexpr size_t kProdSmem = 113 * 1024;   // of a CTA
int gemm_max_clusters(int cluster, size_t smem_budget);   // gemm_tcgen05.cu
void mx_fits(int (&fits)[9]) {
  fits[0] = 0;
  for (int c = 1; c <= 8; ++c) fits[c] = gemm_max_clusters(c, kProdSmem);
}

template <int EPI, int MODE, int kOwn, int TYPE>
static cudaError_t prod_launch_one(const CUtensorMap &tw, const MxArgs &g, const MxPlan &p, size_t smem, cudaStream_t st, bool pdl) {
  static PerDeviceOnce once;
  int dev = -1;
  if (once.needed(&dev)) {
    cudaError_t e = cudaFuncSetAttribute(mx_product_kernel<EPI, MODE, kOwn, TYPE>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
    if (e != cudaSuccess) return e;
    once.done(dev);
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(p.ctas, p.cluster);
  cfg.blockDim = dim3(prod_threads<kOwn>());
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  int n = 0;
  if (p.cluster > 1) {
    at[n].id = cudaLaunchAttributeClusterDimension;
    at[n].val.clusterDim.x = 1;
    at[n].val.clusterDim.y = p.cluster;
    at[n].val.clusterDim.z = 1;
    ++n;
  }
  if (pdl) {
    at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[n].val.programmaticStreamSerializationAllowed = 1;
    ++n;
  }
  cfg.attrs = at;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, mx_product_kernel<EPI, MODE, kOwn, TYPE>, tw, g);
}

template <int EPI, int TYPE>
static cudaError_t prod_launch_own(const CUtensorMap &tw, const MxArgs &g, const MxPlan &p, size_t smem, cudaStream_t st, bool pdl) {
  if (g.M <= 2) return prod_launch_one<EPI, kTile, 1, TYPE>(tw, g, p, smem, st, pdl);
  if (g.M <= 4) return prod_launch_one<EPI, kTile, 2, TYPE>(tw, g, p, smem, st, pdl);
  if constexpr (EPI == MX_STORE && TYPE == MX_BF16) return prod_launch_one<EPI, kTile, 4, TYPE>(tw, g, p, smem, st, pdl);
  return cudaErrorInvalidValue;
}
template <int EPI>
static cudaError_t prod_launch(const CUtensorMap &tw, const MxArgs &g, const MxPlan &p, size_t smem, cudaStream_t st, bool pdl) {
  if (p.stream) return prod_launch_one<EPI, kStream, 0, 0>(tw, g, p, smem, st, pdl);
  if (!p.own) return prod_launch_one<EPI, kTile, 0, 0>(tw, g, p, smem, st, pdl);
  if (g.x_type == MX_BF16) return prod_launch_own<EPI, MX_BF16>(tw, g, p, smem, st, pdl);
  if (g.x_type == MX_PAIR) return prod_launch_own<EPI, MX_PAIR>(tw, g, p, smem, st, pdl);
  if constexpr (EPI == MX_STORE) {   // (a model's activations are of the two types above)
    if (g.x_type == MX_F16) return prod_launch_own<EPI, MX_F16>(tw, g, p, smem, st, pdl);
    if (g.x_type == MX_F32) return prod_launch_own<EPI, MX_F32>(tw, g, p, smem, st, pdl);
  }
  return cudaErrorInvalidValue;
}

MxOut mx_out(int n_kb, int planes, void *scratch, const MxPlan &p) {
  if (p.own) return MxOut{};
  const MxScratch w = mx_scratch(n_kb, planes, p);
  return MxOut{(uint8_t *)scratch, p.Mc, planes, n_kb, (int *)((uint8_t *)scratch + w.flags), p.stream ? (p.apart ? p.chunks : 1) * p.ctas : 0};
}

cudaError_t launch_mx_product(int epi, const CUtensorMap &tw, MxArgs g, const MxInput &in, void *scratch, const MxPlan &p, cudaStream_t st,
                              bool pdl, int *launches) {
  const MxScratch w = mx_scratch(g.n_kb, mx_planes_of(in.type), p);
  g.planes = mx_planes_of(in.type);
  g.Mc = p.Mc;
  g.ldx = in.ldx; g.pair = in.pair; g.x_type = in.type; g.K = in.cols;
  g.vec_x = mx_aligned(in.x, in.ldx, in.type) && (in.type != MX_PAIR || in.pair % 8 == 0);
  g.slabs = (float *)((uint8_t *)scratch + w.slabs);
  const size_t stage = prod_stage_bytes(g.planes, g.Mc), fixed = kProdStaging + sizeof(ProdSmemCtl);
  g.stages = (int)std::min<size_t>(kProdMaxStages, (kProdSmem - fixed) / stage);
  const int ncols = g.planes * g.Mc;
  const int acc = (ncols + 31) & ~31, sets = g.stages * (4 + 4 * ((ncols + 127) / 128));   // columns of an accumulator, of the stages' scales
  g.n_acc = p.stream && 2 * acc + sets <= 256 ? 2 : 1;
  const size_t smem = g.stages * stage + fixed;
  const bool apart = p.stream && p.apart;
  const int passes = apart ? p.chunks : 1;
  g.chunks = apart ? 1 : p.chunks;
  g.units = (long long)g.tiles * g.chunks * g.n_kb;
  if (g.stages < 2 || g.Mc % 8 || ncols % 16 || ncols > kProdAcc || g.n_acc * acc + sets > 256 || p.ctas < 1 || p.cluster < 1 || p.cluster > 8 ||
      p.cluster > g.n_kb || (p.stream && p.ctas > g.units) || (size_t)g.stages * stage < (size_t)g.Mc * kMxTileN * 4 || (p.own && passes != 1))
    return cudaErrorInvalidValue;
  for (int i = 0; i < passes; ++i) {
    g.row0 = i * g.Mc;
    g.M = passes == 1 ? in.rows : std::min(g.Mc, in.rows - g.row0);
    g.x = p.own ? in.x : (const uint8_t *)scratch + (size_t)i * g.n_kb * mx_x_block(ncols);
    g.flags = (int *)((uint8_t *)scratch + w.flags) + (p.stream ? i * p.ctas : 0);
    cudaError_t e = cudaErrorInvalidValue;
    switch (epi) {
      case MX_STORE: e = prod_launch<MX_STORE>(tw, g, p, smem, st, pdl); break;
      case MX_SWIGLU: e = prod_launch<MX_SWIGLU>(tw, g, p, smem, st, pdl); break;
      case MX_LOGITS: e = prod_launch<MX_LOGITS>(tw, g, p, smem, st, pdl); break;
    }
    if (e != cudaSuccess) return e;
    if (g.stamp) g.stamp += 4;   // (the next launch's)
  }
  if (launches) *launches = passes;
  return cudaSuccess;
}

}  // namespace ts
