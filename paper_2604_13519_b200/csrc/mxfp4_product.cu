// y[m][n] = sum_k x[m][k] * W[n][k] with W in MXFP4 and the activations as bf16 planes (their sum is x; one plane for bf16 rows).
//
// The tensor cores multiply bf16: every e2m1 value times a power of two is a bf16 number, so products are exact and sums are
// fp32, as with bf16 weights.  What the four bits save is memory traffic: 17 bytes for 32 weights instead of 64.  The weights are
// widened on their way: threads take a row's 32 codes of a block out of shared memory, turn them into bf16 in registers and put
// them into TENSOR memory, where the product reads its 128-row operand from (lane = weight row, two elements per column).  So the
// widened weights never pass through shared memory, whose bandwidth they would take twice (written, and read by the product).
//
// Roles: warp 0 brings in weight blocks (bulk copies: a block is contiguous) and activation boxes (TMA), warp 1 allocates tensor
// memory and issues the products, the others (four per weight tile) widen and at the end take the sums out.
// Every wait is bounded; on expiry the CTA records an error word and leaves through the normal exit.
#include <cuda_fp16.h>

#include <algorithm>

#include "mxfp4.h"

namespace ts {

static constexpr int kMxMaxStages = 12;
static constexpr int kMxWide = 2;          // widened blocks in tensor memory: one being multiplied while the next is written
static constexpr int kWideCols = kMxTileK / 2;

struct __align__(16) MxSmemCtl {
  uint64_t full[kMxMaxStages];
  uint64_t empty[kMxMaxStages];
  uint64_t wide_full[kMxWide];
  uint64_t wide_empty[kMxWide];
  uint64_t tmem_full;
  uint32_t tmem_base;
  uint32_t abort_flag;
};

__device__ __forceinline__ void mx_error(const MxArgs &g, int code) { if (g.err) atomicExch(g.err, code); }

__device__ __forceinline__ uint32_t bf16x2_mul(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// Eight codes (see mx_place) -> four bf16 pairs.  The masked bits read as bf16 are value x 2^-126 (subnormal for 0.5), which the
// multiplication by 2^(s - 1) brings to value x 2^(s - 127) without rounding.
__device__ __forceinline__ void mx_unpack(uint32_t w, uint32_t mul, uint32_t *r) {
  constexpr uint32_t M = 0x81C081C0u;
  r[0] = bf16x2_mul(w & M, mul);
  r[1] = bf16x2_mul((w << 3) & M, mul);
  r[2] = bf16x2_mul((w << 6) & M, mul);
  uint32_t t = (w >> 4) & 0x00C000C0u;
  t |= (w >> 5) & 0x01000100u;
  t |= (w << 1) & 0x80008000u;
  r[3] = bf16x2_mul(t, mul);
}

// Scale byte -> multiplier pairs: 2^(s - 1) while that is a bf16 number (s <= 128), else 2^127 and a second factor.
__device__ __forceinline__ uint32_t mx_factor(uint32_t s) {
  const uint32_t b = (min(s, 128u) + 126u) << 7;
  return b | b << 16;
}
__device__ __forceinline__ uint32_t mx_factor2(uint32_t s) {   // (255: not a number)
  const uint32_t b = s == 255u ? 0x7FC0u : (s > 128u ? (s - 1u) << 7 : 0x3F80u);
  return b | b << 16;
}

template <int WT, int EPI>
__global__ void __launch_bounds__(64 + 128 * WT, WT == 1 ? 2 : 1)
mx_product_kernel(const __grid_constant__ CUtensorMap tmap_a, const MxArgs g) {
  extern __shared__ __align__(1024) uint8_t smem[];
  const int box_bytes = g.planes * g.Mc * 128;                       // 64 columns of the activations
  const int act_bytes = 2 * box_bytes;
  const int stage_bytes = (act_bytes + WT * kMxTileBytes + 1023) & ~1023;
  MxSmemCtl *ctl = reinterpret_cast<MxSmemCtl *>(smem + (size_t)g.stages * stage_bytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int tile0 = blockIdx.x * WT, nt = min(WT, g.tiles - tile0);   // weight tiles of this CTA (the last may have one of two)
  const int split = blockIdx.y, C = (int)gridDim.y;                   // the CTA's rank in its cluster, which spans the K slices
  const int m0 = blockIdx.z * g.Mc, M = min(g.Mc, g.M - m0);          // its activation rows
  const int kb0 = (int)(((long long)split * g.n_kb) / C), nkb = (int)(((long long)(split + 1) * g.n_kb) / C) - kb0;
  const uint32_t ncols = g.planes * g.Mc, acc_cols = (ncols + 31) & ~31u;
  uint32_t alloc_cols = 32;
  while (alloc_cols < WT * (acc_cols + kMxWide * kWideCols)) alloc_cols <<= 1;

  if (warp == 0 && lane == 0) {
    tma_prefetch_desc(&tmap_a);
    for (int s = 0; s < g.stages; ++s) {
      mbar_init(smem_u32(&ctl->full[s]), 1);
      mbar_init(smem_u32(&ctl->empty[s]), 4 * WT + 1);   // the widening warps have the codes, the products have the activations
    }
    for (int s = 0; s < kMxWide; ++s) {
      mbar_init(smem_u32(&ctl->wide_full[s]), 4 * WT);
      mbar_init(smem_u32(&ctl->wide_empty[s]), 1);
    }
    mbar_init(smem_u32(&ctl->tmem_full), 1);
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
  const uint32_t tmem_base = ctl->tmem_base, wide_base = tmem_base + WT * acc_cols;
  if (threadIdx.x == 0) stamp_min(g.stamp);
  // (placed after this CTA holds its resources, so a waiting dependent can never starve an earlier kernel)
  pdl_launch_dependents();

  if (warp == 0) {
    // ------------------------------------------------------------------ producer
    if (lane == 0) {
      const uint64_t pol_w = policy_evict_first(), pol_a = policy_evict_last();
      const uint32_t w_bytes = nt * kMxTileBytes;
      auto load_w = [&](int s, int kb) {
        const uint32_t bar = smem_u32(&ctl->full[s]);
        mbar_expect_tx(bar, w_bytes + act_bytes);
        bulk_load(smem_u32(smem + (size_t)s * stage_bytes + act_bytes), g.w + ((size_t)kb * g.tiles + tile0) * kMxTileBytes, w_bytes, bar, pol_w);
      };
      auto load_a = [&](int s, int kb) {
        const uint32_t bar = smem_u32(&ctl->full[s]), dst = smem_u32(smem + (size_t)s * stage_bytes);
        tma_load_3d(dst, &tmap_a, kb * kMxTileK, m0, 0, bar, pol_a);
        tma_load_3d(dst + box_bytes, &tmap_a, kb * kMxTileK + 64, m0, 0, bar, pol_a);
      };
      // weights do not depend on the previous kernel: they are on their way before the programmatic-dependency wait
      const int pre = min(g.stages, nkb);
      for (int it = 0; it < pre; ++it) load_w(it, kb0 + it);
      pdl_wait();
      stamp_waited(g.stamp);
      for (int it = 0; it < pre; ++it) load_a(it, kb0 + it);
      int s = pre == g.stages ? 0 : pre, it = pre;
      uint32_t ph = pre == g.stages ? 1 : 0;
      for (; it < nkb; ++it) {
        if (!mbar_wait(smem_u32(&ctl->empty[s]), ph ^ 1)) {
          mx_error(g, DEV_TIMEOUT_EMPTY);
          break;
        }
        load_w(s, kb0 + it);
        load_a(s, kb0 + it);
        if (++s == g.stages) { s = 0; ph ^= 1; }
      }
      // whatever becomes of the other roles, this CTA's shared memory stays until its last copies have arrived
      for (int i = max(0, it - g.stages); i < it; ++i)
        if (!mbar_wait(smem_u32(&ctl->full[i % g.stages]), (i / g.stages) & 1)) break;
    }
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------------ products
    const uint32_t idesc = umma_idesc_bf16(kMxTileN, ncols);
    bool ok = true;
    int s = 0, t = 0;
    uint32_t ph = 0, tp = 0;
    for (int it = 0; it < nkb; ++it) {
      // (the widened weights come from this stage's codes, so the activations are here too, but this thread has to have seen it)
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl->full[s]), ph) && mbar_wait(smem_u32(&ctl->wide_full[t]), tp))) {
        if (lane == 0) mx_error(g, DEV_TIMEOUT_FULL);
        ok = false;
        break;
      }
      tc_fence_after();
      const uint32_t sa = smem_u32(smem + (size_t)s * stage_bytes);
      const uint64_t db0 = umma_desc_sw128(sa), db1 = umma_desc_sw128(sa + box_bytes);
      if (elect_one()) {
#pragma unroll
        for (int i = 0; i < WT; ++i) {
#pragma unroll
          for (int kk = 0; kk < kMxTileK / 16; ++kk)
            umma_f16_ts(tmem_base + i * acc_cols, wide_base + (t * WT + i) * kWideCols + kk * 8, (kk < 4 ? db0 : db1) + 2 * (kk & 3), idesc,
                        (it | kk) != 0);
        }
        umma_commit(smem_u32(&ctl->empty[s]));
        umma_commit(smem_u32(&ctl->wide_empty[t]));
      }
      __syncwarp();
      if (++s == g.stages) { s = 0; ph ^= 1; }
      if (++t == kMxWide) { t = 0; tp ^= 1; }
    }
    if (elect_one()) {
      if (!ok) *reinterpret_cast<volatile uint32_t *>(&ctl->abort_flag) = 1;
      umma_commit(smem_u32(&ctl->tmem_full));
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ widening, then the sums
    const int sub = (warp - 2) >> 2;              // weight tile of the CTA
    const int q = warp & 3;                       // TMEM lane quarter this warp may use
    const int row = q * 32 + lane;
    const uint32_t tq = (uint32_t)(q * 32) << 16;
    bool ok = true;
    {
      int s = 0, t = 0;
      uint32_t ph = 0, tp = 1;
      for (int it = 0; it < nkb; ++it) {
        if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl->full[s]), ph))) {
          if (lane == 0) mx_error(g, DEV_TIMEOUT_FULL);
          ok = false;
          break;
        }
        const uint32_t wb = smem_u32(smem + (size_t)s * stage_bytes + act_bytes) + sub * kMxTileBytes;
        uint4 codes[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) codes[j] = ld_shared_v4(wb + j * (kMxTileN * 16) + row * 16);
        uint32_t sc;
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(sc) : "r"(wb + kMxCodeBytes + row * 4) : "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ctl->empty[s]));
        if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl->wide_empty[t]), tp))) {
          if (lane == 0) mx_error(g, DEV_TIMEOUT_TMEM);
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t dst = wide_base + (t * WT + sub) * kWideCols + tq;
        // (scales above 2^1 need a second factor: rare, so the warp is asked once)
        const bool large = __any_sync(0xffffffffu, (sc & 0x80808080u) != 0 && __vmaxu4(sc, 0x80808080u) != 0x80808080u);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t s8 = (sc >> (8 * j)) & 255u, mul = mx_factor(s8);
          uint32_t r[16];
          mx_unpack(codes[j].x, mul, r);
          mx_unpack(codes[j].y, mul, r + 4);
          mx_unpack(codes[j].z, mul, r + 8);
          mx_unpack(codes[j].w, mul, r + 12);
          if (large) {
            const uint32_t more = mx_factor2(s8);
#pragma unroll
            for (int i = 0; i < 16; ++i) r[i] = bf16x2_mul(r[i], more);
          }
          tmem_st16(dst + j * 16, r);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ctl->wide_full[t]));
        if (++s == g.stages) { s = 0; ph ^= 1; }
        if (++t == kMxWide) { t = 0; tp ^= 1; }
      }
    }
    pdl_wait();   // outputs of this kernel may still be read by the previous one's consumers
    // The sums go through the ring's shared memory (free by now: every load was consumed by a product that has completed) to
    // [tile][row m][128 features]; then a warp takes every fourth row with four consecutive features per lane.  With the K slices
    // in one cluster the rows are dealt out over its CTAs, which add the slices' sums in slice order: the same order whatever the
    // number of rows.
    const bool done = mbar_wait(smem_u32(&ctl->tmem_full), 0);
    if (!done && lane == 0) mx_error(g, DEV_TIMEOUT_TMEM);
    ok = __all_sync(0xffffffffu, ok && done);
    tc_fence_after();
    ok = ok && (*reinterpret_cast<volatile uint32_t *>(&ctl->abort_flag) == 0);
    const uint32_t taddr = tmem_base + sub * acc_cols + tq;
    const uint32_t stg = smem_u32(smem) + sub * (g.Mc * kMxTileN * 4);
    for (int c0 = 0; ok && c0 < M; c0 += 8) {
      uint32_t r[8];
      float v[8];
      tmem_ld8(taddr + c0, r);
      tmem_wait_ld();
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(r[j]);
      for (int p = 1; p < g.planes; ++p) {
        tmem_ld8(taddr + p * g.Mc + c0, r);
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += __uint_as_float(r[j]);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) st_shared_f32(stg + ((c0 + j) * kMxTileN + row) * 4, v[j]);
    }
    if (C > 1) {
      __syncwarp();
      cluster_arrive();
      cluster_wait();
    } else {
      asm volatile("bar.sync 1, %0;" ::"n"(128 * WT) : "memory");
    }
    const int rows_per = (M + C - 1) / C, m_beg = split * rows_per, m_end = min(M, m_beg + rows_per);
    const int n = (tile0 + sub) * kMxTileN + lane * 4;
    if (ok && sub < nt) {
      for (int m = m_beg + (warp - 2 & 3); m < m_end; m += 4) {
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        const uint32_t at = stg + (m * kMxTileN + lane * 4) * 4;
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
        const long long mg = m0 + m;
        if constexpr (EPI == MX_STORE) {
          if (g.y_type == MX_F32) {
            float *d = (float *)g.y + mg * g.ldy + n;
            if (g.vec && n + 4 <= g.N) {
              *reinterpret_cast<float4 *>(d) = make_float4(v[0], v[1], v[2], v[3]);
            } else {
              for (int j = 0; j < 4; ++j) if (n + j < g.N) d[j] = v[j];
            }
          } else {
            uint16_t h[4];
            for (int j = 0; j < 4; ++j)
              h[j] = g.y_type == MX_BF16 ? __bfloat16_as_ushort(__float2bfloat16_rn(v[j])) : __half_as_ushort(__float2half_rn(v[j]));
            uint16_t *d = (uint16_t *)g.y + mg * g.ldy + n;
            if (g.vec && n + 4 <= g.N) {
              *reinterpret_cast<uint2 *>(d) = make_uint2(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16);
            } else {
              for (int j = 0; j < 4; ++j) if (n + j < g.N) d[j] = h[j];
            }
          }
        } else if constexpr (EPI == MX_LOGITS) {
          *reinterpret_cast<float4 *>(g.out + (size_t)mg * g.N + n) = make_float4(v[0], v[1], v[2], v[3]);
          // order-preserving map of the float to an unsigned word; ties resolve to the lowest id (lowest lane, then
          // lowest of its four)
          uint32_t best = 0;
          int bi = 0;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t u = __float_as_uint(v[j]);
            u = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
            if (u > best) { best = u; bi = j; }
          }
          const uint32_t top = __reduce_max_sync(0xffffffffu, best);
          if (lane == __ffs(__ballot_sync(0xffffffffu, best == top)) - 1)
            atomicMax(g.amax + (size_t)mg * kAmaxStride, ((unsigned long long)top << 32) | (unsigned long long)(0xFFFFFFFFu - (uint32_t)(n + bi)));
        } else {  // MX_SWIGLU: even feature row = gate_f, odd = up_f, f = n / 2
          __nv_bfloat16 h0, l0, h1, l1;
          split_bf16(v[0] / (1.f + __expf(-v[0])) * v[1], h0, l0);
          split_bf16(v[2] / (1.f + __expf(-v[2])) * v[3], h1, l1);
          const int F = g.N >> 1, f = n >> 1;
          *reinterpret_cast<__nv_bfloat162 *>(g.act_out + (size_t)mg * F + f) = __halves2bfloat162(h0, h1);
          if (g.out_planes == 2)
            *reinterpret_cast<__nv_bfloat162 *>(g.act_out + ((size_t)g.act_rows + mg) * F + f) = __halves2bfloat162(l0, l1);
        }
      }
    }
  }
  if (C > 1) {
    // (every thread of the cluster takes part in both barriers: the sums are in shared memory, then: nobody reads mine any more)
    __syncwarp();
    if (warp < 2) {
      cluster_arrive();
      cluster_wait();
    }
    cluster_arrive();
    cluster_wait();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, alloc_cols);
  }
  if (threadIdx.x == 0 && g.stamp) stamp_max(g.stamp + 3);
}

static size_t mx_stage_bytes(int wt, int planes, int Mc) {
  return ((size_t)2 * planes * Mc * 128 + wt * kMxTileBytes + 1023) & ~(size_t)1023;
}

template <int WT, int EPI>
static cudaError_t mx_launch_one(const CUtensorMap &ta, const MxArgs &g, dim3 grid, size_t smem, cudaStream_t st, bool pdl) {
  static PerDeviceOnce once;
  int dev = -1;
  if (once.needed(&dev)) {
    cudaError_t e = cudaFuncSetAttribute(mx_product_kernel<WT, EPI>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
    if (e != cudaSuccess) return e;
    once.done(dev);
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(64 + 128 * WT);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  int n = 0;
  if (grid.y > 1) {
    at[n].id = cudaLaunchAttributeClusterDimension;
    at[n].val.clusterDim.x = 1;
    at[n].val.clusterDim.y = grid.y;
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
  return cudaLaunchKernelEx(&cfg, mx_product_kernel<WT, EPI>, ta, g);
}

MxPlan mx_plan(int M, int tiles, int n_kb, int planes, int n_sms) {
  MxPlan p;
  const int step = planes == 1 ? 16 : 8, most = 128 / planes;   // (the instruction's N, planes x rows, is a multiple of 16)
  p.Mc = std::min(most, (M + step - 1) / step * step);
  p.tiles_per_cta = p.Mc * planes > 32 ? 2 : 1;
  const int groups = (tiles + p.tiles_per_cta - 1) / p.tiles_per_cta * ((M + p.Mc - 1) / p.Mc), room = p.tiles_per_cta == 1 ? 2 * n_sms : n_sms;
  p.cluster = std::max(1, std::min(std::min(8, n_kb), room / std::max(1, groups)));
  return p;
}

cudaError_t launch_mx_product(int epi, const CUtensorMap &ta, MxArgs g, int wt, int cluster, cudaStream_t st, bool pdl) {
  const size_t stage = mx_stage_bytes(wt, g.planes, g.Mc);
  const size_t limit = (wt == 1 ? 113 : 227) * 1024 - sizeof(MxSmemCtl);
  g.stages = (int)std::min<size_t>(kMxMaxStages, limit / stage);
  const size_t smem = g.stages * stage + sizeof(MxSmemCtl);
  // the sums pass through the ring; both weight tiles' sums and widened blocks share the 512 columns of tensor memory
  if (wt < 1 || wt > 2 || g.stages < 2 || g.Mc % 8 || (g.planes * g.Mc) % 16 || g.planes * g.Mc > 256 || cluster < 1 || cluster > 8 ||
      cluster > g.n_kb || wt * (((g.planes * g.Mc + 31) & ~31) + kMxWide * kWideCols) > 512 || (size_t)g.stages * stage < (size_t)wt * g.Mc * kMxTileN * 4)
    return cudaErrorInvalidValue;
  const dim3 grid((g.tiles + wt - 1) / wt, cluster, (g.M + g.Mc - 1) / g.Mc);
  if (wt == 1) {
    switch (epi) {
      case MX_STORE: return mx_launch_one<1, MX_STORE>(ta, g, grid, smem, st, pdl);
      case MX_SWIGLU: return mx_launch_one<1, MX_SWIGLU>(ta, g, grid, smem, st, pdl);
      case MX_LOGITS: return mx_launch_one<1, MX_LOGITS>(ta, g, grid, smem, st, pdl);
    }
  } else {
    switch (epi) {
      case MX_STORE: return mx_launch_one<2, MX_STORE>(ta, g, grid, smem, st, pdl);
      case MX_SWIGLU: return mx_launch_one<2, MX_SWIGLU>(ta, g, grid, smem, st, pdl);
      case MX_LOGITS: return mx_launch_one<2, MX_LOGITS>(ta, g, grid, smem, st, pdl);
    }
  }
  return cudaErrorInvalidValue;
}

}  // namespace ts
