// Weights in MXFP4: blocks of 32 elements along K share a scale 2^(s - 127) (one byte, 255 = not a number); an element is a sign
// and one of 0, .5, 1, 1.5, 2, 3, 4, 6 (four bits).  Storage, conversion kernels and the product.
#pragma once
#include "kernels.h"

namespace ts {

constexpr int kMxBlock = 32;          // elements that share a scale
constexpr int kMxTileK = 128;         // reduction columns of a stored block: four MX blocks
constexpr int kMxTileN = 128;         // weight rows of a stored block
constexpr int kMxCodeBytes = kMxTileN * kMxTileK / 2;
constexpr int kMxTileBytes = kMxCodeBytes + kMxTileN * (kMxTileK / kMxBlock);   // codes, then scales: 8704

// A laid-out matrix of N x K: ceil(N / 128) x ceil(K / 128) blocks, a tile's blocks one after the other.  Inside a block: elements
// [128 rows][64 bytes], the even one of two in the low half of a byte, then scales [32][4][4]: bytes of row 32 j + l at [l][j], one per
// MX block (the order in which tcgen05.cp takes them to tensor memory).
__host__ __device__ inline int mx_scale_at(int row) { return kMxCodeBytes + (row & 31) * 16 + (row >> 5) * 4; }

__host__ __device__ inline int mx_block(int tile, int kb, int n_kb) { return tile * n_kb + kb; }

// Element types of activations and results (TS_MX_*); MX_PAIR, a model's activations: two arrays of bf16 whose sum is meant.
enum : int { MX_BF16 = 0, MX_F16 = 1, MX_F32 = 2, MX_PAIR = 3 };
inline int mx_planes_of(int type) { return type == MX_BF16 ? 2 : type == MX_F16 ? 3 : type == MX_F32 ? 5 : 4; }

struct MxArgs {
  const uint8_t *w;          // laid-out matrix
  const void *x;             // the activations' planes, see launch_mx_input; with plan.own the rows themselves:
  long long ldx, pair;       // row stride; MX_PAIR: distance of the two arrays, in elements
  int x_type, vec_x, K;      // type, rows can be read 16 bytes at a time, columns
  float *slabs;              // [CTA][Mc][128] sums of tiles that the CTA has without their last k-blocks
  int *flags;                // [CTA] its slab is there (zero before the launch)
  int N, M, row0;            // features, activation rows of this launch, the first one's place among all rows of the result
  int tiles, n_kb;           // 128-row tiles and 128-column blocks of the matrix
  int planes;                // planes of e4m3 numbers that are added
  int early;                 // the matrix was written long ago: its blocks may be fetched before the previous kernel is done
  int Mc, chunks, stages, n_acc;   // filled in by the launcher: activation rows per tile of the result, their chunks, stages of the ring, accumulators
  long long units;           // tiles x chunks x k-blocks
  int *err;                  // device status word (null: not wanted)
  unsigned long long *stamp;
  // MX_STORE
  void *y;
  long long ldy;
  int y_type;
  int vec;                // rows of y take four elements at a time
  // steps of a model, as in GemmArgs
  float *out;
  __nv_bfloat16 *act_out;
  int act_rows, out_planes;
  unsigned long long *amax;
  MxOut mo;                  // MX_SWIGLU: the output once more as planes
};
// bytes of 128 columns of the activations with `ncols` = planes x Mc instruction columns: elements, then scales
__host__ __device__ inline int mx_x_block(int ncols) { return ncols * kMxTileK + 512 * ((ncols + 127) / 128); }

enum : int { MX_STORE = 0, MX_SWIGLU = 1, MX_LOGITS = 2 };   // what a product does with its sums

#ifdef __CUDACC__
template <int TYPE> struct MxElem;
template <> struct MxElem<MX_BF16> { typedef uint16_t raw; };
template <> struct MxElem<MX_F16> { typedef uint16_t raw; };
template <> struct MxElem<MX_F32> { typedef uint32_t raw; };
template <> struct MxElem<MX_PAIR> { typedef uint16_t raw; };
template <int TYPE> __device__ __forceinline__ float mx_to_f32(typename MxElem<TYPE>::raw r) {
  if constexpr (TYPE == MX_BF16 || TYPE == MX_PAIR) return __uint_as_float((uint32_t)r << 16);
  else if constexpr (TYPE == MX_F16) return __half2float(__ushort_as_half(r));
  else return __uint_as_float(r);
}
template <int TYPE> __device__ __forceinline__ typename MxElem<TYPE>::raw mx_from_f32(float v) {
  if constexpr (TYPE == MX_BF16) return __bfloat16_as_ushort(__float2bfloat16_rn(v));
  else if constexpr (TYPE == MX_F16) return __half_as_ushort(__float2half_rn(v));
  else return __float_as_uint(v);
}

// elements [c, c + 8) of a row of `cols` as they are, zeros behind its end and where `there` is false.  (Coherent loads, in the order in which
// they stand: most callers run while the kernel ahead of them still writes these rows, up to the dependency wait, and __ldg is for data that
// nobody writes during the kernel.)
template <int TYPE> struct MxRaw8 { uint32_t w[TYPE == MX_F32 || TYPE == MX_PAIR ? 8 : 4]; };
template <int TYPE>
__device__ __forceinline__ void mx_fetch8(const typename MxElem<TYPE>::raw *p, long long pair, bool there, int c, int cols, bool vec, MxRaw8<TYPE> &x) {
  constexpr int kArrays = TYPE == MX_PAIR ? 2 : 1;
#pragma unroll
  for (int h = 0; h < kArrays; ++h) {
    const typename MxElem<TYPE>::raw *q = p + h * pair + c;
    uint32_t *w = x.w + 4 * h;
    if (vec && there && c + 8 <= cols) {
      if constexpr (TYPE == MX_F32) {
        if (((uintptr_t)q & 31) == 0) {
          ld_global_v8(q, w);   // (whole sectors)
          continue;
        }
      }
#pragma unroll
      for (int i = 0; i < (TYPE == MX_F32 ? 2 : 1); ++i) ld_global_v4(reinterpret_cast<const uint4 *>(q) + i, w + 4 * i);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t e = there && c + i < cols ? q[i] : 0u;
        if constexpr (TYPE == MX_F32) w[i] = e;
        else w[i >> 1] = i & 1 ? w[i >> 1] | e << 16 : e;
      }
    }
  }
}
template <int TYPE> __device__ __forceinline__ float mx_elem(const MxRaw8<TYPE> &x, int i, int array) {
  if constexpr (TYPE == MX_F32) return __uint_as_float(x.w[i]);
  else return mx_to_f32<TYPE>((typename MxElem<TYPE>::raw)(x.w[4 * array + (i >> 1)] >> (16 * (i & 1))));
}
template <int TYPE> __device__ __forceinline__ void mx_widen8(const MxRaw8<TYPE> &x, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = mx_elem<TYPE>(x, i, 0);
    if constexpr (TYPE == MX_PAIR) v[i] += mx_elem<TYPE>(x, i, 1);   // (exact: the second is the rounding remainder of the first)
  }
}

// NE elements at columns col .. col + NE - 1 of row m (m: within its chunk) into the planes of a block of 128 columns (col: within it) at
// `blk`; its scales lie `act_bytes` further on.  32 / NE neighbouring threads share an MX block.
//
// x as planes of e4m3 numbers (four significant bits each).  A block's first scale puts its largest magnitude into [2^7, 2^8), so that
// it and what rounding leaves of it, at most 2^3, stay in range (448); the next plane holds sixteen times the remainder with a scale
// of a sixteenth, and so on.  With two planes all bf16 numbers down to 2^-13 of the block's largest come out exactly (eight bits), and
// what is lost of smaller ones is at most 2^-21 of it; three planes do the same for fp16 (eleven bits, 2^-25), five for fp32 (24 bits down to 2^-9,
// 2^-33).  Scales end at 2^-127: of blocks that would need smaller ones up to 2^-137 is lost.  Each remainder is exact in fp32.  A block with an infinity or NaN gets the scale byte 255, which makes its products NaN.
template <int NE>
__device__ __forceinline__ void mx_to_planes(float (&v)[NE], bool there, uint8_t *blk, int act_bytes, int Mc, int planes, int m, int col) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < NE; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
#pragma unroll
  for (int o = 1; o < 32 / NE; o *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (!there) return;
  const uint32_t e = top >> 23;
  uint32_t s = e > 7u ? e - 7u : 0u;
  const float f = e == 255u ? 0.f : __uint_as_float((254u - s) << 23);   // 2^(127 - s)
#pragma unroll
  for (int j = 0; j < NE; ++j) v[j] = e == 255u ? 0.f : v[j] * f;
  uint8_t *sc = blk + act_bytes + (col >> 5);
  for (int p = 0; p < planes; ++p) {
    uint32_t q[(NE + 3) / 4];
#pragma unroll
    for (int h = 0; h < NE / 2; ++h) {
      uint16_t a;
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(a) : "f"(v[2 * h + 1]), "f"(v[2 * h]));
      q[h >> 1] = h & 1 ? q[h >> 1] | (uint32_t)a << 16 : a;
      uint32_t back;
      asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(back) : "h"(a));
      const float2 fa = __half22float2(*reinterpret_cast<const __half2 *>(&back));
      v[2 * h] -= fa.x;
      v[2 * h + 1] -= fa.y;
    }
    const int c = p * Mc + m;
    uint8_t *d = blk + c * kMxTileK + (((col >> 4) ^ (c & 7)) << 4) + (col & 15);
    if constexpr (NE == 8) *reinterpret_cast<uint2 *>(d) = make_uint2(q[0], q[1]);
    else if constexpr (NE == 4) *reinterpret_cast<uint32_t *>(d) = q[0];
    else *reinterpret_cast<uint16_t *>(d) = (uint16_t)q[0];
    if ((col & 31) == 0) sc[(c >> 7) * 512 + (c & 31) * 16 + ((c >> 5) & 3) * 4] = (uint8_t)(e == 255u ? 255u : s);
    const uint32_t next = s > 4u ? s - 4u : 0u;
    const float up = __uint_as_float((127u + s - next) << 23);
#pragma unroll
    for (int j = 0; j < NE; ++j) v[j] *= up;
    s = next;
  }
}

// The same for a kernel that leaves its output as planes: row m and columns of the whole matrix, the elements as the bf16 planes beside
// them have them.  By whole warps.
template <int NE>
__device__ __forceinline__ void mx_put(const MxOut &o, int m, int col, const __nv_bfloat16 (&hi)[NE], const __nv_bfloat16 (&lo)[NE], int bf16_planes) {
  float v[NE];
#pragma unroll
  for (int j = 0; j < NE; ++j) v[j] = __bfloat162float(hi[j]) + (bf16_planes == 2 ? __bfloat162float(lo[j]) : 0.f);
  const int z = m / o.Mc, ncols = o.planes * o.Mc;
  mx_to_planes<NE>(v, true, o.out + ((size_t)z * o.n_kb + (col >> 7)) * mx_x_block(ncols), ncols * kMxTileK, o.Mc, o.planes, m - z * o.Mc, col & 127);
}
__device__ __forceinline__ void mx_clear_flags(const MxOut &o, int thread, int threads) {
  for (int i = thread; i < o.n_flags; i += threads) o.flags[i] = 0;
}

// What becomes of four finished sums: row mg, features n .. n + 3 (a warp's lanes hold 128 consecutive ones)
template <int EPI> __device__ __forceinline__ void mx_finish(const MxArgs &g, long long mg, int n, const float (&v)[4], int lane) {
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
    if (g.mo.out) {
      const __nv_bfloat16 hi[2] = {h0, h1}, lo[2] = {l0, l1};
      mx_put<2>(g.mo, (int)mg, f, hi, lo, g.out_planes);
    }
  }
}
#endif

// How a product is dealt out: activation rows per chunk (a multiple of 8, planes x rows one of 16), chunks; runs of k-blocks
// (stream; apart: a launch per chunk) or a tile to each of `ctas` clusters; whether it makes the planes itself.
struct MxPlan { int Mc, chunks, ctas, cluster; bool stream, apart, own; };
// fits[c]: clusters of c CTAs that the device runs at once, two CTAs to an SM (mx_fits); null: none are made.  alone: no kernel before the product
// could leave the planes.
MxPlan mx_plan(int M, int tiles, int n_kb, int planes, int n_sms, const int *fits, bool alone);
void mx_fits(int (&fits)[9]);

// Activations, and the scratch memory of a product with them: planes, and for products dealt out in runs flags and slabs.
struct MxInput {
  const void *x;
  int type, rows, cols;
  long long ldx, pair;   // (see MxArgs)
};
struct MxScratch { uint64_t flags, slabs, bytes; };
MxScratch mx_scratch(int n_kb, int planes, const MxPlan &p);
// Enough for products with matrices of `tiles` x `n_kb` blocks or fewer with up to `rows` rows, whatever the device.
uint64_t mx_scratch_most(int rows, int tiles, int n_kb, int planes);
constexpr int kMxMostSms = 256;
// whether rows of 16- or 32-bit elements can be read 16 bytes at a time
inline bool mx_aligned(const void *p, long long ld, int type) { return ((uintptr_t)p & 15) == 0 && ld * (type == MX_F32 ? 4 : 2) % 16 == 0; }

// `tw`: the matrix's elements, blocks of 128 x 128, widened to bytes by the copy, 128-byte swizzle.
// Before it, unless the plan says `own`, launch_mx_input.  `g` holds the matrix, err, stamp and the outputs; launches: how many.
cudaError_t launch_mx_product(int epi, const CUtensorMap &tw, MxArgs g, const MxInput &in, void *scratch, const MxPlan &p, cudaStream_t st,
                              bool pdl, int *launches);
// early: as in MxArgs; else the product is let start when all that came before this kernel is done.
cudaError_t launch_mx_input(const MxInput &in, void *scratch, const MxPlan &p, bool early, cudaStream_t st, bool pdl);
// ... or what makes the input leaves it there.
MxOut mx_out(int n_kb, int planes, void *scratch, const MxPlan &p);

cudaError_t launch_mx_quantise(const void *x, int type, int rows, int cols, long long ldx, uint8_t *codes, uint8_t *scales, cudaStream_t st);
cudaError_t launch_mx_dequantise(const uint8_t *codes, const uint8_t *scales, int rows, int cols, void *y, int type, long long ldy,
                                 cudaStream_t st);
// Rows [r0, r0 + n_rows) of a quantised matrix with nb MX blocks a row (codes, scales: the first of these rows) into the blocks of
// the laid-out matrix (rm as for launch_retile).
cudaError_t launch_mx_lay_out(const uint8_t *codes, const uint8_t *scales, int n_rows, int r0, int nb, RowMap rm, uint8_t *w, cudaStream_t st);
// The descriptor of a laid-out matrix of `blocks` blocks; returns a CUresult.
int mx_weight_map(CUtensorMap *map, const void *data, uint64_t blocks);

// Planes (mx_planes8_kernel) lie in blocks as the product's shared memory holds them: [chunk of Mc rows][128 columns] { elements [column c
// of the instruction = plane * Mc + row][128 bytes, 16-byte pieces swizzled: piece ^ (c & 7)], scales [c / 128][lane c % 32]
// [word c / 32 % 4][4 bytes, one per MX block] }.  Rows behind the last one of a chunk stay as they are.

}  // namespace ts
