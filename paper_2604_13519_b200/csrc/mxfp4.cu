// MXFP4 conversions (quantise, dequantise, the product's storage, activations as planes of e4m3) and the entry points of the operators
// on MXFP4 matrices.  The conversions are bound by memory traffic: one pass, eight elements per thread, 16-byte accesses where
// alignment allows.  24576 x 4096 from bf16 and back to fp32, 657 MB: 123 us (5.3 TB/s); 4096 x 4096 to bf16, 42 MB: 9.4 us.
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>
#include <cstring>

#include "mxfp4.h"
#include "toolspec.h"

namespace ts {
ts_status set_error(ts_status code, const char *fmt, ...);   // model.cu

namespace {

constexpr int kConvThreads = 256, kConvUnroll = 4;   // groups of eight elements: a block's threads take four each

// How the conversions walk a matrix.
//   kFlat: rows follow one another and end with whole MX blocks: one long row.  kRows: rows can be read 16 bytes at a time.  In both a
//   thread takes eight elements at a time, four neighbouring threads an MX block, and a block of threads four such rounds.
//   kLanes: any alignment.  A lane takes one element, a warp an MX block, eight blocks at a time, so that accesses stay contiguous (with
//   eight elements per thread a warp's stores of four bytes each went to 32 sectors: 2047 x 8190 fp32 72 us).
enum : int { kFlat = 0, kRows = 1, kLanes = 2 };

// Where group u of a block's groups of eight lies: row and first column.  (One 64-bit division per block, 32-bit ones per group.)
struct Place { long long row; int col; };
struct Placer {
  long long row0;
  uint32_t off, per;
  __device__ Placer(int groups_per_row) {
    const long long g0 = (long long)blockIdx.x * (kConvThreads * kConvUnroll);
    per = groups_per_row;
    row0 = g0 / per;
    off = (uint32_t)(g0 - row0 * per);
  }
  __device__ Place at(int u) const {
    const uint32_t l = off + u, r = l / per;
    return Place{row0 + r, (int)(l - r * per) * 8};
  }
};

// Eight fp32 values -> eight e2m1 codes (round to nearest even, saturating), the first in the lowest four bits
__device__ __forceinline__ uint32_t to_e2m1x8(const float (&v)[8]) {
  uint32_t d;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(d)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return d;
}
__device__ __forceinline__ uint32_t to_e2m1x2(float lo, float hi) {
  uint32_t d;
  asm("{\n\t.reg .b8 a;\n\tcvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tmov.b32 %0, {a, a, a, a};\n\t}" : "=r"(d) : "f"(lo), "f"(hi));
  return d & 255u;
}
// Two codes -> two fp32 values
__device__ __forceinline__ float2 from_e2m1x2(uint32_t byte) {
  uint32_t h;
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\t}" : "=r"(h) : "r"(byte));
  return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}

// The largest magnitude of an MX block is found on the bits (a NaN is larger than an infinity, which is larger than all numbers); its
// exponent field e gives the scale byte: floor(log2) - 2 + 127 = e - 2, at least 0 (numbers below 2^-125 and zeros), 255 where the
// block has an infinity or NaN.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  const uint32_t e = top >> 23;
  return e == 255u ? 255u : (e > 2u ? e - 2u : 0u);
}
// 2^(127 - s): exact, and no result that matters is subnormal
__device__ __forceinline__ float scale_inverse(uint32_t s) { return s == 255u ? 0.f : __uint_as_float((254u - s) << 23); }
// 2^(s - 127); 2^-127 is subnormal
__device__ __forceinline__ float scale_value(uint32_t s) {
  return s == 255u ? __uint_as_float(0x7fc00000u) : s == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(s << 23);
}

template <int TYPE, int MODE>
__global__ void __launch_bounds__(kConvThreads)
mx_quantise_kernel(const typename MxElem<TYPE>::raw *x, long long rows, int cols, long long ldx, int nb, uint8_t *codes, uint8_t *scales,
                   long long groups) {
  if constexpr (MODE == kLanes) {
    // groups: of eight MX blocks, per * rows of them
    const uint32_t w = blockIdx.x * (kConvThreads / 32) + (threadIdx.x >> 5), per = (nb + 8) / 8, row = w / per;   // (fewer than 2^32 fit any memory)
    const int lane = threadIdx.x & 31, b0 = (int)(w - row * per) * 8;
    if (row >= rows) return;
    const typename MxElem<TYPE>::raw *p = x + row * ldx;
    uint8_t *row_codes = codes + ((long long)row * nb + b0) * 16, *row_scales = scales + (long long)row * nb + b0;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = (b0 + i) * kMxBlock + lane;
      v[i] = c < cols ? mx_to_f32<TYPE>(p[c]) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (b0 + i >= nb) break;
      const uint32_t s = scale_byte(__reduce_max_sync(0xffffffffu, __float_as_uint(v[i]) & 0x7fffffffu));
      const float u = s == 255u ? 0.f : v[i] * scale_inverse(s);
      const float next = __shfl_down_sync(0xffffffffu, u, 1);
      if ((lane & 1) == 0) row_codes[i * 16 + (lane >> 1)] = (uint8_t)to_e2m1x2(u, next);
      if (lane == 0) row_scales[i] = (uint8_t)s;
    }
  } else {
    const long long g0 = (long long)blockIdx.x * (kConvThreads * kConvUnroll) + threadIdx.x;
    MxRaw8<TYPE> raw[kConvUnroll];
    long long at[kConvUnroll];   // the group's number in codes, -1: none
    if constexpr (MODE == kFlat) {
#pragma unroll
      for (int i = 0; i < kConvUnroll; ++i) {
        at[i] = g0 + i * kConvThreads < groups ? g0 + i * kConvThreads : -1;
        mx_fetch8<TYPE>(x + (at[i] < 0 ? 0 : at[i]) * 8, 0, at[i] >= 0, 0, 8, true, raw[i]);
      }
    } else {
      const Placer pl(4 * nb);
#pragma unroll
      for (int i = 0; i < kConvUnroll; ++i) {
        const Place q = pl.at(i * kConvThreads + threadIdx.x);
        at[i] = q.row < rows ? q.row * (4ll * nb) + (q.col >> 3) : -1;
        mx_fetch8<TYPE>(x + (at[i] < 0 ? 0 : q.row) * ldx, 0, at[i] >= 0, q.col, cols, true, raw[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < kConvUnroll; ++i) {
      float v[8];
      mx_widen8<TYPE>(raw[i], v);
      uint32_t top = 0;
      if constexpr (TYPE == MX_BF16) {   // (two at a time: their bits are the upper halves of fp32's)
        const uint32_t *h = raw[i].w;
        uint32_t m = __vmaxu2(__vmaxu2(h[0] & 0x7fff7fffu, h[1] & 0x7fff7fffu), __vmaxu2(h[2] & 0x7fff7fffu, h[3] & 0x7fff7fffu));
        top = max(m & 0xffff0000u, m << 16);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
      }
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const uint32_t s = scale_byte(top);
      const float f = scale_inverse(s);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = s == 255u ? 0.f : v[j] * f;
      const uint32_t c = to_e2m1x8(v);
      if (at[i] >= 0) {
        reinterpret_cast<uint32_t *>(codes)[at[i]] = c;
        if ((threadIdx.x & 3) == 0) scales[at[i] >> 2] = (uint8_t)s;
      }
    }
  }
}

template <int TYPE, int MODE>
__global__ void __launch_bounds__(kConvThreads)
mx_dequantise_kernel(const uint8_t *codes, const uint8_t *scales, long long rows, int cols, int nb, typename MxElem<TYPE>::raw *y, long long ldy,
                     long long groups) {
  typedef typename MxElem<TYPE>::raw raw;
  if constexpr (MODE == kLanes) {
    // A warp takes 256 elements as the other modes do, eight to a lane, and turns them in shared memory.  They begin at a multiple of 32
    // elements in memory, wherever a row begins, so that the stores are whole lines.
    __shared__ float turned[kConvThreads / 32][256 + 8];
    const uint32_t w = blockIdx.x * (kConvThreads / 32) + (threadIdx.x >> 5), per = (nb + 8) / 8, row = w / per;
    if (row >= rows) return;
    const int lane = threadIdx.x & 31;
    raw *d = y + row * ldy;
    float *mine = turned[threadIdx.x >> 5];
    // the warp's columns c0 .. c0 + 255 lie in the groups of eight from g0 on, `off` elements into them
    const int c0 = (int)(w - row * per) * 256 - (int)((uintptr_t)d / sizeof(raw) % 32), g0 = c0 >> 3, off = c0 & 7;
    const uint32_t *row_codes = reinterpret_cast<const uint32_t *>(codes) + (long long)row * nb * 4;
    const uint8_t *row_scales = scales + (long long)row * nb;
    for (int g = lane; g < 33; g += 32) {
      const int at = max(0, min(g0 + g, 4 * nb - 1));
      const uint32_t c = __ldg(row_codes + at);
      const float f = scale_value(__ldg(row_scales + (at >> 2)));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 t = from_e2m1x2(c >> (8 * j));
        mine[8 * g + 2 * j] = t.x * f;
        mine[8 * g + 2 * j + 1] = t.y * f;
      }
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int col = c0 + 32 * i + lane;
      if (col >= 0 && col < cols) d[col] = mx_from_f32<TYPE>(mine[off + 32 * i + lane]);
    }
  } else {
    const long long g0 = (long long)blockIdx.x * (kConvThreads * kConvUnroll) + threadIdx.x;
    uint32_t c[kConvUnroll], s[kConvUnroll];
    long long at[kConvUnroll];
    raw *d[kConvUnroll];
    int left[kConvUnroll];   // elements of the row from the group's first on
    if constexpr (MODE == kFlat) {
#pragma unroll
      for (int i = 0; i < kConvUnroll; ++i) {
        at[i] = g0 + i * kConvThreads < groups ? g0 + i * kConvThreads : -1;
        d[i] = y + at[i] * 8;
        left[i] = 8;
      }
    } else {
      const Placer pl(4 * nb);
#pragma unroll
      for (int i = 0; i < kConvUnroll; ++i) {
        const Place q = pl.at(i * kConvThreads + threadIdx.x);
        at[i] = q.row < rows && q.col < cols ? q.row * (4ll * nb) + (q.col >> 3) : -1;
        d[i] = y + q.row * ldy + q.col;
        left[i] = cols - q.col;
      }
    }
#pragma unroll
    for (int i = 0; i < kConvUnroll; ++i) {
      c[i] = at[i] < 0 ? 0 : __ldg(reinterpret_cast<const uint32_t *>(codes) + at[i]);
      s[i] = at[i] < 0 ? 0 : __ldg(scales + (at[i] >> 2));
    }
#pragma unroll
    for (int i = 0; i < kConvUnroll; ++i) {
      if (at[i] < 0) continue;
      const float f = scale_value(s[i]);
      uint32_t w[sizeof(raw) * 2];   // the eight elements, in words
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 t = from_e2m1x2(c[i] >> (8 * j));
        if constexpr (sizeof(raw) == 4) {
          w[2 * j] = mx_from_f32<TYPE>(t.x * f);
          w[2 * j + 1] = mx_from_f32<TYPE>(t.y * f);
        } else {
          w[j] = mx_from_f32<TYPE>(t.x * f) | (uint32_t)mx_from_f32<TYPE>(t.y * f) << 16;
        }
      }
      if (left[i] >= 8) {
        if (sizeof(raw) == 4 && ((uintptr_t)d[i] & 31) == 0) {
          st_global_v8(reinterpret_cast<float *>(d[i]), w);   // (whole sectors)
        } else {
#pragma unroll
          for (int j = 0; j < (int)sizeof(raw) / 2; ++j) reinterpret_cast<uint4 *>(d[i])[j] = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < left[i]) d[i][j] = (raw)(sizeof(raw) == 4 ? w[j] : w[j >> 1] >> (16 * (j & 1)));
      }
    }
  }
}

// One thread per (row, MX block), four neighbouring threads on a row's 64 bytes of a block.  Rows [n_rows, n_fill) and MX blocks
// [nb, 4 n_kb) of the storage are filled with zeros.
__global__ void __launch_bounds__(256)
mx_lay_out_kernel(const uint4 *codes, const uint8_t *scales, int n_rows, int n_fill, int r0, int nb, int n_kb, RowMap rm, uint8_t *w) {
  const int i = blockIdx.x * 32 + (threadIdx.x >> 3), b = blockIdx.y * 8 + (threadIdx.x & 7);
  if (i >= n_fill || b >= 4 * n_kb) return;
  const int r = r0 + i;
  int row;
  if (rm.hd) {
    const int e = r % rm.hd, half = rm.hd >> 1;
    row = rm.base + (r / rm.hd) * rm.hd + (e < half ? 2 * e : 2 * (e - half) + 1);
  } else {
    row = rm.base + r * rm.mul;
  }
  const bool there = i < n_rows && b < nb;
  uint8_t *blk = w + (size_t)mx_block(row >> 7, b >> 2, n_kb) * kMxTileBytes;
  *reinterpret_cast<uint4 *>(blk + (row & 127) * 64 + (b & 3) * 16) = there ? codes[(size_t)i * nb + b] : make_uint4(0, 0, 0, 0);
  blk[mx_scale_at(row & 127) + (b & 3)] = there ? scales[(size_t)i * nb + b] : 0;
}

// The activations of a product as planes, eight elements per thread.  Clears n_flags words at `flags`.
template <int TYPE, bool VEC>
__global__ void __launch_bounds__(kConvThreads)
mx_planes8_kernel(const typename MxElem<TYPE>::raw *x, long long rows, int cols, long long ldx, long long pair, uint8_t *out, int ldo, int Mc,
                  int planes, int *flags, int n_flags, bool early) {
  // (the product waits for this kernel's end before it reads activations, but fetches weights at once)
  if (early) pdl_launch_dependents();
  pdl_wait();   // (x may come from the kernel before, whose activations may be in the same scratch memory)
  if (!early) pdl_launch_dependents();
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < n_flags; i += kConvThreads) flags[i] = 0;
  const long long i = (long long)blockIdx.x * kConvThreads + threadIdx.x;
  const int per = ldo / 8;
  const long long row = i / per;
  const int col = (int)(i - row * per) * 8;
  MxRaw8<TYPE> x8;
  float v[8];
  mx_fetch8<TYPE>(x + row * ldx, pair, row < rows, col, cols, VEC, x8);
  mx_widen8<TYPE>(x8, v);
  const int z = (int)(row / Mc), m = (int)(row - (long long)z * Mc), ncols = planes * Mc;
  mx_to_planes(v, row < rows, out + ((size_t)z * (ldo >> 7) + (col >> 7)) * mx_x_block(ncols), ncols * kMxTileK, Mc, planes, m, col & 127);
}

unsigned conv_blocks(long long rows, int per_row) {
  return (unsigned)((rows * per_row + kConvThreads * kConvUnroll - 1) / (kConvThreads * kConvUnroll));
}

}  // namespace

#define MX_BY_TYPE(type, vec, F)                                                 \
  switch (type) {                                                                \
    case MX_BF16: if (vec) F(MX_BF16, true); else F(MX_BF16, false); break;      \
    case MX_F16: if (vec) F(MX_F16, true); else F(MX_F16, false); break;         \
    default: if (vec) F(MX_F32, true); else F(MX_F32, false); break;             \
  }
#define MX_BY_MODE(type, mode, F)                                                                                               \
  switch (type) {                                                                                                               \
    case MX_BF16: if (mode == kFlat) F(MX_BF16, kFlat); else if (mode == kRows) F(MX_BF16, kRows); else F(MX_BF16, kLanes); break;  \
    case MX_F16: if (mode == kFlat) F(MX_F16, kFlat); else if (mode == kRows) F(MX_F16, kRows); else F(MX_F16, kLanes); break;      \
    default: if (mode == kFlat) F(MX_F32, kFlat); else if (mode == kRows) F(MX_F32, kRows); else F(MX_F32, kLanes); break;          \
  }

// How a matrix is walked, and the blocks of threads that takes.
static int conv_mode(const void *p, int type, int rows, int cols, long long ld, unsigned *blocks, long long *groups) {
  const int nb = (cols + kMxBlock - 1) / kMxBlock;
  *groups = (long long)rows * 4 * nb;
  const int mode = !mx_aligned(p, ld, type) ? kLanes : cols % kMxBlock == 0 && (ld == cols || rows == 1) ? kFlat : kRows;
  if (mode == kLanes) {
    const long long warps = (long long)rows * ((nb + 8) / 8);   // (a row to be read takes one in eight MX blocks, one to be written may take one more)
    *blocks = (unsigned)((warps + kConvThreads / 32 - 1) / (kConvThreads / 32));
  } else {
    *blocks = conv_blocks(rows, 4 * nb);
  }
  return mode;
}

cudaError_t launch_mx_quantise(const void *x, int type, int rows, int cols, long long ldx, uint8_t *codes, uint8_t *scales, cudaStream_t st) {
  const int nb = (cols + kMxBlock - 1) / kMxBlock;
  if (rows <= 0 || cols <= 0) return cudaSuccess;
  unsigned blocks;
  long long groups;
  const int mode = conv_mode(x, type, rows, cols, ldx, &blocks, &groups);
#define F(T, V) mx_quantise_kernel<T, V><<<blocks, kConvThreads, 0, st>>>((const MxElem<T>::raw *)x, rows, cols, ldx, nb, codes, scales, groups)
  MX_BY_MODE(type, mode, F)
#undef F
  return cudaGetLastError();
}

cudaError_t launch_mx_dequantise(const uint8_t *codes, const uint8_t *scales, int rows, int cols, void *y, int type, long long ldy,
                                 cudaStream_t st) {
  const int nb = (cols + kMxBlock - 1) / kMxBlock;
  if (rows <= 0 || cols <= 0) return cudaSuccess;
  unsigned blocks;
  long long groups;
  const int mode = conv_mode(y, type, rows, cols, ldy, &blocks, &groups);
#define F(T, V) mx_dequantise_kernel<T, V><<<blocks, kConvThreads, 0, st>>>(codes, scales, rows, cols, nb, (MxElem<T>::raw *)y, ldy, groups)
  MX_BY_MODE(type, mode, F)
#undef F
  return cudaGetLastError();
}

static cudaError_t lay_out(const uint8_t *codes, const uint8_t *scales, int n_rows, int n_fill, int r0, int nb, RowMap rm, uint8_t *w, cudaStream_t st) {
  if (n_fill <= 0) return cudaSuccess;
  const int n_kb = (nb + 3) / 4;
  mx_lay_out_kernel<<<dim3((n_fill + 31) / 32, (4 * n_kb + 7) / 8), 256, 0, st>>>((const uint4 *)codes, scales, n_rows, n_fill, r0, nb, n_kb, rm, w);
  return cudaGetLastError();
}
cudaError_t launch_mx_lay_out(const uint8_t *codes, const uint8_t *scales, int n_rows, int r0, int nb, RowMap rm, uint8_t *w, cudaStream_t st) {
  return lay_out(codes, scales, n_rows, n_rows, r0, nb, rm, w, st);
}

template <int TYPE, bool VEC>
static cudaError_t planes8(const MxInput &in, uint8_t *out, int Mc, int *flags, int n_flags, bool early, cudaStream_t st, bool pdl) {
  const int ldo = (in.cols + kMxTileK - 1) / kMxTileK * kMxTileK;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(((long long)in.rows * (ldo / 8) + kConvThreads - 1) / kConvThreads));
  cfg.blockDim = dim3(kConvThreads);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = pdl ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, mx_planes8_kernel<TYPE, VEC>, (const typename MxElem<TYPE>::raw *)in.x, (long long)in.rows, in.cols, in.ldx, in.pair,
                            out, ldo, Mc, mx_planes_of(TYPE), flags, n_flags, early);
}
cudaError_t launch_mx_input(const MxInput &in, void *scratch, const MxPlan &p, bool early, cudaStream_t st, bool pdl) {
  const MxScratch w = mx_scratch((in.cols + kMxTileK - 1) / kMxTileK, mx_planes_of(in.type), p);
  uint8_t *out = (uint8_t *)scratch;
  int *flags = (int *)(out + w.flags);
  const int n_flags = p.stream ? (p.apart ? p.chunks : 1) * p.ctas : 0;
  const bool vec = mx_aligned(in.x, in.ldx, in.type) && (in.type != MX_PAIR || in.pair % 8 == 0);
  if (in.type == MX_PAIR) return vec ? planes8<MX_PAIR, true>(in, out, p.Mc, flags, n_flags, early, st, pdl) : planes8<MX_PAIR, false>(in, out, p.Mc, flags, n_flags, early, st, pdl);
#define F(T, V) return planes8<T, V>(in, out, p.Mc, flags, n_flags, early, st, pdl)
  MX_BY_TYPE(in.type, vec, F)
#undef F
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static std::atomic<EncodeTiledFn> g_encode{nullptr};
static EncodeTiledFn encode_fn() {
  EncodeTiledFn fn = g_encode.load(std::memory_order_acquire);
  if (!fn) {   // (two threads that come here at once find the same)
    void *p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) return nullptr;
    fn = (EncodeTiledFn)p;
    g_encode.store(fn, std::memory_order_release);
  }
  return fn;
}
int mx_weight_map(CUtensorMap *map, const void *data, uint64_t blocks) {
  const EncodeTiledFn encode = encode_fn();
  if (!encode) return CUDA_ERROR_NOT_FOUND;
  const cuuint64_t dims[3] = {kMxTileK, kMxTileN, blocks}, strides[2] = {kMxTileK / 2, kMxTileBytes};
  const cuuint32_t box[3] = {kMxTileK, kMxTileN, 1}, es[3] = {1, 1, 1};
  return (int)encode(map, CU_TENSOR_MAP_DATA_TYPE_16U4_ALIGN16B, 3, const_cast<void *>(data), dims, strides, box, es,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

}  // namespace ts

// ---- entry points ---------------------------------------------------------------------------------------------------------------
namespace {

using ts::set_error;

constexpr int64_t kMostSide = 1 << 21;   // rows and columns of a matrix

// What a device offers, asked for once per device.
struct MxDevice {
  int sms = 0;
  int fits[9] = {};   // (see mx_plan)
};
constexpr int kMaxDevices = 64;
MxDevice g_dev[kMaxDevices];
std::atomic<uint64_t> g_dev_known{0};

ts_status device_of_call(MxDevice *out) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return set_error(TS_ERR_CUDA, "cudaGetDevice: %s", cudaGetErrorString(e));
  if (dev < 0 || dev >= kMaxDevices) return set_error(TS_ERR_ARG, "device ordinal %d not supported", dev);
  if (!((g_dev_known.load(std::memory_order_acquire) >> dev) & 1)) {
    int major = 0, sms = 0;
    e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return set_error(TS_ERR_CUDA, "cudaDeviceGetAttribute: %s", cudaGetErrorString(e));
    if (major != 10) return set_error(TS_ERR_CUDA, "device is not an sm_100 part; this library is built for sm_100a only");
    g_dev[dev].sms = sms;   // (two threads that come here at once store the same)
    ts::mx_fits(g_dev[dev].fits);
    g_dev_known.fetch_or(1ull << dev, std::memory_order_release);
  }
  *out = g_dev[dev];
  return TS_OK;
}

bool type_ok(int32_t t) { return t == TS_MX_BF16 || t == TS_MX_F16 || t == TS_MX_F32; }
size_t type_size(int32_t t) { return t == TS_MX_F32 ? 4 : 2; }

ts_status matrix_ok(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0 || rows > kMostSide || cols > kMostSide)
    return set_error(TS_ERR_ARG, "matrix of %lld x %lld: sides must be 0 to %lld", (long long)rows, (long long)cols, (long long)kMostSide);
  return TS_OK;
}
ts_status strided_ok(const char *name, const void *p, int32_t type, int64_t rows, int64_t cols, int64_t ld) {
  if (!type_ok(type)) return set_error(TS_ERR_ARG, "%s: unknown element type %d", name, type);
  if (ld < cols) return set_error(TS_ERR_ARG, "%s: row stride %lld is less than the row's %lld elements", name, (long long)ld, (long long)cols);
  if (rows && cols && !p) return set_error(TS_ERR_ARG, "%s is null", name);
  if ((uintptr_t)p % type_size(type)) return set_error(TS_ERR_ARG, "%s is not aligned to its elements", name);
  return TS_OK;
}
ts_status packed_ok(const void *codes, const void *scales, int64_t rows, int64_t cols) {
  if (!rows || !cols) return TS_OK;
  if (!codes || !scales) return set_error(TS_ERR_ARG, "codes or scales are null");
  if ((uintptr_t)codes % 16) return set_error(TS_ERR_ARG, "codes must be 16-byte aligned");
  return TS_OK;
}
uint64_t tiles_of(int64_t n) { return (uint64_t)(n + ts::kMxTileN - 1) / ts::kMxTileN; }
uint64_t kblocks_of(int64_t k) { return (uint64_t)(k + ts::kMxTileK - 1) / ts::kMxTileK; }

#define MX_TRY(call)                                                                                      \
  do {                                                                                                    \
    cudaError_t e_ = (call);                                                                              \
    if (e_ != cudaSuccess) return set_error(TS_ERR_CUDA, "%s: %s", #call, cudaGetErrorString(e_));        \
  } while (0)
#define MX_OK(call)                     \
  do {                                  \
    ts_status s_ = (call);              \
    if (s_ != TS_OK) return s_;         \
  } while (0)

}  // namespace

extern "C" {

ts_status ts_mxfp4_quantise(const void *x, int32_t x_type, int64_t rows, int64_t cols, int64_t ldx, void *codes, void *scales, void *stream) {
  MX_OK(matrix_ok(rows, cols));
  MX_OK(strided_ok("x", x, x_type, rows, cols, ldx));
  MX_OK(packed_ok(codes, scales, rows, cols));
  MxDevice d;
  MX_OK(device_of_call(&d));
  MX_TRY(ts::launch_mx_quantise(x, x_type, (int)rows, (int)cols, ldx, (uint8_t *)codes, (uint8_t *)scales, (cudaStream_t)stream));
  return TS_OK;
}

ts_status ts_mxfp4_dequantise(const void *codes, const void *scales, int64_t rows, int64_t cols, void *y, int32_t y_type, int64_t ldy, void *stream) {
  MX_OK(matrix_ok(rows, cols));
  MX_OK(strided_ok("y", y, y_type, rows, cols, ldy));
  MX_OK(packed_ok(codes, scales, rows, cols));
  MxDevice d;
  MX_OK(device_of_call(&d));
  MX_TRY(ts::launch_mx_dequantise((const uint8_t *)codes, (const uint8_t *)scales, (int)rows, (int)cols, y, y_type, ldy, (cudaStream_t)stream));
  return TS_OK;
}

ts_status ts_mxfp4_matrix_bytes(int64_t n, int64_t k, uint64_t *bytes) {
  if (!bytes) return set_error(TS_ERR_ARG, "null argument");
  MX_OK(matrix_ok(n, k));
  *bytes = tiles_of(n) * kblocks_of(k) * ts::kMxTileBytes;
  return TS_OK;
}

ts_status ts_mxfp4_lay_out(const void *codes, const void *scales, int64_t n, int64_t k, void *matrix, void *stream) {
  MX_OK(matrix_ok(n, k));
  MX_OK(packed_ok(codes, scales, n, k));
  if (!n || !k) return TS_OK;
  if (!matrix || (uintptr_t)matrix % 128) return set_error(TS_ERR_ARG, "matrix is null or not 128-byte aligned");
  MxDevice d;
  MX_OK(device_of_call(&d));
  const int tiles = (int)tiles_of(n);
  MX_TRY(ts::lay_out((const uint8_t *)codes, (const uint8_t *)scales, (int)n, tiles * ts::kMxTileN, 0, (int)((k + 31) / 32),
                     ts::RowMap{0, 1, 0, tiles}, (uint8_t *)matrix, (cudaStream_t)stream));
  return TS_OK;
}

ts_status ts_mxfp4_matrix_init(ts_mxfp4_matrix *m, const void *data, int64_t n, int64_t k) {
  if (!m) return set_error(TS_ERR_ARG, "null argument");
  MX_OK(matrix_ok(n, k));
  std::memset(m, 0, sizeof *m);
  m->n = n;
  m->k = k;
  if (!n || !k) return TS_OK;
  if (!data || (uintptr_t)data % 128) return set_error(TS_ERR_ARG, "matrix is null or not 128-byte aligned");
  MxDevice d;
  MX_OK(device_of_call(&d));
  CUtensorMap map;
  static_assert(sizeof map == sizeof m->map, "a descriptor has 128 bytes");
  const CUresult r = (CUresult)ts::mx_weight_map(&map, data, tiles_of(n) * kblocks_of(k));
  if (r != CUDA_SUCCESS) return set_error(TS_ERR_CUDA, "cuTensorMapEncodeTiled failed with code %d", (int)r);
  m->data = data;
  std::memcpy(m->map, &map, sizeof map);
  return TS_OK;
}

ts_status ts_mxfp4_product_workspace(int64_t rows, int64_t n, int64_t k, int32_t x_type, uint64_t *bytes) {
  if (!bytes) return set_error(TS_ERR_ARG, "null argument");
  MX_OK(matrix_ok(n, k));
  MX_OK(matrix_ok(rows, k));
  if (!type_ok(x_type)) return set_error(TS_ERR_ARG, "unknown element type %d", x_type);
  *bytes = ts::mx_scratch_most((int)rows, (int)tiles_of(n), (int)kblocks_of(k), ts::mx_planes_of(x_type));
  return TS_OK;
}

ts_status ts_mxfp4_product(const ts_mxfp4_product_args *a, void *stream) {
  if (!a || !a->matrix) return set_error(TS_ERR_ARG, "null argument");
  const ts_mxfp4_matrix *w = a->matrix;
  const int64_t M = a->rows, N = w->n, K = w->k;
  MX_OK(matrix_ok(N, K));
  MX_OK(matrix_ok(M, K));
  MX_OK(strided_ok("x", a->x, a->x_type, M, K, a->ldx));
  MX_OK(strided_ok("y", a->y, a->y_type, M, N, a->ldy));
  if ((uintptr_t)a->status % 4) return set_error(TS_ERR_ARG, "status is not aligned");
  if (!M || !N) return TS_OK;
  cudaStream_t st = (cudaStream_t)stream;
  MxDevice d;
  MX_OK(device_of_call(&d));
  if (!K) {   // an empty sum
    MX_TRY(cudaMemset2DAsync(a->y, a->ldy * type_size(a->y_type), 0, N * type_size(a->y_type), M, st));
    return TS_OK;
  }
  if (!w->data) return set_error(TS_ERR_ARG, "the matrix has no data");

  ts::MxArgs g{};
  g.w = (const uint8_t *)w->data;
  g.N = (int)N;
  g.tiles = (int)tiles_of(N); g.n_kb = (int)kblocks_of(K);
  g.err = a->status;
  g.y = a->y; g.ldy = a->ldy; g.y_type = a->y_type;
  const size_t ysz = type_size(a->y_type);
  g.vec = a->ldy % 4 == 0 && (uintptr_t)a->y % (4 * ysz) == 0;
  const ts::MxInput in{a->x, a->x_type, (int)M, (int)K, a->ldx, 0};
  const int planes = ts::mx_planes_of(a->x_type);
  const ts::MxPlan p = ts::mx_plan((int)M, g.tiles, g.n_kb, planes, d.sms, d.fits, true);
  const uint64_t need = ts::mx_scratch(g.n_kb, planes, p).bytes;
  if (need && (!a->workspace || a->workspace_bytes < need || (uintptr_t)a->workspace % 128))
    return set_error(TS_ERR_ARG, "workspace of %llu bytes, 128-byte aligned, needed for these rows", (unsigned long long)need);
  // (the matrix may have been laid out by the kernel just before: nothing of it is read until that is done)
  g.early = !p.own;
  if (!p.own) MX_TRY(ts::launch_mx_input(in, a->workspace, p, false, st, true));
  CUtensorMap tw;
  std::memcpy(&tw, w->map, sizeof tw);
  MX_TRY(ts::launch_mx_product(ts::MX_STORE, tw, g, in, a->workspace, p, st, true, nullptr));
  return TS_OK;
}

}  // extern "C"
