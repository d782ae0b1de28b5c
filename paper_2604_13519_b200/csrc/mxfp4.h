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

// A laid-out matrix of N x K: ceil(N / 128) x ceil(K / 128) blocks, k-block major (as the bf16 matrices are, see w_block).  Inside a
// block: codes [4 MX blocks][128 rows][16 bytes], scales [128 rows][4 MX blocks].
//
// The 32 codes of a row and MX block are four words of eight, in the order in which a thread takes them apart (mx_unpack): the low
// half of word i holds elements 8i, 8i + 2, 8i + 4, 8i + 6, the high half those after them, each half with the bits of its four
// elements at
//     element 0: sign 15, code 8..6    1: sign 12, code 5..3    2: sign 9, code 2..0    3: sign 14, code bits 13, 11, 10
// so that three of the four pairs come out as bf16 (sign at 15, the code's exponent and mantissa bits at 8..6) with one shift and one
// mask for both halves, and the fourth with three of each: 11 logical instructions and four multiplications for eight weights.
// Nibbles in their plain order take 16.
__host__ __device__ inline uint32_t mx_place(uint32_t nib, int j) {   // the 16-bit half's bits of element j
  const uint32_t s = nib >> 3, c = nib & 7;
  switch (j) {
    case 0: return s << 15 | c << 6;
    case 1: return s << 12 | c << 3;
    case 2: return s << 9 | c;
    default: return s << 14 | (c >> 2) << 13 | (c & 3) << 10;
  }
}

enum : int { MX_BF16 = 0, MX_F16 = 1, MX_F32 = 2 };   // element types of activations and results (TS_MX_*)

struct MxArgs {
  const uint8_t *w;       // laid-out matrix
  int N, M;               // features, activation rows
  int tiles, n_kb;        // 128-row tiles and 128-column blocks of the matrix
  int Mc, planes;         // activation rows per CTA (a multiple of 8, planes x Mc one of 16), bf16 planes that are added
  int stages;             // filled in by the launcher
  int *err;               // device status word (null: not wanted)
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
};
enum : int { MX_STORE = 0, MX_SWIGLU = 1, MX_LOGITS = 2 };   // what a product does with its sums

// How a product is dealt out.
struct MxPlan { int Mc, tiles_per_cta, cluster; };
MxPlan mx_plan(int M, int tiles, int n_kb, int planes, int n_sms);

// `ta`: bf16 activations [planes][rows][K], box {64, Mc, planes}, 128-byte swizzle.  cluster: CTAs along K that complete a tile's
// sums together.  tiles_per_cta: 1 or 2 weight tiles.
cudaError_t launch_mx_product(int epi, const CUtensorMap &ta, MxArgs g, int tiles_per_cta, int cluster, cudaStream_t st, bool pdl);

cudaError_t launch_mx_quantise(const void *x, int type, int rows, int cols, long long ldx, uint8_t *codes, uint8_t *scales, cudaStream_t st);
cudaError_t launch_mx_dequantise(const uint8_t *codes, const uint8_t *scales, int rows, int cols, void *y, int type, long long ldy,
                                 cudaStream_t st);
// Rows [r0, r0 + n_rows) of a quantised matrix with nb MX blocks a row (codes, scales: the first of these rows) into the blocks of
// the laid-out matrix (rm as for launch_retile).
cudaError_t launch_mx_lay_out(const uint8_t *codes, const uint8_t *scales, int n_rows, int r0, int nb, RowMap rm, uint8_t *w, cudaStream_t st);
// x [rows][cols] (row stride ldx) as bf16 planes whose sum is x: out [planes][rows][ldo]
cudaError_t launch_mx_planes(const void *x, int type, int rows, int cols, long long ldx, __nv_bfloat16 *out, int ldo, int planes, cudaStream_t st);

}  // namespace ts
