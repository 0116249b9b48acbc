// Internal interface between the C-ABI front end of the rotary positions and
// the cross attention (wbmm_attn_api.cpp) and their kernels (wbmm_rotary.hip,
// wbmm_attn.hip).  Not installed, not part of the ABI.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime.h>

#include "wbmm_internal.h"

namespace wbmm {

// [B, S, H, D] tokens: address and strides in bytes, D contiguous.
struct Tokens {
  char *p;
  int64_t b, s, h;
};

constexpr int kMaxAxes = 4;
constexpr int kMaxPairs = 256;      // rotary pairs of a head
constexpr int kMaxRotaryDim = 4096; // components of a head
constexpr int kMaxHeadDim = 128;    // attention

struct RotaryArgs {
  Tokens x, y;
  const void *pos;
  int64_t pos_a, pos_b, pos_s;  // strides in elements
  int pos64;
  const float *freqs;
  int64_t B, S;
  int H, D, P, axes;
  int first[kMaxAxes];  // pairs before axis a + 1
  int adjacent;
  int reverse;  // rotate by the negative angle
};

hipError_t launch_rotary(Dt dt, const RotaryArgs &a, hipStream_t stream);

struct AttnArgs {
  Tokens q, k, v, o;
  Tokens dout, dq, dk, dv;
  float *lse;  // [B, Hq, Sq]
  const int32_t *lens;
  const uint8_t *mask;
  int64_t mask_b, mask_s;
  int64_t B;
  int Sq, Sk, Hq, Hk, G, D;
  int R;  // rows of a key head: Sq * G, row r is query r / G of head r % G
  float scale, c;  // c = scale * log2(e)
  // Rows of a workgroup's tile in the forward and for dq; with 32 of them the
  // states go in `splits` parts with partial results part_o [splits, B Hk, R, D]
  // and, forward, part_l [splits, B Hk, R] (lse in log2 units).
  int tile_rows, splits;
  int one_pass;  // backward: one kernel for all gradients, of `splits` parts
  int powers;    // backward: sum_do and top_v are taken
  float *part_o, *part_l;
  // backward: two statistics per row, [B Hk, R]; for float16's powers of two
  // sums of |dout| per row and the largest |v| of 32 states, [B Hk, ceil(Sk / 32)]
  float2 *rowstat;
  float *sum_do, *top_v;
  // backward: dk, dv in `row_parts` parts of the rows, with partial sums
  // part_dk, part_dv [row_parts, B Hk, Sk, D]
  int row_parts;
  float *part_dk, *part_dv;
};

// Rows of a key head whose gradients are taken in one pass over the states
// (16-bit), for heads of D components: dq of all rows is held in registers
// beside dk and dv of a block.  Twice the rows need the registers of two waves
// or spill, and were slower: 1024 heads of 128 components, 64 rows, 784 states
// 772 us against 333 in separate kernels; 64 components, 128 rows 203 against 202;
// 32 components, 100 rows 69 against 99.  64 components of 64 rows spill
// 9 registers of 256 as it is.
constexpr int one_pass_rows(int D) { return D <= 32 ? 128 : D <= 64 ? 64 : 32; }

template <class Tag>
struct AttnEntry {
  // VEC: rows of all tensors are whole 16-byte pieces
  template <bool VEC> static hipError_t forward(const AttnArgs &a, hipStream_t stream);
  template <bool VEC> static hipError_t backward(const AttnArgs &a, hipStream_t stream);
};

// Tiles and parts of a call (functions of its sizes alone).
void attn_plan_forward(Dt dt, AttnArgs *a);
void attn_plan_backward(Dt dt, AttnArgs *a);
// Whether every launch of a planned call is within the grid's limits.
bool attn_grids_fit(const AttnArgs &a, bool back);

}  // namespace wbmm
