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
  // forward: the states of a sequence in `splits` parts with partial results
  // part_o [splits, B Hk, R, D], part_l [splits, B Hk, R] (log2 units)
  int splits;
  float *part_o, *part_l;
  // backward: per row {lse in log2 units, delta}, [B Hk, R]
  float2 *rowstat;
  // backward: dk, dv in `row_parts` parts of the rows, partial sums float32
  // part_dk, part_dv [row_parts, B Hk, Sk, D]
  int row_parts;
  float *part_dk, *part_dv;
  int vec;  // 16-byte accesses to rows
};

template <class Tag>
struct AttnEntry {
  static hipError_t forward(const AttnArgs &a, hipStream_t stream);
  static hipError_t backward(const AttnArgs &a, hipStream_t stream);
};

// Parts of the states in a forward call, of the rows in the dk / dv pass.
int attn_splits(Dt dt, int64_t B, int Sq, int Sk, int Hq, int Hk);
int attn_row_parts(Dt dt, int64_t B, int Sq, int Sk, int Hq, int Hk);

}  // namespace wbmm
