// Cross attention kernels for gfx950: device code and launchers, instantiated
// per dtype by wbmm_attn.hip.
//
// Per batch entry and key head, row r = s G + g stands for query s of head g
// of the G query heads that share the key head, so the rows of a group read
// one set of keys and values:
//   out_r = sum_j p_rj v_j,  p_rj = exp(scale q_r.k_j - lse_r)
// over the visible states j (below the sequence's length, not masked).
//
// Matrix-core layout
// ------------------
// All products run through 32 x 32 tiles (v_mfma_f32_32x32x16_{bf16,f16},
// 32x32x2_f32).  A lane's result column is l % 32, its 16 result rows are
// 8 (i / 4) + 4 h + i % 4 with h = l / 32.  Scores are taken transposed,
// S^T = K Q^T, so a lane holds scores of one query only: maxima and sums run
// inside the lane and join one partner lane.  The sum over keys of the second
// product, O^T = V^T P^T, may take the keys in any order as long as both
// operands agree; with the order in which a lane already holds them, the
// probabilities are the second operand as they are, without a shuffle.
// V^T comes from the transposing LDS reads (16-bit) or single-element reads
// (float32) of the row-major tile.
//
// LDS tiles are row-major; 16-byte chunk c of row r sits at slot c ^ swz(r).
// swz makes both kinds of reads free of bank conflicts: 16 rows at one chunk,
// and 4 rows at 64 consecutive bytes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "wbmm_attn_internal.h"
#include "wbmm_kernels.h"

namespace wbmm {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// ------------------------------------------------------------ tile geometry

template <class Tag, int DP>
struct Tile {
  static constexpr int ES = Tag::ES;
  static constexpr int CE = 16 / ES;                              // elements of a chunk
  static constexpr int PITCH = (DP == 96 ? 128 : DP) * ES;        // bytes of an LDS row
  static constexpr int LPC = PITCH / 16;                          // chunks of an LDS row
  static constexpr int NU = DP / (2 * CE);                        // chunk pairs of a row
  static constexpr int DT = DP / 32;
  // The chunk of a row that belongs at a slot.
  __host__ __device__ static constexpr int chunk_at(int slot, int row) { return slot ^ swz(row); }
  __host__ __device__ static constexpr int swz(int row) {
    if constexpr (ES == 2) {
      if constexpr (PITCH == 256) return ((row & 3) << 2) | ((row >> 2) & 3);
      if constexpr (PITCH == 128) return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
      return (row >> 2) & 3;
    } else {
      if constexpr (PITCH >= 256) return (((row >> 2) & 1) << 3) | (row & 3) | (((row >> 3) & 1) << 2);
      return (row >> 1) & 7;
    }
  }
  // Row reads: lane l reads chunk 2 u + h of row base + l % 32 (base a
  // multiple of 32) at rowlane() ^ (u << 5), plus base * PITCH.
  __device__ static int rowlane(int lane) {
    const int l31 = lane & 31, h = lane >> 5;
    return l31 * PITCH + ((h ^ swz(l31)) << 4);
  }
  // Column reads, 16-bit: four rows 16 t + 8 g + 4 h + 0..3 of column
  // 32 dt + l % 32 at (collane() ^ (dt << 6) ^ (g << 5)) + (16 t + 8 g) * PITCH.
  // float32: row 8 (i / 4) + 4 h + i % 4 of that column at
  // (collane() ^ colxor32(dt, i)) + (8 (i / 4) + i % 4) * PITCH.
  __device__ static int collane(int lane) {
    const int h = lane >> 5;
    if constexpr (ES == 2) {
      const int r = (lane >> 2) & 3, q = lane & 3, cg = (lane >> 4) & 1;
      int slot = cg * 2 + (q >> 1);
      if constexpr (PITCH == 256) slot ^= r << 2;
      if constexpr (PITCH == 128) slot ^= ((r >> 1) & 1) << 2;
      slot ^= h;
      return (4 * h + r) * PITCH + (slot << 4) + (q & 1) * 8;
    } else {
      const int l31 = lane & 31;
      const int slot = (l31 >> 2) ^ (PITCH >= 256 ? h << 3 : h << 1);
      return 4 * h * PITCH + (slot << 4) + (l31 & 3) * 4;
    }
  }
  __device__ static constexpr int colxor32(int dt, int i) {
    if (PITCH >= 256) return (dt << 7) ^ ((i % 4) << 4) ^ (((i / 4) & 1) << 6);
    return ((((i / 4) & 1) << 2) | ((i % 4) >> 1)) << 4;
  }
};

// ----------------------------------------------------------------- products

// acc += A B over one chunk pair (16 or 8 components): chunks of both halves.
template <class Tag> __device__ inline f32x16 mma_chunk(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (Tag::W16) {
    if constexpr (__is_same(Tag, TagBF16))
      return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                     0, 0);
    else
      return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0,
                                                    0, 0);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[j]), __uint_as_float(b[j]), c, 0, 0,
                                               0);
    return c;
  }
}

// Result of a 32 x 32 product over the row fragments of an LDS tile (rows
// base..base+31) with fragments in registers; `at` is the tile's offset plus
// rowlane().  (The tile is part of what the chunk's bits are xored into: the
// address costs one instruction a read, and no registers between tiles.)
template <class Tag, int DP>
__device__ inline f32x16 rows_product(const char *smem, int at, int base, const u32x4 *b, f32x16 acc = {}) {
  using T = Tile<Tag, DP>;
#pragma unroll
  for (int u = 0; u < T::NU; ++u) {
    const u32x4 a = *(const u32x4 *)(smem + (at ^ (u << 5)) + base * T::PITCH);
    acc = mma_chunk<Tag>(a, b[u], acc);
  }
  return acc;
}

// Nothing is scheduled across this point.
__device__ inline void pin_order() { __builtin_amdgcn_sched_barrier(0); }

// As rows_product for NB blocks of 32 rows, with the reads P ahead of the
// products (left to itself the compiler reads each fragment right before its
// product and waits).
template <class Tag, int DP, int NB, int P>
__device__ inline void rows_products(const char *smem, int at, int base, const u32x4 *b, f32x16 *acc) {
  using T = Tile<Tag, DP>;
  constexpr int N = T::NU * NB;
  constexpr int Q = P < N ? P : N;
  u32x4 f[Q];
  auto read = [&](int n) { return *(const u32x4 *)(smem + (at ^ ((n / NB) << 5)) + (base + 32 * (n % NB)) * T::PITCH); };
#pragma unroll
  for (int k = 0; k < NB; ++k) acc[k] = (f32x16){};
#pragma unroll
  for (int n = 0; n < Q; ++n) f[n] = read(n);
  pin_order();
#pragma unroll
  for (int n = 0; n < N; ++n) {
    acc[n % NB] = mma_chunk<Tag>(f[n % Q], b[n / NB], acc[n % NB]);
    if (n + Q < N) f[n % Q] = read(n + Q);
    pin_order();
  }
}

// Column fragment dt of rows base .. base + 15 of an LDS tile (16-bit).
template <class Tag, int DP>
__device__ inline u32x4 col_read(const char *smem, int at, int base, int dt) {
  using T = Tile<Tag, DP>;
  s16x4 v[2];
#pragma unroll
  for (int g = 0; g < 2; ++g)
    v[g] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (lds_s16x4 *)(smem + (at ^ (dt << 6) ^ (g << 5)) + (base + 8 * g) * T::PITCH));
  const u32x2 lo = __builtin_bit_cast(u32x2, v[0]), hi = __builtin_bit_cast(u32x2, v[1]);
  return (u32x4){lo[0], lo[1], hi[0], hi[1]};
}

// Column fragments of rows base .. base + 15 of an LDS tile.
template <class Tag, int DP>
__device__ inline void cols_read(const char *smem, int at, int base, u32x4 *f) {
#pragma unroll
  for (int dt = 0; dt < Tile<Tag, DP>::DT; ++dt) f[dt] = col_read<Tag, DP>(smem, at, base, dt);
}

// Second operand over 32 rows made of a lane's 16 results.
template <class Tag> struct Weights { u32x4 w[2]; };
template <> struct Weights<TagF32> { f32x16 w; };
template <class Tag> __device__ inline Weights<Tag> to_weights(const f32x16 &p) {
  Weights<Tag> r;
  if constexpr (Tag::W16) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) r.w[t][j] = pack2<Tag>(p[8 * t + 2 * j], p[8 * t + 2 * j + 1]);
  } else {
    r.w = p;
  }
  return r;
}

// acc[dt] += (columns of the LDS tile's rows base..base+31)^T weights; `at` is
// the tile's offset plus collane().
template <class Tag, int DP>
__device__ inline void cols_product(const char *smem, int at, int base, const Weights<Tag> &p, f32x16 *acc) {
  using T = Tile<Tag, DP>;
  if constexpr (Tag::W16) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int dt = 0; dt < T::DT; ++dt) {
        s16x4 v[2];
#pragma unroll
        for (int g = 0; g < 2; ++g)
          v[g] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (lds_s16x4 *)(smem + (at ^ (dt << 6) ^ (g << 5)) + (base + 16 * t + 8 * g) * T::PITCH));
        const u32x2 lo = __builtin_bit_cast(u32x2, v[0]), hi = __builtin_bit_cast(u32x2, v[1]);
        const u32x4 a = {lo[0], lo[1], hi[0], hi[1]};
        acc[dt] = mma_chunk<Tag>(a, p.w[t], acc[dt]);
      }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int dt = 0; dt < T::DT; ++dt) {
        const float a =
            *(const float *)(smem + (at ^ T::colxor32(dt, i)) + (base + 8 * (i / 4) + i % 4) * T::PITCH);
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, p.w[i], acc[dt], 0, 0, 0);
      }
  }
}

// ------------------------------------------------------------------- memory

// Chunk (16 bytes from component d0 on) of a row of D components; what lies
// past D is zero.  VEC: rows are whole 16-byte pieces.  (A template parameter
// of the kernels: with both forms in one kernel, short calls spent more time
// on fetching code than on their work.)
template <class Tag, bool VEC>
__device__ inline u32x4 load_chunk(const char *row, int d0, int D) {
  u32x4 v = {0, 0, 0, 0};
  if (d0 >= D) return v;
  if constexpr (VEC) return *(const u32x4 *)(row + d0 * Tag::ES);
  if constexpr (Tag::W16) {
    const u16 *p = (const u16 *)row + d0;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (d0 + j < D) v[j / 2] |= (uint32_t)p[j] << (16 * (j & 1));
  } else {
    const uint32_t *p = (const uint32_t *)row + d0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (d0 + j < D) v[j] = p[j];
  }
  return v;
}

template <class Tag, bool VEC>
__device__ inline void store_chunk(char *row, int d0, int D, u32x4 v) {
  if (d0 >= D) return;
  if constexpr (VEC) {
    *(u32x4 *)(row + d0 * Tag::ES) = v;
  } else if constexpr (Tag::W16) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (d0 + j < D) ((u16 *)row)[d0 + j] = (u16)(v[j / 2] >> (16 * (j & 1)));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (d0 + j < D) ((uint32_t *)row)[d0 + j] = v[j];
  }
}

template <class Tag> __device__ inline void store1(char *row, int d, float v) {
  if constexpr (Tag::W16)
    ((u16 *)row)[d] = (u16)pack2<Tag>(v, 0.f);
  else
    ((float *)row)[d] = v;
}

// Order between a wave's own writes and reads of LDS that no other wave uses.
__device__ inline void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Results of 32 rows (lane: row l % 32, components 32 dt + 8 (i / 4) + 4 h +
// i % 4), multiplied by f, rounded once and stored through this wave's piece of
// LDS (32 rows), so that each row leaves in whole 16-byte pieces of
// neighbouring lanes.  row_at(n): address of row n, or null.  Rows whose bit in
// `keep` is not set are stored as zeros.
template <class Tag, int DP, bool VEC, class RowAt>
__device__ inline void store_rows(char *piece, const f32x16 *acc, float f, int D, int lane, RowAt row_at,
                                  uint32_t keep = 0xffffffffu) {
  using T = Tile<Tag, DP>;
  const int h = lane >> 5, l31 = lane & 31;
#pragma unroll
  for (int dt = 0; dt < T::DT; ++dt)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const float a = acc[dt][i] * f, b = acc[dt][i + 1] * f, c = acc[dt][i + 2] * f, d = acc[dt][i + 3] * f;
      const int byte = (32 * dt + 2 * i + 4 * h) * Tag::ES;  // a half chunk (16-bit) or a chunk
      char *at = piece + l31 * T::PITCH + ((((byte >> 4) ^ T::swz(l31)) << 4) | (byte & 15));
      if constexpr (Tag::W16)
        *(u32x2 *)at = (u32x2){pack2<Tag>(a, b), pack2<Tag>(c, d)};
      else
        *(f32x4 *)at = (f32x4){a, b, c, d};
    }
  wave_lds_fence();
  constexpr int RPP = 64 / T::LPC, NP = 32 / RPP;
  const int c = lane % T::LPC;
  u32x4 v[NP];
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int rw = p * RPP + lane / T::LPC;
    v[p] = *(const u32x4 *)(piece + rw * T::PITCH + ((c ^ T::swz(rw)) << 4));
  }
  if (keep != 0xffffffffu) {
#pragma unroll
    for (int p = 0; p < NP; ++p)
      if (!((keep >> (p * RPP + lane / T::LPC)) & 1)) v[p] = (u32x4){0, 0, 0, 0};
  }
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    char *row = row_at(p * RPP + lane / T::LPC);
    if (row) store_chunk<Tag, VEC>(row, c * T::CE, D, v[p]);
  }
  wave_lds_fence();
}

// A tile of ROWS rows on its way from memory to LDS through registers.
template <class Tag, int DP, int ROWS, int THREADS>
struct Mover {
  using T = Tile<Tag, DP>;
  static constexpr int RPP = THREADS / T::LPC;  // rows a pass
  static constexpr int NP = (ROWS + RPP - 1) / RPP;
  u32x4 r[NP];
  __host__ __device__ static constexpr int chunk(int tid) { return tid % T::LPC; }
  __host__ __device__ static constexpr int row(int tid, int p) { return tid / T::LPC + p * RPP; }
  // zeroes chunks past D
  __device__ void cut(int D, int tid) {
    if (D <= (T::LPC - 1) * T::CE && chunk(tid) * T::CE >= D) {
#pragma unroll
      for (int p = 0; p < NP; ++p) r[p] = (u32x4){0, 0, 0, 0};
    }
  }
  // zeroes rows from n on
  __device__ void cut_rows(int n, int tid) {
#pragma unroll
    for (int p = 0; p < NP; ++p)
      if (row(tid, p) >= n) r[p] = (u32x4){0, 0, 0, 0};
  }
  __device__ void store(char *tile, int tid) const {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int rw = row(tid, p);
      if (ROWS % RPP == 0 || rw < ROWS)
        *(u32x4 *)(tile + rw * T::PITCH + ((chunk(tid) ^ T::swz(rw)) << 4)) = r[p];
    }
  }
};

// Rows first .. first + ROWS - 1 of the states of one head.  Every lane loads:
// rows from `end` on repeat the last one, chunks past D the row's first, so
// the loads stand side by side without branches (rows in whole pieces; others
// go element by element, under masks).  hide() zeroes what must not be seen on
// the way to LDS: rows whose bit in `see` is not set, since a masked state may
// hold anything, and chunks past D.
template <class Tag, int DP, bool VEC, int ROWS, int THREADS>
struct StateMover : Mover<Tag, DP, ROWS, THREADS> {
  using M = Mover<Tag, DP, ROWS, THREADS>;
  __device__ void load(const char *base, int64_t stride, int first, int end, int D, int tid) {
    const int d0 = M::chunk(tid) * M::T::CE;
    if constexpr (VEC) base += (d0 < D ? d0 : 0) * Tag::ES;
#pragma unroll
    for (int p = 0; p < M::NP; ++p) {
      const int n = first + M::row(tid, p), j = n < end ? n : end - 1;
      if constexpr (VEC)
        this->r[p] = *(const u32x4 *)(base + j * stride);
      else
        this->r[p] = load_chunk<Tag, VEC>(base + j * stride, d0, D);
    }
  }
  __device__ void hide(bool rows, uint64_t see, int D, int tid) {
    if (rows) {
#pragma unroll
      for (int p = 0; p < M::NP; ++p)
        if (!((see >> (M::row(tid, p) & 63)) & 1)) this->r[p] = (u32x4){0, 0, 0, 0};
    }
    this->cut(D, tid);
  }
};

// ----------------------------------------------- from memory straight to LDS
//
// Tiles of whole 16-byte pieces skip the registers: each lane names the 16
// bytes that belong at its place in LDS, so the swizzle is in the choice of the
// chunk.  This frees the registers of the tile in flight (32 of 256 in the
// forward at 128 components), and a head of 72 components, padded to 96, takes
// less time than one of 128.  Lanes whose chunk lies past D do not load; their
// places are zeroed once.  Rows that must not be seen are zeroed in LDS when
// they have arrived, by the lanes that loaded them.  Written as
// assembly because the compiler, which cannot tell the two halves of the
// double buffer apart, would wait for the loads of the next tile before each
// read of the present one.  `lds` is the wave's first byte; lane l's piece goes
// 16 l bytes behind it.  The pause covers a base or M0 that a vector instruction
// wrote just before (five wait states), which the compiler cannot see to.
__device__ inline void lds_load16(uint32_t lds, const char *base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(offset), "s"(base) : "m0");
}
__device__ inline void lds_load16(uint32_t lds, const char *at) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(lds), "v"(at) : "m0");
}
// The wave's loads have arrived (a barrier then tells the others).
__device__ inline void lds_loads_done() { asm volatile("s_waitcnt vmcnt(0)" : : : "memory"); }

__device__ inline uint32_t lds_offset(const char *p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char *)p;
}

// Places of a thread in tiles of ROWS rows that four waves load.  PLAIN: D = DP
// and no mask, known ahead, so that every place has its piece where the tile's
// rows are as long as the tensors'.  (96 components lie in rows of 128, whose
// last chunks have nothing behind them in memory.)
template <class Tag, int DP, int ROWS, bool PLAIN>
struct DirectTile {
  using M = Mover<Tag, DP, ROWS, 256>;
  __host__ __device__ static constexpr bool has(int tid, int p, int D) {
    if (PLAIN && M::T::PITCH == DP * Tag::ES) return true;
    // (the swizzle has a period of 16 rows)
    return M::T::chunk_at(M::chunk(tid), M::row(tid, M::RPP % 16 == 0 ? 0 : p)) * M::T::CE < (PLAIN ? DP : D);
  }
  // Zeroes the places past D of `tiles` tiles.
  __device__ static void clear(char *tile, int tiles, int D, int tid) {
    if (PLAIN || D == DP) return;
#pragma unroll
    for (int p = 0; p < M::NP; ++p)
      if ((ROWS % M::RPP == 0 || M::row(tid, p) < ROWS) && !has(tid, p, D))
        for (int n = 0; n < tiles; ++n) *(u32x4 *)(tile + n * ROWS * M::T::PITCH + p * 4096 + tid * 16) = (u32x4){0, 0, 0, 0};
  }
  // Zeroes the rows that must not be seen.  (Nothing of it is to be computed
  // ahead of the loop and kept there.)
  __device__ static void hide(char *tile, uint64_t see, int tid) {
    asm volatile("" : "+v"(tid));
#pragma unroll
    for (int p = 0; p < M::NP; ++p)
      if ((ROWS % M::RPP == 0 || M::row(tid, p) < ROWS) && !((see >> (M::row(tid, p) & 63)) & 1))
        *(u32x4 *)(tile + p * 4096 + tid * 16) = (u32x4){0, 0, 0, 0};
  }
};

// A tile of ROWS states by four waves.  Strides are below 2^24 bytes (the
// front end checks), so a lane's offset in a tile fits 32 bits.  ANEW: a lane's
// places are worked out anew for each tile, where a kernel has no registers to
// keep them in (the gradients: 128 components, 512 queries over 1001 masked
// states 143 -> 135 us; the forward, which has: 790 -> 835 us).
template <class Tag, int DP, int ROWS, bool PLAIN, bool ANEW>
struct DirectStates : DirectTile<Tag, DP, ROWS, PLAIN> {
  using M = Mover<Tag, DP, ROWS, 256>;
  static_assert(ROWS % M::RPP == 0, "whole passes");
  __device__ static void load(uint32_t lds, const char *base, int64_t stride, int first, int end, int D, int tid, int wave) {
    if constexpr (ANEW) asm volatile("" : "+v"(tid));
    const int c = M::chunk(tid);
    const char *tile = base + first * stride;
#pragma unroll
    for (int p = 0; p < M::NP; ++p) {
      const int rw = M::row(tid, p), last = end - 1 - first, j = rw < last ? rw : last;
      if (DirectTile<Tag, DP, ROWS, PLAIN>::has(tid, p, D))
        lds_load16(lds + p * 4096 + wave * 1024, tile, (uint32_t)j * (uint32_t)stride + (M::T::chunk_at(c, rw) << 4));
    }
  }
};

__device__ inline float other_half_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false,
                                                  false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ inline float other_half_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false,
                                                  false);
  return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}
__device__ inline float exp2_(float v) { return __builtin_amdgcn_exp2f(v); }

// Visibility of the n <= 64 states from `first` on: the mask's byte of lane's
// state is loaded ahead, like the rows, and the bits are formed when they are
// needed, alike in all lanes.
__device__ inline uint32_t load_sight(const uint8_t *mask, int64_t mask_s, int first, int n, int len, int lane) {
  return mask && lane < n && first + lane < len ? mask[(first + lane) * mask_s] : 1;
}
__device__ inline uint64_t sight_bits(uint32_t sight, int first, int n, int len, int lane) {
  return __ballot(lane < n && first + lane < len && sight);
}

// Workgroup `id` of `n` onto a unit of work such that each die (workgroups
// are dealt to the eight in turn) takes one run of consecutive units, which
// share keys and values in its L2.
__device__ inline int64_t unit_of(int64_t id, int64_t n) {
  const int64_t per = n >> 3, rem = n & 7, die = id & 7, slot = id >> 3;
  return die * per + (die < rem ? die : rem) + slot;
}

__device__ inline int length_of(const AttnArgs &a, int64_t b) {
  int len = a.Sk;
  if (a.lens) {
    len = a.lens[b];
    len = len < 0 ? 0 : len > a.Sk ? a.Sk : len;
  }
  return len;
}

// The chunks 2 u + h of one row, zeros past D.  (D > DP - 32, so only the last
// chunks can lie past it.)
template <class Tag, int DP, bool VEC>
__device__ inline void load_row(const char *row, int D, int lane, u32x4 *f) {
  using T = Tile<Tag, DP>;
  const int h = lane >> 5;
#pragma unroll
  for (int u = 0; u < T::NU; ++u) {
    const int d0 = (2 * u + h) * T::CE;
    if constexpr (!VEC)
      f[u] = load_chunk<Tag, VEC>(row, d0, D);
    else if ((2 * u + 2) * T::CE <= DP - 32)
      f[u] = *(const u32x4 *)(row + d0 * Tag::ES);
    else
      f[u] = *(const u32x4 *)(row + (d0 < D ? d0 : 0) * Tag::ES);
  }
  if constexpr (VEC) {
    if (D < DP) {
#pragma unroll
      for (int u = 0; u < T::NU; ++u)
        if ((2 * u + 2) * T::CE > DP - 32 && (2 * u + h) * T::CE >= D) f[u] = (u32x4){0, 0, 0, 0};
    }
  }
}

// Row fragments of 32 rows of a group (second operand): lane l has chunks
// 2 u + h of row r; rows from R on repeat the last one, in columns of results
// that nobody reads.
template <class Tag, int DP, bool VEC>
__device__ inline void load_rows(const AttnArgs &a, const Tokens &t, int64_t b, int hk, int r, int lane, u32x4 *f) {
  const int at = r < a.R ? r : a.R - 1, s = at / a.G, g = at - s * a.G;
  load_row<Tag, DP, VEC>(t.p + b * t.b + s * t.s + (int64_t)(hk * a.G + g) * t.h, a.D, lane, f);
}

// The fragments have arrived.  (Loads still under way when a loop is entered
// make the compiler wait inside it, every time round, and that wait would take
// in the loads of the next tile.)
template <int N> __device__ inline void arrived(u32x4 (&f)[N]) {
#pragma unroll
  for (int u = 0; u < N; ++u) asm volatile("" : "+v"(f[u]));
}

// Address of row r of a group in an output, or null past the last.
__device__ inline char *group_row(const AttnArgs &a, const Tokens &t, int64_t b, int hk, int r) {
  if (r >= a.R) return nullptr;
  const int s = r / a.G, g = r - s * a.G;
  return t.p + b * t.b + s * t.s + (int64_t)(hk * a.G + g) * t.h;
}

// Scores of 32 states (one lane: 16 of one query) to weights: running maximum
// `top` (in log2 units, with lag) and the lane's part of the sum.  Returns
// through `scale` what the earlier results have to be multiplied by where any
// lane's maximum moved.
constexpr float kLag = 8.f;
// float16 weights are kept 2^6 larger, up to 2^14, away from the type's
// smallest numbers.
template <class Tag> constexpr float kRaise = __is_same(Tag, TagF16) ? 6.f : 0.f;

template <int NB>
__device__ inline bool running_top(const f32x16 *s, float c, float *top, float *fix) {
  float m = s[0][0];
#pragma unroll
  for (int k = 0; k < NB; ++k)
#pragma unroll
    for (int i = 0; i < 16; ++i) m = fmaxf(m, s[k][i]);
  m = other_half_max(m) * c;
  // The maximum may lag by up to kLag: weights then reach 2^kLag, which costs
  // no precision in floating point, and nearly all tiles skip the rescaling.
  const bool move = m > *top + kLag;
  if (!__any(move)) return false;
  const float t = fmaxf(*top, m);
  *fix = t == -INFINITY ? 1.f : exp2_(*top - t);
  *top = t;
  return true;
}

// ------------------------------------------------------------------ forward

// A workgroup takes 32 (4 / WK) rows and runs over the states in tiles of BN,
// double-buffered in LDS, the next tile on its way: straight to LDS (VEC) or
// in registers.  WK waves share 32 rows and split each tile's states, joined at
// the end.  32 rows a wave leave room for two waves a SIMD, of two workgroups,
// whose softmax and products overlap without further arrangement.
// Measured, bfloat16, 128 components, 4 x 32 heads of 2048 queries over 6272
// states: 780 us, 1.08 PFLOP/s, where a large library product reaches 1.24.
// The matrix cores are busy 56 % of the cycles, the vector units 57 %, and the
// clock has fallen to 1.82 GHz (from 2.04 at 49 %): what bounds it is power.
// Ablations, of 777 us: no softmax 676, no tile loads 702, no fragment reads
// 695; products alone 478.  Scores of the next tile taken during the softmax of this
// one, with or without a pinned interleaving: 820 to 850 us.
template <class Tag, int DP, int WK>
struct FwdShape {
  static constexpr int WR = 4 / WK;
  static constexpr int BM = 32 * WR;
  static constexpr int KW = Tag::W16 && WK == 1 ? 64 : 32;  // states of a wave per tile
  static constexpr int BN = KW * WK;
  static constexpr int NB = KW / 32;
  static constexpr int TILE = BN * Tile<Tag, DP>::PITCH;
  static constexpr int LDS = 4 * TILE;
};

template <class Tag, int DP, int WK, bool VEC, bool PLAIN>
__global__ __launch_bounds__(256, 2) void attn_fwd_kernel(AttnArgs a) {
  using T = Tile<Tag, DP>;
  using F = FwdShape<Tag, DP, WK>;
  using Direct = DirectStates<Tag, DP, F::BN, PLAIN, false>;
  constexpr int NB = F::NB, DT = T::DT;
  extern __shared__ __align__(512) char attn_smem[];
  char *const smem = attn_smem;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = wave % F::WR, wk = wave / F::WR, h = lane >> 5;
  const int tiles = (a.R + F::BM - 1) / F::BM;
  const int64_t unit = unit_of(blockIdx.x, gridDim.x), bh = unit / tiles;
  const int rt = (int)(unit - bh * tiles);
  const int64_t b = bh / a.Hk;
  const int hk = (int)(bh - b * a.Hk);
  const int len = length_of(a, b);
  const int t1 = (len + F::BN - 1) / F::BN;
  const int r = rt * F::BM + wr * 32 + (lane & 31);

  u32x4 qf[T::NU];
  load_rows<Tag, DP, VEC>(a, a.q, b, hk, r, lane, qf);
  const char *kb = a.k.p + b * a.k.b + hk * a.k.h, *vb = a.v.p + b * a.v.b + hk * a.v.h;
  const uint8_t *mask = !PLAIN && a.mask ? a.mask + b * a.mask_b : nullptr;
  StateMover<Tag, DP, VEC, F::BN, 256> mk, mv;
  uint32_t sight = 1;
  const int rowlane = T::rowlane(lane), collane = T::collane(lane);

  f32x16 acc[DT] = {};
  float top = -INFINITY, sum = 0.f;
  auto load = [&](int t) {
    sight = load_sight(mask, a.mask_s, t * F::BN, F::BN, len, lane);
    if constexpr (VEC) {
      const uint32_t to = lds_offset(smem) + (t & 1) * 2 * F::TILE;
      Direct::load(to, kb, a.k.s, t * F::BN, len, a.D, tid, wave);
      Direct::load(to + F::TILE, vb, a.v.s, t * F::BN, len, a.D, tid, wave);
    } else {
      mk.load(kb, a.k.s, t * F::BN, len, a.D, tid);
      mv.load(vb, a.v.s, t * F::BN, len, a.D, tid);
    }
  };
  if constexpr (VEC) Direct::clear(smem, 4, a.D, tid);
  if (t1 > 0) load(0);
  arrived(qf);
  for (int t = 0; t < t1; ++t) {
    const int kt = (t & 1) * 2 * F::TILE, vt = kt + F::TILE;
    uint64_t see = ~(uint64_t)0;
    if (mask || (t + 1) * F::BN > len) see = sight_bits(sight, t * F::BN, F::BN, len, lane);
    const bool hide = see != ~(uint64_t)0;
    if constexpr (VEC) {
      lds_loads_done();
      if (hide) Direct::hide(smem + vt, see, tid);
    } else {
      mk.hide(hide, see, a.D, tid);
      mv.hide(hide, see, a.D, tid);
      mk.store(smem + kt, tid);
      mv.store(smem + vt, tid);
    }
    __syncthreads();
    if (t + 1 < t1) load(t + 1);
    f32x16 s[NB];
    rows_products<Tag, DP, NB, Tag::W16 ? 8 : 4>(smem, kt + rowlane, wk * F::KW, qf, s);
    if (hide) {
#pragma unroll
      for (int k = 0; k < NB; ++k) {
        const uint32_t bits = (uint32_t)(see >> (wk * F::KW + 32 * k)) >> (4 * h);
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (!((bits >> (8 * (i / 4) + i % 4)) & 1)) s[k][i] = -INFINITY;
      }
    }
    u32x4 vf[2][DT];
    if constexpr (Tag::W16) {
      cols_read<Tag, DP>(smem, vt + collane, wk * F::KW, vf[0]);
      pin_order();
    }
    float fix;
    if (running_top<NB>(s, a.c, &top, &fix)) {
      sum *= fix;
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[d] *= fix;
    }
    const float sub = top == -INFINITY ? 0.f : top - kRaise<Tag>;
    if constexpr (Tag::W16) {
      // Eight weights at a time: those of the next step are formed while the
      // matrix cores take this step's.  They are rounded to the inputs' type for
      // the product; their sum is taken before that, in float32.
      u32x4 w[2];
      auto weights = [&](int n, u32x4 *to) {
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = exp2_(__builtin_fmaf(s[n / 2][8 * (n & 1) + i], a.c, -sub));
        sum += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
#pragma unroll
        for (int j = 0; j < 4; ++j) (*to)[j] = pack2<Tag>(p[2 * j], p[2 * j + 1]);
      };
      weights(0, &w[0]);
#pragma unroll
      for (int n = 0; n < 2 * NB; ++n) {
        if (n + 1 < 2 * NB) cols_read<Tag, DP>(smem, vt + collane, wk * F::KW + 16 * (n + 1), vf[(n + 1) & 1]);
        pin_order();
#pragma unroll
        for (int d = 0; d < DT; ++d) acc[d] = mma_chunk<Tag>(vf[n & 1][d], w[n & 1], acc[d]);
        if (n + 1 < 2 * NB) weights(n + 1, &w[(n + 1) & 1]);

        pin_order();
      }
    } else {
#pragma unroll
      for (int k = 0; k < NB; ++k) {
        float part[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[k][i] = exp2_(__builtin_fmaf(s[k][i], a.c, -sub));
          part[i & 1] += s[k][i];
        }
        sum += part[0] + part[1];
        cols_product<Tag, DP>(smem, vt + collane, wk * F::KW + 32 * k, to_weights<Tag>(s[k]), acc);
      }
    }
  }
  sum = other_half_sum(sum);

  if constexpr (WK > 1) {
    // join the waves that share rows
    float *xo = (float *)smem;  // [wave][16 DT][64], then top and sum
    constexpr int PER = (16 * DT + 2) * 64;
    static_assert((4 - F::WR) * PER * 4 <= F::LDS, "the waves' results fit the tiles' space");
    __syncthreads();
    if (wk > 0) {
      float *o = xo + (wave - F::WR) * PER + lane;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[(d * 16 + i) * 64] = acc[d][i];
      o[16 * DT * 64] = top;
      o[(16 * DT + 1) * 64] = sum;
    }
    __syncthreads();
    for (int w = 1; w < (wk > 0 ? 0 : WK); ++w) {
      const float *o = xo + (wave + (w - 1) * F::WR) * PER + lane;
      const float top2 = o[16 * DT * 64], sum2 = o[(16 * DT + 1) * 64];
      const float t = fmaxf(top, top2);
      const float f1 = top == t ? 1.f : exp2_(top - t), f2 = top2 == t ? 1.f : exp2_(top2 - t);
      sum = sum * f1 + sum2 * f2;
      top = t;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = acc[d][i] * f1 + o[(d * 16 + i) * 64] * f2;
    }
  }
  // a row that sees nothing: zeros, and minus infinity
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  if (a.lse && h == 0 && wk == 0 && r < a.R) {
    const int sq = r / a.G, hq = hk * a.G + r - sq * a.G;
    a.lse[(b * a.Hq + hq) * a.Sq + sq] = sum == 0.f ? -INFINITY : (top - kRaise<Tag> + __builtin_amdgcn_logf(sum)) * kLn2;
  }
  __syncthreads();
  if (wk > 0) return;
  store_rows<Tag, DP, VEC>(smem + wave * 32 * T::PITCH, acc, inv, a.D, lane,
                           [&](int n) { return group_row(a, a.o, b, hk, rt * F::BM + wr * 32 + n); });
}

// ------------------------------------------------------- forward, few rows

// Where the tiles of 128 rows would leave much of the chip idle (single
// tokens above all, whose time is the reading of the states): a workgroup
// takes 32 rows and a part of the states, in blocks of 32, and each of its
// waves every fourth block.  Keys go from memory straight into the product's
// first operand, values through a piece of LDS that only this wave uses, so
// the loop has no barrier.  The waves' results are joined through LDS, the
// parts' by attn_join_kernel.  Measured, bfloat16, 32 tokens of 32 heads over up
// to 12544 states of 8 x 128 (1.17 GB): 217 us, 5.4 TB/s.  A variant with 16-row
// products and eight waves a workgroup was no faster: a compute unit reads about
// 50 GB/s, whatever its waves.
template <class Tag, int DP>
struct FewShape {
  static constexpr int TILE = 32 * Tile<Tag, DP>::PITCH;
  static constexpr int OP = DP + 4;  // floats of a row when joining
  static int lds(int R) {
    const int tiles = 4 * TILE, rows = R < 32 ? R : 32, join = (4 * rows * OP + 256) * 4;
    return tiles > join ? tiles : join;
  }
};

// Row fragments (first operand) of the 32 states from `first` on; those from
// `len` on repeat the last one.
template <class Tag, int DP, bool VEC>
__device__ inline void load_states(const char *base, int64_t stride, int first, int len, int D, int lane, u32x4 *f) {
  const int n = first + (lane & 31);
  load_row<Tag, DP, VEC>(base + (n < len ? n : len - 1) * stride, D, lane, f);
}

template <class Tag, int DP, bool VEC>
__global__ __launch_bounds__(256, Tag::W16 || DP <= 64 ? 2 : 1) void attn_few_kernel(AttnArgs a) {
  using T = Tile<Tag, DP>;
  using F = FewShape<Tag, DP>;
  constexpr int DT = T::DT;
  extern __shared__ __align__(512) char attn_smem[];
  char *const smem = attn_smem;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5, l31 = lane & 31;
  const int tiles = (a.R + 31) / 32;
  int64_t unit = unit_of(blockIdx.x, gridDim.x);
  const int rt = (int)(unit % tiles);
  unit /= tiles;
  const int split = (int)(unit % a.splits);
  const int64_t bh = unit / a.splits;
  const int64_t b = bh / a.Hk;
  const int hk = (int)(bh - b * a.Hk);
  const int len = length_of(a, b);
  const int all = (len + 31) / 32;
  const int t0 = (int)((int64_t)all * split / a.splits), t1 = (int)((int64_t)all * (split + 1) / a.splits);
  const int rows = a.R - rt * 32 < 32 ? a.R - rt * 32 : 32;

  u32x4 qf[T::NU], kf[T::NU];
  const char *kb = a.k.p + b * a.k.b + hk * a.k.h, *vb = a.v.p + b * a.v.b + hk * a.v.h;
  const uint8_t *mask = a.mask ? a.mask + b * a.mask_b : nullptr;
  StateMover<Tag, DP, VEC, 32, 64> mv;
  const int vt = wave * F::TILE;
  uint32_t sight = 1;
  const int collane = T::collane(lane);
  f32x16 acc[DT] = {};
  float top = -INFINITY, sum = 0.f;
  int t = t0 + wave;
  if (t < t1) {
    load_states<Tag, DP, VEC>(kb, a.k.s, t * 32, len, a.D, lane, kf);
    mv.load(vb, a.v.s, t * 32, len, a.D, lane);
    sight = load_sight(mask, a.mask_s, t * 32, 32, len, lane);
  }
  load_rows<Tag, DP, VEC>(a, a.q, b, hk, rt * 32 + l31, lane, qf);
  for (; t < t1; t += 4) {
    f32x16 s = {};
#pragma unroll
    for (int u = 0; u < T::NU; ++u) s = mma_chunk<Tag>(kf[u], qf[u], s);
    uint32_t see = 0xffffffffu;
    if (mask || (t + 1) * 32 > len) see = (uint32_t)sight_bits(sight, t * 32, 32, len, lane);
    mv.hide(see != 0xffffffffu, see, a.D, lane);
    mv.store(smem + vt, lane);
    // (the next block's loads leave behind the last use of this one's: where
    // they may or may not have left, a wait would have to take them in)
    if (t + 4 < t1) {
      load_states<Tag, DP, VEC>(kb, a.k.s, (t + 4) * 32, len, a.D, lane, kf);
      mv.load(vb, a.v.s, (t + 4) * 32, len, a.D, lane);
      sight = load_sight(mask, a.mask_s, (t + 4) * 32, 32, len, lane);
    }
    if (see != 0xffffffffu) {
      const uint32_t bits = see >> (4 * h);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (!((bits >> (8 * (i / 4) + i % 4)) & 1)) s[i] = -INFINITY;
    }
    float fix;
    if (running_top<1>(&s, a.c, &top, &fix)) {
      sum *= fix;
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[d] *= fix;
    }
    const float sub = top == -INFINITY ? 0.f : top - kRaise<Tag>;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = exp2_(__builtin_fmaf(s[i], a.c, -sub));
      sum += s[i];
    }
    wave_lds_fence();
    const Weights<Tag> w = to_weights<Tag>(s);
    cols_product<Tag, DP>(smem, vt + collane, 0, w, acc);
    wave_lds_fence();
  }
  sum = other_half_sum(sum);

  // join the four waves: [wave][row][OP] results, then tops and sums
  float *xo = (float *)smem, *xt = xo + 4 * rows * F::OP, *xs = xt + 128;
  __syncthreads();
  if (l31 < rows) {
    float *o = xo + (wave * rows + l31) * F::OP;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *(f32x4 *)(o + 32 * d + 8 * (i / 4) + 4 * h) = (f32x4){acc[d][i], acc[d][i + 1], acc[d][i + 2], acc[d][i + 3]};
    if (h == 0) {
      xt[wave * 32 + l31] = top;
      xs[wave * 32 + l31] = sum;
    }
  }
  __syncthreads();
  for (int e = tid; e < rows * DP; e += 256) {
    const int n = e / DP, d = e % DP;
    if (d >= a.D) continue;
    float t4 = -INFINITY, s4 = 0.f, o4 = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) t4 = fmaxf(t4, xt[w * 32 + n]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float tw = xt[w * 32 + n];
      const float f = tw == t4 ? 1.f : exp2_(tw - t4);
      s4 += xs[w * 32 + n] * f;
      o4 += xo[(w * rows + n) * F::OP + d] * f;
    }
    // a row that sees nothing: zeros, and minus infinity
    const float inv = s4 == 0.f ? 0.f : 1.f / s4;
    const float lse2 = s4 == 0.f ? -INFINITY : t4 - kRaise<Tag> + __builtin_amdgcn_logf(s4);
    const int r = rt * 32 + n;
    if (a.splits > 1) {
      const int64_t at = (split * a.B * a.Hk + bh) * a.R + r;
      a.part_o[at * a.D + d] = o4 * inv;
      if (d == 0) a.part_l[at] = lse2;
    } else {
      store1<Tag>(group_row(a, a.o, b, hk, r), d, o4 * inv);
      const int sq = r / a.G, hq = hk * a.G + r - sq * a.G;
      if (a.lse && d == 0) a.lse[(b * a.Hq + hq) * a.Sq + sq] = lse2 * kLn2;
    }
  }
}

// Components of a row that a thread of the joining kernels takes (a thread a
// component, with its position from 64-bit divisions, spent 20 us on 25 MB).
template <bool VEC> constexpr int kJoin = VEC ? 4 : 1;
template <bool VEC> __device__ inline void load_part(const float *p, float *v) {
  if constexpr (VEC) {
    const f32x4 x = *(const f32x4 *)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = x[i];
  } else {
    v[0] = *p;
  }
}
template <class Tag, bool VEC> __device__ inline void store_part(char *row, int d, const float *v) {
  if constexpr (!VEC)
    store1<Tag>(row, d, v[0]);
  else if constexpr (Tag::W16)
    *(u32x2 *)(row + d * 2) = (u32x2){pack2<Tag>(v[0], v[1]), pack2<Tag>(v[2], v[3])};
  else
    *(f32x4 *)(row + d * 4) = (f32x4){v[0], v[1], v[2], v[3]};
}

// Joins the partial results of the splits, weighted by their shares of the
// sum, in their order.  The loads of eight splits leave together.
template <class Tag, bool VEC>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a) {
  constexpr int V = kJoin<VEC>;
  const uint32_t n = (uint32_t)a.B * a.Hk * a.R, e = blockIdx.x * 256 + threadIdx.x;  // (n D is at most 2^31)
  const uint32_t per = (uint32_t)a.D / V, row = e / per;
  if (row >= n) return;
  const int d = (int)(e - row * per) * V;
  float top = -INFINITY, sum = 0.f, o[V] = {};
  for (int s0 = 0; s0 < a.splits; s0 += 8) {
    float l[8], p[8][V];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int s = s0 + i < a.splits ? s0 + i : a.splits - 1;
      const int64_t at = (int64_t)s * n + row;
      l[i] = a.part_l[at];
      load_part<VEC>(a.part_o + at * a.D + d, p[i]);
    }
    float t = top;
#pragma unroll
    for (int i = 0; i < 8; ++i) t = fmaxf(t, l[i]);
    const float sub = t == -INFINITY ? 0.f : t, fix = exp2_(top - sub);
    sum *= fix;
#pragma unroll
    for (int k = 0; k < V; ++k) o[k] *= fix;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (s0 + i >= a.splits) continue;  // (its loads repeat the last part, which may be infinite)
      const float w = exp2_(l[i] - sub);
      sum += w;
#pragma unroll
      for (int k = 0; k < V; ++k) o[k] += w * p[i][k];
    }
    top = t;
  }
#pragma unroll
  for (int k = 0; k < V; ++k) o[k] = sum == 0.f ? 0.f : o[k] / sum;
  const uint32_t bh = row / (uint32_t)a.R, b = bh / (uint32_t)a.Hk;
  const int r = (int)(row - bh * a.R), hk = (int)(bh - b * a.Hk);
  store_part<Tag, VEC>(group_row(a, a.o, b, hk, r), d, o);
  const int sq = r / a.G, hq = hk * a.G + r - sq * a.G;
  if (a.lse && d == 0)
    a.lse[((int64_t)b * a.Hq + hq) * a.Sq + sq] = (sum == 0.f ? -INFINITY : top + __builtin_amdgcn_logf(sum)) * kLn2;
}

// ----------------------------------------------------------------- backward
//
// With p recomputed from the forward's lse, delta_r = do_r.o_r and
// ds = p (do.v - delta):  dq = scale ds K,  dk = scale ds^T Q,  dv = p^T do.
// The scores are recomputed twice, by the owners of rows for dq and by the
// owners of states for dk and dv, so every sum has one owner and a fixed order:
// no atomics, and the same bits every time.  In 16 bits delta is that of the
// rounded out (a float32 out would be an output more), off by half a step of
// each of its components, and p and ds are rounded for the matrix cores.

// Statistics of the lane's row.  16-bit: what its products start from,
// {-lse / scale, -delta}, so that they come out as the weight's exponent and as
// dp - delta, without an instruction more (float16 weights 2^12 larger, which
// the first of them takes in: kRaiseBack); a row that sees nothing starts from
// minus infinity, and its weights come out as zero.  In float32 the sums would
// round at lse's size instead of the products' own (errors of the gradients
// 1.3e-6 instead of 0.8e-6), so there it is {lse in log2 units, delta}, taken
// off afterwards.
template <class Tag> constexpr bool kStart = Tag::W16;
template <class Tag> constexpr int kRaiseBack = __is_same(Tag, TagF16) ? 12 : 0;
constexpr float kBlind = -INFINITY;  // start of a row that sees nothing; float32: its negative
template <class Tag> __device__ inline float2 blind_stat() { return make_float2(kStart<Tag> ? kBlind : -kBlind, 0.f); }

template <class Tag> __device__ inline float chunk_dot(u32x4 x, u32x4 y) {
  float d = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (Tag::W16)
      d += to_f32<Tag>((u16)(x[j] & 0xffff)) * to_f32<Tag>((u16)(y[j] & 0xffff)) +
           to_f32<Tag>((u16)(x[j] >> 16)) * to_f32<Tag>((u16)(y[j] >> 16));
    else
      d += __uint_as_float(x[j]) * __uint_as_float(y[j]);
  }
  return d;
}

// Statistics of row r of a group, whose do.o is d.
template <class Tag> __device__ inline float2 stat_of(const AttnArgs &a, int64_t b, int hk, int r, float d) {
  const int sq = r / a.G, hq = hk * a.G + r - sq * a.G;
  const float lse = a.lse[(b * a.Hq + hq) * a.Sq + sq];
  if (lse == -INFINITY) return blind_stat<Tag>();
  return kStart<Tag> ? make_float2((kRaiseBack<Tag> * kLn2 - lse) / a.scale, -d) : make_float2(lse * kLog2e, d);
}

// float16's ds.  It goes with the upstream gradient and with the weights: over
// thousands of states, or without a loss scale, it lies below the type's normal
// numbers, and with a large loss scale above its largest (64 rows over 6272
// states, dout of std 1e-3: dq off by 0.0047 of itself as it is, by 0.00031 as
// follows, where its last rounding alone makes 0.00021).  So it is multiplied by
// a power of two on its way to the product, taken from a bound that is known
// ahead: with |dp_rj| <= B = sum |do_r| max |v| over all visible states (delta
// comes from all of them), and delta_r the mean of dp_rj by p_rj,
//   |ds_rj| = p_rj (1 - p_rj) |dp_rj - mean of the others| <= B / 2,
// for dk with the largest of the rows.  The largest ds then lies below 2^15, and
// each keeps 2^-40 B of absolute precision (2^-25, half of the type's smallest
// step, over the power), where it would need 2^-11 of itself.  Powers: 2^14 over
// the bound's own power of two, at most 2^100.
template <class Tag> constexpr bool kPower = __is_same(Tag, TagF16);

__device__ inline int power_for(float bound) {  // its exponent
  const int e = (int)(__float_as_uint(bound) >> 23) & 255;  // (255: not finite)
  return 141 - (e > 41 ? e : 41);
}
// 2^e, |e| < 127
__device__ inline float exponent(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

// Sum of the magnitudes of a chunk, and their largest as a 16-bit pattern in
// either half of the result (patterns of magnitudes are in the numbers' order).
template <class Tag> __device__ inline float chunk_sum(u32x4 x) {
  float d = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    d += __builtin_fabsf(to_f32<Tag>((u16)(x[j] & 0xffff))) + __builtin_fabsf(to_f32<Tag>((u16)(x[j] >> 16)));
  return d;
}
typedef u16 u16x2 __attribute__((ext_vector_type(2)));
__device__ inline u16x2 chunk_top(u32x4 x, u16x2 top) {
#pragma unroll
  for (int j = 0; j < 4; ++j) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, x[j] & 0x7fff7fffu));
  return top;
}
__device__ inline uint32_t top_of(u16x2 top) { return top[0] > top[1] ? top[0] : top[1]; }

// Largest value of the wave, in all lanes.
template <int CTRL> __device__ inline uint32_t turned_max(uint32_t v) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false);
  return v > o ? v : o;
}
__device__ inline uint32_t wave_max(uint32_t v) {
  // rotations by 8, 4, 2, 1 within the rows of 16 lanes, then across the rows
  v = turned_max<0x121>(turned_max<0x122>(turned_max<0x124>(turned_max<0x128>(v))));
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = a[0] > a[1] ? a[0] : a[1];
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return b[0] > b[1] ? b[0] : b[1];
}
// Largest of p[first .. end), magnitudes, in all lanes; eight loads at a time.
__device__ inline float wave_top(const float *p, int first, int end, int lane) {
  float m = 0.f;
  for (int i = first + lane; i - lane < end; i += 512) {
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = p[i + 64 * k < end ? i + 64 * k : end - 1];
#pragma unroll
    for (int k = 0; k < 8; ++k) m = fmaxf(m, v[k]);
  }
  return __uint_as_float(wave_max(__float_as_uint(m)));
}

// max |v| of the visible ones of 32 states, a wave each, four states at a time
// (all loads leave together, those of hidden states too); workgroup `id` takes
// 128 states.
template <class Tag, bool VEC>
__device__ inline void take_top_v(const AttnArgs &a, uint32_t id) {
  constexpr int CE = 16 / Tag::ES;
  const uint32_t tiles = ((uint32_t)a.Sk + 127) / 128, bh = id / tiles;
  const int64_t b = bh / (uint32_t)a.Hk;
  const int lane = threadIdx.x & 63, hk = (int)(bh - (uint32_t)b * a.Hk);
  const int first = (int)(id - bh * tiles) * 128 + (int)(threadIdx.x >> 6) * 32;
  if (first >= a.Sk) return;
  const int len = length_of(a, b);
  const char *vb = a.v.p + b * a.v.b + hk * a.v.h;
  u16x2 top = {0, 0};
  u32x4 v[8];
  uint32_t see[8];
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const int n = first + 4 * p + (lane >> 4), j = n < a.Sk ? n : a.Sk - 1;
    v[p] = load_chunk<Tag, VEC>(vb + j * a.v.s, (lane & 15) * CE, a.D);
    see[p] = a.mask ? a.mask[b * a.mask_b + j * a.mask_s] : 1;
    if (j >= len) see[p] = 0;
  }
#pragma unroll
  for (int p = 0; p < 8; ++p) top = see[p] ? chunk_top(v[p], top) : top;
  const uint32_t all = wave_max(top_of(top));
  if (lane == 0) a.top_v[(int64_t)bh * ((a.Sk + 31) / 32) + first / 32] = to_f32<Tag>((u16)all);
}

// Those of all rows, ahead of the gradients: 16 lanes a row, bound by memory
// (131072 rows of 128 components, bfloat16: 15 us, 4.5 TB/s).  Taken by the
// owners of dq instead, the owners of dk and dv would have to wait for them.
// float16: the sums of |do| too, and ahead of the rows' workgroups the `of_v` of
// the states' largest values (8 x 3136 x 8 heads of 128 components: 10 us more).
template <class Tag, bool VEC>
__global__ __launch_bounds__(256) void attn_stat_kernel(AttnArgs a, uint32_t of_v) {
  constexpr int CE = 16 / Tag::ES;
  if constexpr (kPower<Tag>) {
    if (blockIdx.x < of_v) return take_top_v<Tag, VEC>(a, blockIdx.x);
  }
  const int64_t row = (int64_t)(blockIdx.x - of_v) * 16 + (threadIdx.x >> 4);
  const int lane = threadIdx.x & 15;
  if (row >= a.B * a.Hk * (int64_t)a.R) return;
  const int64_t bh = row / a.R, b = bh / a.Hk;
  const int r = (int)(row - bh * a.R), hk = (int)(bh - b * a.Hk);
  const char *o = group_row(a, a.o, b, hk, r), *g = group_row(a, a.dout, b, hk, r);
  float d = 0.f, n = 0.f;
  for (int c = lane; c * CE < a.D; c += 16) {
    const u32x4 y = load_chunk<Tag, VEC>(g, c * CE, a.D);
    d += chunk_dot<Tag>(load_chunk<Tag, VEC>(o, c * CE, a.D), y);
    if constexpr (kPower<Tag>) n += chunk_sum<Tag>(y);
  }
#pragma unroll
  for (int m = 8; m > 0; m /= 2) {
    d += __shfl_xor(d, m, 16);
    if constexpr (kPower<Tag>) n += __shfl_xor(n, m, 16);
  }
  if (lane == 0) {
    a.rowstat[row] = stat_of<Tag>(a, b, hk, r, d);
    if constexpr (kPower<Tag>) a.sum_do[row] = n;
  }
}

// The lane's row of what attn_stat_kernel left.
template <class Tag> __device__ inline float2 load_stat(const AttnArgs &a, int64_t bh, int r) {
  float2 st = blind_stat<Tag>();
  if (r < a.R) st = a.rowstat[bh * a.R + r];
  return st;
}

// The largest |v| of the head's visible states.
__device__ inline float head_top_v(const AttnArgs &a, int64_t bh, int len, int lane) {
  return wave_top(a.top_v + bh * ((a.Sk + 31) / 32), 0, (len + 31) / 32, lane);
}

// dq's power of two for the lane's row: into the statistics that its weights
// start from; returns what takes it off.
template <class Tag>
__device__ inline float raise_row(const AttnArgs &a, int64_t bh, int r, int len, int lane, float2 *st) {
  if constexpr (!kPower<Tag>) return 1.f;
  const float v = head_top_v(a, bh, len, lane);
  const int e = power_for(r < a.R ? 0.5f * a.sum_do[bh * a.R + r] * v : 0.f);
  st->x += (float)(e - kRaiseBack<Tag>) / a.c;
  return exponent(-e);
}

// (The value is made anew each time: sixteen copies of it would otherwise be
// kept in registers across a loop.)
__device__ inline f32x16 splat(float v) {
  asm volatile("" : "+v"(v));
  f32x16 r;
#pragma unroll
  for (int i = 0; i < 16; ++i) r[i] = v;
  return r;
}

// Weight of one state and ds, from what the products gave.
template <class Tag> __device__ inline float weight(float s, float c, float x) {
  return kStart<Tag> ? exp2_(s * c) : exp2_(__builtin_fmaf(s, c, -x));
}
template <class Tag> __device__ inline float ds_of(float p, float dp, float y) { return kStart<Tag> ? p * dp : p * (dp - y); }

// The products' results to ds (one lane: 16 states of one row), zero where not
// visible.
template <class Tag>
__device__ inline void to_ds(f32x16 *s, const f32x16 &dp, float c, float2 st, uint32_t seen, int h) {
#pragma unroll
  for (int i = 0; i < 16; ++i) (*s)[i] = ds_of<Tag>(weight<Tag>((*s)[i], c, st.x), dp[i], st.y);
  if (seen != 0xffffffffu) {
    const uint32_t bits = seen >> (4 * h);
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (!((bits >> (8 * (i / 4) + i % 4)) & 1)) (*s)[i] = 0.f;
  }
}

// dq: as the forward, a workgroup takes 32 (4 / WK) rows and runs over all
// states, WK waves sharing rows and splitting each tile.  Measured on its own,
// bfloat16, 8 x 32 heads of 512 queries over 3136 states of 128 components:
// 285 us for three products, 1.1 PFLOP/s.
template <class Tag, int DP, int WK, bool VEC, bool PLAIN>
__device__ inline void take_dq(const AttnArgs &a, char *smem, int64_t id, int64_t units) {
  using T = Tile<Tag, DP>;
  using F = FwdShape<Tag, DP, WK>;
  using Direct = DirectStates<Tag, DP, F::BN, PLAIN, !PLAIN>;
  constexpr int DT = T::DT, NB = F::NB;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
  const int wr = wave % F::WR, wk = wave / F::WR;
  const int tiles = (a.R + F::BM - 1) / F::BM;
  const int64_t unit = unit_of(id, units), bh = unit / tiles, b = bh / a.Hk;
  const int rt = (int)(unit - bh * tiles), hk = (int)(bh - b * a.Hk);
  const int len = length_of(a, b);
  const int t1 = (len + F::BN - 1) / F::BN;
  const int r = rt * F::BM + wr * 32 + (lane & 31);
  u32x4 qf[T::NU], gf[T::NU];
  load_rows<Tag, DP, VEC>(a, a.q, b, hk, r, lane, qf);
  load_rows<Tag, DP, VEC>(a, a.dout, b, hk, r, lane, gf);
  float2 st = load_stat<Tag>(a, bh, r);
  const char *kb = a.k.p + b * a.k.b + hk * a.k.h, *vb = a.v.p + b * a.v.b + hk * a.v.h;
  const uint8_t *mask = !PLAIN && a.mask ? a.mask + b * a.mask_b : nullptr;
  StateMover<Tag, DP, VEC, F::BN, 256> mk, mv;
  uint32_t sight = 1;
  const int rowlane = T::rowlane(lane), collane = T::collane(lane);
  f32x16 acc[DT] = {};
  auto load = [&](int t) {
    sight = load_sight(mask, a.mask_s, t * F::BN, F::BN, len, lane);
    if constexpr (VEC) {
      const uint32_t to = lds_offset(smem) + (t & 1) * 2 * F::TILE;
      Direct::load(to, kb, a.k.s, t * F::BN, len, a.D, tid, wave);
      Direct::load(to + F::TILE, vb, a.v.s, t * F::BN, len, a.D, tid, wave);
    } else {
      mk.load(kb, a.k.s, t * F::BN, len, a.D, tid);
      mv.load(vb, a.v.s, t * F::BN, len, a.D, tid);
    }
  };
  if constexpr (VEC) Direct::clear(smem, 4, a.D, tid);
  if (t1 > 0) load(0);
  const float lower = raise_row<Tag>(a, bh, r, len, lane, &st);
  arrived(qf);
  arrived(gf);
  for (int t = 0; t < t1; ++t) {
    const int kt = (t & 1) * 2 * F::TILE, vt = kt + F::TILE;
    uint64_t see = ~(uint64_t)0;
    if (mask || (t + 1) * F::BN > len) see = sight_bits(sight, t * F::BN, F::BN, len, lane);
    const bool hide = see != ~(uint64_t)0;
    if constexpr (VEC) {
      lds_loads_done();
      if (hide) Direct::hide(smem + kt, see, tid);
    } else {
      mk.hide(hide, see, a.D, tid);
      mv.hide(hide, see, a.D, tid);
      mk.store(smem + kt, tid);
      mv.store(smem + vt, tid);
    }
    __syncthreads();
    if (t + 1 < t1) load(t + 1);
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      const int base = wk * F::KW + 32 * k;
      f32x16 s = splat(kStart<Tag> ? st.x : 0.f), dp = splat(kStart<Tag> ? st.y : 0.f);
      const uint32_t seen = (uint32_t)(see >> base);
      if constexpr (Tag::W16 && VEC) {
        // One stream of fragment reads, some products ahead of their use: keys
        // for the scores, values for dp (while which the weights are formed),
        // columns of the keys for dq.
        constexpr int NU = T::NU, N = 2 * NU + 2 * DT, P = 8 < N ? 8 : N;
        u32x4 f[P], w[2];
        auto read = [&](int n) {
          if (n < 2 * NU)
            return *(const u32x4 *)(smem + (((n < NU ? kt : vt) + rowlane) ^ (n % NU << 5)) + base * T::PITCH);
          return col_read<Tag, DP>(smem, kt + collane, base + (n - 2 * NU) / DT * 16, (n - 2 * NU) % DT);
        };
        // ds of eight states, rounded to the inputs' type for the product
        const uint32_t bits = seen >> (4 * h);
        auto weights = [&](int t, u32x4 *to) {
          float ds[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) ds[i] = s[8 * t + i] * dp[8 * t + i];
          if (seen != 0xffffffffu) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (!((bits >> (16 * t + 8 * (i / 4) + i % 4)) & 1)) ds[i] = 0.f;
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) (*to)[j] = pack2<Tag>(ds[2 * j], ds[2 * j + 1]);
        };
#pragma unroll
        for (int n = 0; n < P; ++n) f[n] = read(n);
        pin_order();
#pragma unroll
        for (int n = 0; n < N; ++n) {
          if (n == 2 * NU) weights(0, &w[0]);
          if (n == 2 * NU + DT) weights(1, &w[1]);
          if (n < NU)
            s = mma_chunk<Tag>(f[n % P], qf[n], s);
          else if (n < 2 * NU)
            dp = mma_chunk<Tag>(f[n % P], gf[n - NU], dp);
          else
            acc[(n - 2 * NU) % DT] = mma_chunk<Tag>(f[n % P], w[(n - 2 * NU) / DT], acc[(n - 2 * NU) % DT]);
          if (n + P < N) f[n % P] = read(n + P);
          if (n >= NU && n < 2 * NU) {
#pragma unroll
            for (int i = (n - NU) * 16 / NU; i < (n - NU + 1) * 16 / NU; ++i) s[i] = exp2_(s[i] * a.c);
          }
          pin_order();
        }
      } else {
        s = rows_product<Tag, DP>(smem, kt + rowlane, base, qf, s);
        dp = rows_product<Tag, DP>(smem, vt + rowlane, base, gf, dp);
        to_ds<Tag>(&s, dp, a.c, st, seen, h);
        cols_product<Tag, DP>(smem, kt + collane, base, to_weights<Tag>(s), acc);
      }
    }
  }
  __syncthreads();
  if constexpr (WK > 1) {
    float *xo = (float *)smem;  // [wave][16 DT][64]
    constexpr int PER = 16 * DT * 64;
    static_assert((4 - F::WR) * PER * 4 <= F::LDS, "the waves' results fit the tiles' space");
    if (wk > 0) {
      float *o = xo + (wave - F::WR) * PER + lane;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[(d * 16 + i) * 64] = acc[d][i];
    }
    __syncthreads();
    for (int w = 1; w < (wk > 0 ? 0 : WK); ++w) {
      const float *o = xo + (wave + (w - 1) * F::WR) * PER + lane;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] += o[(d * 16 + i) * 64];
    }
    __syncthreads();
    if (wk > 0) return;
  }
  store_rows<Tag, DP, VEC>(smem + wave * 32 * T::PITCH, acc, a.scale * lower, a.D, lane,
                           [&](int n) { return group_row(a, a.dq, b, hk, rt * F::BM + wr * 32 + n); });
}

// dq, few rows: as attn_few_kernel.  A block's keys are written to this wave's
// piece of LDS from the fragments of the first product.
template <class Tag, int DP, bool VEC>
__device__ inline void take_few_dq(const AttnArgs &a, char *smem, int64_t id, int64_t units) {
  using T = Tile<Tag, DP>;
  using F = FewShape<Tag, DP>;
  constexpr int DT = T::DT;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5, l31 = lane & 31;
  const int tiles = (a.R + 31) / 32;
  int64_t unit = unit_of(id, units);
  const int rt = (int)(unit % tiles);
  unit /= tiles;
  const int split = (int)(unit % a.splits);
  const int64_t bh = unit / a.splits;
  const int64_t b = bh / a.Hk;
  const int hk = (int)(bh - b * a.Hk);
  const int len = length_of(a, b);
  const int all = (len + 31) / 32;
  const int t0 = (int)((int64_t)all * split / a.splits), t1 = (int)((int64_t)all * (split + 1) / a.splits);
  const int rows = a.R - rt * 32 < 32 ? a.R - rt * 32 : 32;

  u32x4 qf[T::NU], gf[T::NU], kf[T::NU], vf[T::NU];
  const char *kb = a.k.p + b * a.k.b + hk * a.k.h, *vb = a.v.p + b * a.v.b + hk * a.v.h;
  const uint8_t *mask = a.mask ? a.mask + b * a.mask_b : nullptr;
  load_rows<Tag, DP, VEC>(a, a.q, b, hk, rt * 32 + l31, lane, qf);
  load_rows<Tag, DP, VEC>(a, a.dout, b, hk, rt * 32 + l31, lane, gf);
  float2 st = load_stat<Tag>(a, bh, rt * 32 + l31);
  const int kt = wave * F::TILE;
  uint32_t sight = 1;
  const int rowlane = T::rowlane(lane), collane = T::collane(lane);
  f32x16 acc[DT] = {};
  int t = t0 + wave;
  if (t < t1) {
    load_states<Tag, DP, VEC>(kb, a.k.s, t * 32, len, a.D, lane, kf);
    load_states<Tag, DP, VEC>(vb, a.v.s, t * 32, len, a.D, lane, vf);
    sight = load_sight(mask, a.mask_s, t * 32, 32, len, lane);
  }
  const float lower = raise_row<Tag>(a, bh, rt * 32 + l31, len, lane, &st);
  for (; t < t1; t += 4) {
    uint32_t see = 0xffffffffu;
    if (mask || (t + 1) * 32 > len) see = (uint32_t)sight_bits(sight, t * 32, 32, len, lane);
    if (mask && !((see >> l31) & 1)) {
#pragma unroll
      for (int u = 0; u < T::NU; ++u) kf[u] = (u32x4){0, 0, 0, 0};
    }
    f32x16 s = splat(kStart<Tag> ? st.x : 0.f), dp = splat(kStart<Tag> ? st.y : 0.f);
#pragma unroll
    for (int u = 0; u < T::NU; ++u) {
      s = mma_chunk<Tag>(kf[u], qf[u], s);
      *(u32x4 *)(smem + ((kt + rowlane) ^ (u << 5))) = kf[u];
    }
#pragma unroll
    for (int u = 0; u < T::NU; ++u) dp = mma_chunk<Tag>(vf[u], gf[u], dp);
    if (t + 4 < t1) {
      load_states<Tag, DP, VEC>(kb, a.k.s, (t + 4) * 32, len, a.D, lane, kf);
      load_states<Tag, DP, VEC>(vb, a.v.s, (t + 4) * 32, len, a.D, lane, vf);
      sight = load_sight(mask, a.mask_s, (t + 4) * 32, 32, len, lane);
    }
    // (what a hidden state's values make of dp is replaced by zero)
    to_ds<Tag>(&s, dp, a.c, st, see, h);
    wave_lds_fence();
    const Weights<Tag> w = to_weights<Tag>(s);
    cols_product<Tag, DP>(smem, kt + collane, 0, w, acc);
    wave_lds_fence();
  }
  if constexpr (kPower<Tag>) {
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] *= lower;
  }
  float *xo = (float *)smem;
  __syncthreads();
  if (l31 < rows) {
    float *o = xo + (wave * rows + l31) * F::OP;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *(f32x4 *)(o + 32 * d + 8 * (i / 4) + 4 * h) = (f32x4){acc[d][i], acc[d][i + 1], acc[d][i + 2], acc[d][i + 3]};
  }
  __syncthreads();
  for (int e = tid; e < rows * DP; e += 256) {
    const int n = e / DP, d = e % DP;
    if (d >= a.D) continue;
    float o = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) o += xo[(w * rows + n) * F::OP + d];
    o *= a.scale;
    const int r = rt * 32 + n;
    if (a.splits > 1)
      a.part_o[((split * a.B * a.Hk + bh) * a.R + r) * a.D + d] = o;
    else
      store1<Tag>(group_row(a, a.dq, b, hk, r), d, o);
  }
}

// dk, dv: a workgroup takes 128 states, 32 a wave, and runs over the rows of
// the key head (or its part of them) in tiles of 32.  Scores are taken as
// S = Q K^T here, so a lane holds weights of one state and they are the second
// operand of dv^T = do^T p and dk^T = q^T ds as they are.  Measured as dq: 458 us
// for four products, 0.92 PFLOP/s; two accumulators of 32 x 128 a wave fill the
// registers of two waves a SIMD, and its fragment reads (40 KB a wave and tile)
// keep LDS busy a third of the time.
template <class Tag, int DP>
struct DkvShape {
  static constexpr int BR = 32;
  static constexpr int TILE = BR * Tile<Tag, DP>::PITCH;
  // 16-bit heads of more than 64 components: the values' fragments are read
  // from LDS each time, so that two waves fit a SIMD.
  static constexpr bool VLDS = Tag::W16 && DP > 64;
  static constexpr int VAL = 4 * TILE;
  static constexpr int STAT = VAL + (VLDS ? 128 * Tile<Tag, DP>::PITCH : 0);  // two tiles of row statistics
  static constexpr int OUT = 32 * Tile<TagF32, DP>::PITCH;                    // a wave's results, float32
  static constexpr int LDS = STAT + 2 * 2 * BR * 4 > 4 * OUT ? STAT + 2 * 2 * BR * 4 : 4 * OUT;
};

// Tiles of ROWS rows of a group, one after the other.  The query and head of a
// thread's rows are carried along, so that only the first tile divides.  Rows
// from R on repeat the last one, with weights of zero.  Their upstream gradients
// have to be zero too, since the last row's may be infinite: element by element
// they are loaded as zero; whole pieces are zeroed on their way to LDS (cut_rows)
// or when they have arrived there (DirectTile::hide).
template <class Tag, int DP, bool VEC, int ROWS>
struct RowWalk {
  using M = Mover<Tag, DP, ROWS, 256>;
  int s[M::NP], g[M::NP], step_s, step_g;
  __device__ void start(const AttnArgs &a, int first, int tid) {
    step_s = ROWS / a.G;
    step_g = ROWS - step_s * a.G;
#pragma unroll
    for (int p = 0; p < M::NP; ++p) {
      const int r = first + M::row(tid, p);
      s[p] = r / a.G;
      g[p] = r - s[p] * a.G;
    }
  }
  // To registers, or (DIRECT) to the tiles of LDS at `lds`.
  template <bool DIRECT, bool PLAIN>
  __device__ void load(const AttnArgs &a, const char *qb, const char *gb, int tid, M *mq, M *mg, uint32_t lds, int wave) {
    const int d0 = M::chunk(tid) * M::T::CE, dc = VEC ? (d0 < a.D ? d0 : 0) * Tag::ES : 0;
#pragma unroll
    for (int p = 0; p < M::NP; ++p) {
      const bool in = s[p] < a.Sq;
      const int sp = in ? s[p] : a.Sq - 1, gp = in ? g[p] : a.G - 1;
      const char *q = qb + sp * a.q.s + gp * a.q.h, *o = gb + sp * a.dout.s + gp * a.dout.h;
      if constexpr (!DIRECT) q += dc, o += dc;
      if constexpr (DIRECT) {
        const int c = M::T::chunk_at(M::chunk(tid), M::row(tid, p)) << 4;
        const uint32_t to = lds + p * 4096 + wave * 1024;
        if ((ROWS % M::RPP == 0 || wave * (M::RPP / 4) < ROWS) && DirectTile<Tag, DP, ROWS, PLAIN>::has(tid, p, a.D)) {
          lds_load16(to, q + c);
          lds_load16(to + ROWS * M::T::PITCH, o + c);
        }
      } else if constexpr (VEC) {
        mq->r[p] = *(const u32x4 *)q;
        mg->r[p] = *(const u32x4 *)o;
      } else {
        mq->r[p] = load_chunk<Tag, VEC>(q, d0, a.D);
        mg->r[p] = load_chunk<Tag, VEC>(o, d0, in ? a.D : 0);
      }
      s[p] += step_s;
      g[p] += step_g;
      if (g[p] >= a.G) {
        g[p] -= a.G;
        ++s[p];
      }
    }
  }
};

template <class Tag, int DP, bool VEC, bool PLAIN>
__device__ inline void take_dkv(const AttnArgs &a, char *smem, int64_t id, int64_t units) {
  using T = Tile<Tag, DP>;
  using F = DkvShape<Tag, DP>;
  constexpr int DT = T::DT;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5, l31 = lane & 31;
  const int tiles = (a.Sk + 127) / 128;
  int64_t unit = unit_of(id, units);
  const int kt0 = (int)(unit % tiles);
  unit /= tiles;
  const int part = (int)(unit % a.row_parts);
  const int64_t bh = unit / a.row_parts, b = bh / a.Hk;
  const int hk = (int)(bh - b * a.Hk);
  const int len = length_of(a, b);
  const int j0 = kt0 * 128 + wave * 32, j = j0 + l31;
  const int all = (a.R + F::BR - 1) / F::BR;
  const int t0 = (int)((int64_t)all * part / a.row_parts);
  int t1 = (int)((int64_t)all * (part + 1) / a.row_parts);
  if (kt0 * 128 >= len) t1 = t0;  // no state of the tile is visible

  const bool see = j < len && (PLAIN || !a.mask || a.mask[b * a.mask_b + j * a.mask_s]);
  u32x4 kf[T::NU], vf[T::NU];
  const int rowlane = T::rowlane(lane), collane = T::collane(lane);
  const int val = F::VAL + wave * 32 * T::PITCH + rowlane;  // this wave's values
  // (a hidden state's column of results is its own, and is replaced by zeros)
  load_states<Tag, DP, VEC>(a.k.p + b * a.k.b + hk * a.k.h, a.k.s, j0, a.Sk, a.D, lane, kf);
  load_states<Tag, DP, VEC>(a.v.p + b * a.v.b + hk * a.v.h, a.v.s, j0, a.Sk, a.D, lane, vf);
  if constexpr (F::VLDS) {
#pragma unroll
    for (int u = 0; u < T::NU; ++u) *(u32x4 *)(smem + (val ^ (u << 5))) = vf[u];
  }
  Mover<Tag, DP, F::BR, 256> mq, mg;
  RowWalk<Tag, DP, VEC, F::BR> walk;
  const char *qb = a.q.p + b * a.q.b + (int64_t)hk * a.G * a.q.h, *gb = a.dout.p + b * a.dout.b + (int64_t)hk * a.G * a.dout.h;
  walk.start(a, t0 * F::BR, tid);
  float2 st;
  auto load = [&](int t) {
    walk.template load<VEC, PLAIN>(a, qb, gb, tid, &mq, &mg, lds_offset(smem) + (t & 1) * 2 * F::TILE, wave);
    if (tid < F::BR) st = load_stat<Tag>(a, bh, t * F::BR + tid);
  };
  f32x16 dk[DT] = {}, dv[DT] = {};
  if constexpr (VEC) DirectTile<Tag, DP, F::BR, PLAIN>::clear(smem, 4, a.D, tid);
  if (t0 < t1) load(t0);
  // the power of two of ds, beside that of the weights, and what takes both off
  float up = 1.f, lower = 1.f;
  if constexpr (kPower<Tag>) {
    const int last = t1 * F::BR < a.R ? t1 * F::BR : a.R;
    const float sums = wave_top(a.sum_do + bh * a.R, t0 * F::BR, last, lane);
    const int e = power_for(0.5f * sums * head_top_v(a, bh, len, lane));
    up = exponent(e - kRaiseBack<Tag>);
    lower = exponent(-e);
  }
  arrived(kf);
  if constexpr (!F::VLDS) arrived(vf);
  for (int t = t0; t < t1; ++t) {
    const int qt = (t & 1) * 2 * F::TILE, gt = qt + F::TILE;
    float *stat = (float *)(smem + F::STAT) + (t & 1) * 2 * F::BR;
    if constexpr (VEC) {
      lds_loads_done();
      if ((t + 1) * F::BR > a.R)
        DirectTile<Tag, DP, F::BR, PLAIN>::hide(smem + gt, ((uint64_t)1 << (a.R - t * F::BR)) - 1, tid);
    } else {
      mq.cut(a.D, tid);
      mg.cut(a.D, tid);
      mq.store(smem + qt, tid);
      mg.store(smem + gt, tid);
    }
    if (tid < F::BR) {
      stat[tid] = st.x;
      stat[F::BR + tid] = st.y;
    }
    __syncthreads();
    if (t + 1 < t1) load(t + 1);
    f32x16 s = {}, dp = {};
    if constexpr (kStart<Tag>) {
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const f32x4 x = *(const f32x4 *)(stat + 2 * i + 4 * h), y = *(const f32x4 *)(stat + F::BR + 2 * i + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i + e] = x[e], dp[i + e] = y[e];
      }
    }
    if constexpr (VEC && F::VLDS) {
      // One stream of fragment reads, some products ahead of their use: queries
      // for the scores, do and the values for dp, while which the weights are
      // formed, then the columns of do and of the queries.
      constexpr int NU = T::NU, N = 2 * NU + 4 * DT, P = 4, PV = 2;
      u32x4 f[P], v[PV], w[2];
      auto read = [&](int n) {
        if (n < 2 * NU) return *(const u32x4 *)(smem + (((n < NU ? qt : gt) + rowlane) ^ (n % NU << 5)));
        const int m = n - 2 * NU;
        return col_read<Tag, DP>(smem, (m < 2 * DT ? gt : qt) + collane, m / DT % 2 * 16, m % DT);
      };
      // p and ds are rounded to the inputs' type for their products
      auto pack8 = [&](const f32x16 &x, int t, u32x4 *to) {
#pragma unroll
        for (int j = 0; j < 4; ++j) (*to)[j] = pack2<Tag>(x[8 * t + 2 * j], x[8 * t + 2 * j + 1]);
      };
      auto to_ds8 = [&](int t) {
#pragma unroll
        for (int i = 8 * t; i < 8 * t + 8; ++i) {
          dp[i] *= s[i];
          if constexpr (kPower<Tag>) dp[i] *= up;
        }
      };
#pragma unroll
      for (int n = 0; n < P; ++n) f[n] = read(n);
      pin_order();
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const int m = n - 2 * NU;
        if (m == 0) pack8(s, 0, &w[0]);
        if (m == DT) pack8(s, 1, &w[1]), to_ds8(0);
        if (m == 2 * DT) pack8(dp, 0, &w[0]), to_ds8(1);
        if (m == 3 * DT) pack8(dp, 1, &w[1]);
        if (n < NU)
          s = mma_chunk<Tag>(f[n % P], kf[n], s);
        else if (n < 2 * NU)
          dp = mma_chunk<Tag>(f[n % P], v[n % PV], dp);
        else if (m < 2 * DT)
          dv[m % DT] = mma_chunk<Tag>(f[n % P], w[m / DT], dv[m % DT]);
        else
          dk[m % DT] = mma_chunk<Tag>(f[n % P], w[m / DT - 2], dk[m % DT]);
        if (n + P < N) f[n % P] = read(n + P);
        if (n + PV >= NU && n + PV < 2 * NU) v[n % PV] = *(const u32x4 *)(smem + (val ^ ((n + PV) % NU << 5)));
        if (n >= NU && n < 2 * NU) {
#pragma unroll
          for (int i = (n - NU) * 16 / NU; i < (n - NU + 1) * 16 / NU; ++i) s[i] = exp2_(s[i] * a.c);
        }
        pin_order();
      }
    } else {
      s = rows_product<Tag, DP>(smem, qt + rowlane, 0, kf, s);
      dp = rows_product<Tag, DP>(smem, gt + rowlane, 0, vf, dp);
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        f32x4 x = {}, y = {};
        if constexpr (!kStart<Tag>) {
          x = *(const f32x4 *)(stat + 2 * i + 4 * h);
          y = *(const f32x4 *)(stat + F::BR + 2 * i + 4 * h);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[i + e] = weight<Tag>(s[i + e], a.c, x[e]);
          dp[i + e] = ds_of<Tag>(s[i + e], dp[i + e], y[e]);
          if constexpr (kPower<Tag>) dp[i + e] *= up;
        }
      }
      cols_product<Tag, DP>(smem, gt + collane, 0, to_weights<Tag>(s), dv);
      cols_product<Tag, DP>(smem, qt + collane, 0, to_weights<Tag>(dp), dk);
    }
  }
  if (!see) {
    // a state that is not visible has its column of results to itself
#pragma unroll
    for (int d = 0; d < DT; ++d) dk[d] = dv[d] = (f32x16){};
  }
  __syncthreads();
  const float fk = a.scale * lower, fv = exponent(-kRaiseBack<Tag>);
  if (a.row_parts > 1) {
    float *pk = a.part_dk + (part * a.B * a.Hk + bh) * a.Sk * a.D, *pv = a.part_dv + (pk - a.part_dk);
    auto row = [&](float *p, int n) { return j0 + n < a.Sk ? (char *)(p + (int64_t)(j0 + n) * a.D) : nullptr; };
    store_rows<TagF32, DP, VEC>(smem + wave * F::OUT, dk, fk, a.D, lane, [&](int n) { return row(pk, n); });
    store_rows<TagF32, DP, VEC>(smem + wave * F::OUT, dv, fv, a.D, lane, [&](int n) { return row(pv, n); });
    return;
  }
  auto row = [&](const Tokens &t, int n) {
    return j0 + n < a.Sk ? t.p + b * t.b + (j0 + n) * t.s + hk * t.h : nullptr;
  };
  store_rows<Tag, DP, VEC>(smem + wave * F::OUT, dk, fk, a.D, lane, [&](int n) { return row(a.dk, n); });
  store_rows<Tag, DP, VEC>(smem + wave * F::OUT, dv, fv, a.D, lane, [&](int n) { return row(a.dv, n); });
}

// dq and dk, dv in one launch: the owners of states take the first `n_dkv`
// workgroups or (dq_first) the last, the longer ones ahead, so that the chip is
// filled by the one kind where the other leaves off.  WK: waves that share the
// rows of dq, 0 for few rows.  PLAIN: whole rows without a mask, which needs
// fewer registers.  As many waves a SIMD as the owners of states can have on
// their own.  Measured against kernels one after the other (the first taking
// the rows' statistics on its way), bfloat16: 2 x 8 heads of 200 queries over
// 1001 states of 64 components 24 -> 19 us; float16, 12 x 6 heads of 333 over
// 1001 masked states of 72 components 79 -> 56 (60 with its powers of two); 8 x
// 32 heads of 2048 over 6272 of 128 components 2685 -> 2652.
template <class Tag, int DP, int WK, bool VEC, bool PLAIN>
__global__ __launch_bounds__(256, Tag::W16 ? (DP <= 32 ? 4 : DP <= 64 ? 3 : 2) : DP <= 64 ? 2 : 1) void attn_grads_kernel(AttnArgs a, int n_dq, int n_dkv,
                                                                                      int dq_first) {
  extern __shared__ __align__(512) char attn_smem[];
  const int id = blockIdx.x, at = dq_first ? id - n_dq : id;
  if (at >= 0 && at < n_dkv) {
    take_dkv<Tag, DP, VEC, PLAIN>(a, attn_smem, at, n_dkv);
  } else {
    const int dq = dq_first ? id : id - n_dkv;
    if constexpr (WK == 0)
      take_few_dq<Tag, DP, VEC>(a, attn_smem, dq, n_dq);
    else
      take_dq<Tag, DP, WK, VEC, PLAIN>(a, attn_smem, dq, n_dq);
  }
}

// All gradients of a handful of rows in one pass over the states (16-bit, at
// most one_pass_rows a key head: learned queries that read a map): the states,
// read and written once, bound it.  A workgroup keeps a key head's
// rows in LDS and takes a part of its states; each wave runs over every fourth
// block of 32, on its own.  The scores are taken as for dk and dv; for dq the
// block's ds goes through LDS to turn a lane's rows into its column.  dq is
// summed over the waves at the end, over the parts by attn_sum_kernel.
// Measured, bfloat16, 1024 heads of 64 queries over 784 states of 64 components:
// 96 us, 4.5 TB/s (dq, then dk and dv, in kernels of their own: 155 us).
template <class Tag, int DP, int NRB_>
struct RowsShape {
  static constexpr int PITCH = Tile<Tag, DP>::PITCH;
  static constexpr int NRB = NRB_, ROWS = 32 * NRB;
  static constexpr int Q = 0, G = ROWS * PITCH, STAT = 2 * ROWS * PITCH;
  static constexpr int DS = 32 * Tile<Tag, 32>::PITCH;  // a wave's ds: 32 states of 32 rows
  static constexpr int WAVE = 2 * 32 * PITCH + DS;      // a wave's keys, values and ds
  static constexpr int NORM = STAT + 2 * ROWS * 4;      // float16: the waves' largest sums of |do| and |delta|
  static constexpr int W0 = NORM + (kPower<Tag> ? 256 : 0);
  static constexpr int JOIN = 3 * NRB * 16 * (DP / 32) * 64 * 4;
  static constexpr int LDS = W0 + 4 * WAVE > JOIN ? W0 + 4 * WAVE : JOIN;
};

template <class Tag, int DP, int NRB, bool VEC>
__global__ __launch_bounds__(256, DP <= 64 ? 2 : 1) void attn_rows_bwd_kernel(AttnArgs a) {
  using T = Tile<Tag, DP>;
  using T32 = Tile<Tag, 32>;
  using F = RowsShape<Tag, DP, NRB>;
  constexpr int DT = T::DT, NU = T::NU;
  extern __shared__ __align__(512) char attn_smem[];
  char *const smem = attn_smem;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5, l31 = lane & 31;
  const int64_t unit = unit_of(blockIdx.x, gridDim.x), bh = unit / a.splits, b = bh / a.Hk;
  const int split = (int)(unit - bh * a.splits), hk = (int)(bh - b * a.Hk);
  const int len = length_of(a, b);
  const int all = (a.Sk + 31) / 32;
  const int t0 = (int)((int64_t)all * split / a.splits), t1 = (int)((int64_t)all * (split + 1) / a.splits);
  const int nrb = (a.R + 31) / 32;
  const char *kb = a.k.p + b * a.k.b + hk * a.k.h, *vb = a.v.p + b * a.v.b + hk * a.v.h;
  const uint8_t *mask = a.mask ? a.mask + b * a.mask_b : nullptr;
  const int rowlane = T::rowlane(lane), collane = T::collane(lane), col32 = T32::collane(lane);
  const int kt = F::W0 + wave * F::WAVE, vt = kt + 32 * F::PITCH, dst = vt + 32 * F::PITCH;

  StateMover<Tag, DP, VEC, 32, 64> mk, mv;
  uint32_t sight = 1;
  auto load = [&](int t) {
    if (t * 32 >= len) return;
    mk.load(kb, a.k.s, t * 32, len, a.D, lane);
    mv.load(vb, a.v.s, t * 32, len, a.D, lane);
    sight = load_sight(mask, a.mask_s, t * 32, 32, len, lane);
  };
  int t = t0 + wave;
  if (t < t1) load(t);
  {
    Mover<Tag, DP, F::ROWS, 256> mq, mg;
    RowWalk<Tag, DP, VEC, F::ROWS> walk;
    walk.start(a, 0, tid);
    walk.template load<false, false>(a, a.q.p + b * a.q.b + (int64_t)hk * a.G * a.q.h,
                              a.dout.p + b * a.dout.b + (int64_t)hk * a.G * a.dout.h, tid, &mq, &mg, 0, 0);
    mq.cut(a.D, tid);
    mg.cut(a.D, tid);
    if constexpr (VEC) mg.cut_rows(a.R, tid);
    mq.store(smem + F::Q, tid);
    mg.store(smem + F::G, tid);
    if (wave < F::NRB) {  // (at most four)
      u32x4 gf[NU];
      const int r = wave * 32 + l31;
      load_rows<Tag, DP, VEC>(a, a.dout, b, hk, r, lane, gf);
      u32x4 of[NU];
      load_rows<Tag, DP, VEC>(a, a.o, b, hk, r, lane, of);
      float d = 0.f;
#pragma unroll
      for (int u = 0; u < NU; ++u) d += chunk_dot<Tag>(of[u], gf[u]);
      d = other_half_sum(d);
      if constexpr (kPower<Tag>) {
        float n = 0.f;
#pragma unroll
        for (int u = 0; u < NU; ++u) n += chunk_sum<Tag>(gf[u]);
        n = other_half_sum(n);
        // (a row that is not finite makes its own gradients what they are)
        const float x = __builtin_fabsf(d);
        const uint32_t sums = wave_max(n < INFINITY ? __float_as_uint(n) : 0);
        const uint32_t deltas = wave_max(n < INFINITY && x < INFINITY ? __float_as_uint(x) : 0);
        if (lane == 0) {
          ((uint32_t *)(smem + F::NORM))[wave] = sums;
          ((uint32_t *)(smem + F::NORM))[4 + wave] = deltas;
        }
      }
      const float2 st = r < a.R ? stat_of<Tag>(a, b, hk, r, d) : blind_stat<Tag>();
      if (h == 0) {
        ((float *)(smem + F::STAT))[r] = st.x;
        ((float *)(smem + F::STAT))[F::ROWS + r] = st.y;
      }
    }
  }
  __syncthreads();

  f32x16 dq[F::NRB][DT] = {};
  // float16's power of two: of all rows together, since the same ds serves dk
  // and dq, from |ds| <= |dp| + |delta|; lowered where a block of states has
  // larger values than those before
  float sum_do = 0.f, delta = 0.f;
  int power = 100;
  if constexpr (kPower<Tag>) {
#pragma unroll
    for (int n = 0; n < F::NRB; ++n) {
      sum_do = fmaxf(sum_do, ((const float *)(smem + F::NORM))[n]);
      delta = fmaxf(delta, ((const float *)(smem + F::NORM))[4 + n]);
    }
  }
  for (; t < t1; t += 4) {
    const int j0 = t * 32;
    f32x16 dk[DT] = {}, dv[DT] = {};
    // A hidden state's column is its own, whatever the rows hold: zeroed in the
    // registers, or (128 components, where the branch around them made the
    // compiler move them out and back) on the way out.  Masked, 512 heads of 784
    // states: 64 components 47.0 us, 50.3 on the way out; 128 components 199 us,
    // 108 on the way out.
    uint32_t keep = 0xffffffffu;
    if (j0 < len) {
      uint32_t see = 0xffffffffu;
      if (mask || j0 + 32 > len) see = (uint32_t)sight_bits(sight, j0, 32, len, lane);
      const bool hide = see != 0xffffffffu;
      mk.hide(hide, see, a.D, lane);
      mv.hide(hide, see, a.D, lane);
      mk.store(smem + kt, lane);
      mv.store(smem + vt, lane);
      if (t + 4 < t1) load(t + 4);
      wave_lds_fence();
      if constexpr (kPower<Tag>) {
        // (read back from LDS: from the registers it made others spill)
        u16x2 top = {0, 0};
#pragma unroll
        for (int p = 0; p < StateMover<Tag, DP, VEC, 32, 64>::NP; ++p)
          top = chunk_top(*(const u32x4 *)(smem + vt + p * 1024 + lane * 16), top);
        const float bound = to_f32<Tag>((u16)wave_max(top_of(top))) * sum_do;
        const int e = __builtin_amdgcn_readfirstlane(power_for(bound + delta));
        const int low = e < power ? e : power;
        const float fix = power - low < 126 ? exponent(low - power) : 0.f;
        power = low;
#pragma unroll
        for (int n = 0; n < F::NRB; ++n)
#pragma unroll
          for (int d = 0; d < DT; ++d) dq[n][d] *= fix;
      }
#pragma unroll
      for (int rb = 0; rb < F::NRB; ++rb) {
        if (rb >= nrb) continue;
        const float *stat = (const float *)(smem + F::STAT) + rb * 32;
        f32x16 s, dp;
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const f32x4 x = *(const f32x4 *)(stat + 2 * i + 4 * h), y = *(const f32x4 *)(stat + F::ROWS + 2 * i + 4 * h);
#pragma unroll
          for (int e = 0; e < 4; ++e) s[i + e] = x[e], dp[i + e] = y[e];
        }
#pragma unroll
        for (int u = 0; u < NU; ++u) {
          const int x = u << 5;
          s = mma_chunk<Tag>(*(const u32x4 *)(smem + ((F::Q + rowlane) ^ x) + rb * 32 * F::PITCH),
                             *(const u32x4 *)(smem + ((kt + rowlane) ^ x)), s);
          dp = mma_chunk<Tag>(*(const u32x4 *)(smem + ((F::G + rowlane) ^ x) + rb * 32 * F::PITCH),
                              *(const u32x4 *)(smem + ((vt + rowlane) ^ x)), dp);
        }
        if (hide && !((see >> l31) & 1)) s = splat(-INFINITY), dp = splat(0.f);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[i] = exp2_(s[i] * a.c);
          dp[i] *= s[i];
          if constexpr (kPower<Tag>) dp[i] *= exponent(power - kRaiseBack<Tag>);
        }
        // p and ds are rounded to the inputs' type for their products
        const Weights<Tag> wd = to_weights<Tag>(dp);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *(u32x2 *)(smem + dst + l31 * T32::PITCH + ((i ^ T32::swz(l31)) << 4) + 8 * h) =
              (u32x2){wd.w[i / 2][i % 2 * 2], wd.w[i / 2][i % 2 * 2 + 1]};
        cols_product<Tag, DP>(smem, F::G + collane, rb * 32, to_weights<Tag>(s), dv);
        cols_product<Tag, DP>(smem, F::Q + collane, rb * 32, wd, dk);
        wave_lds_fence();
        Weights<Tag> wq;
#pragma unroll
        for (int i = 0; i < 2; ++i) wq.w[i] = col_read<Tag, 32>(smem, dst + col32, 16 * i, 0);
        cols_product<Tag, DP>(smem, kt + collane, 0, wq, dq[rb]);
        wave_lds_fence();
      }
      if constexpr (DP > 96) {
        keep = see;
      } else if (hide && !((see >> l31) & 1)) {
#pragma unroll
        for (int d = 0; d < DT; ++d) dk[d] = dv[d] = (f32x16){};
      }
    }
    auto row = [&](const Tokens &o, int n) {
      return j0 + n < a.Sk ? o.p + b * o.b + (j0 + n) * o.s + hk * o.h : nullptr;
    };
    const float fk = kPower<Tag> ? a.scale * exponent(-power) : a.scale;
    store_rows<Tag, DP, VEC>(smem + vt, dv, exponent(-kRaiseBack<Tag>), a.D, lane, [&](int n) { return row(a.dv, n); }, keep);
    store_rows<Tag, DP, VEC>(smem + kt, dk, fk, a.D, lane, [&](int n) { return row(a.dk, n); }, keep);
  }

  // the waves' parts of dq, without their powers of two
  __syncthreads();
  float *xo = (float *)smem;  // [wave - 1][16 NRB DT][64]
  constexpr int PER = 16 * F::NRB * DT * 64;
  const float lower = exponent(kPower<Tag> ? -power : 0);
  if (wave > 0) {
    float *o = xo + (wave - 1) * PER + lane;
#pragma unroll
    for (int rb = 0; rb < F::NRB; ++rb)
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[((rb * DT + d) * 16 + i) * 64] = dq[rb][d][i] * lower;
  }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int rb = 0; rb < F::NRB; ++rb)
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float x = dq[rb][d][i] * lower;
#pragma unroll
        for (int w = 0; w < 3; ++w) x += xo[w * PER + ((rb * DT + d) * 16 + i) * 64 + lane];
        dq[rb][d][i] = x;
      }
#pragma unroll
  for (int rb = 0; rb < F::NRB; ++rb) {
    if (rb >= nrb) continue;
    if (a.splits > 1) {
      float *p = a.part_o + (split * a.B * a.Hk + bh) * a.R * a.D;
      store_rows<TagF32, DP, VEC>(smem, dq[rb], a.scale, a.D, lane, [&](int n) {
        const int r = rb * 32 + n;
        return r < a.R ? (char *)(p + (int64_t)r * a.D) : nullptr;
      });
    } else {
      store_rows<Tag, DP, VEC>(smem, dq[rb], a.scale, a.D, lane,
                               [&](int n) { return group_row(a, a.dq, b, hk, rb * 32 + n); });
    }
  }
}

// Sums of partial gradients, in the order of the parts: rows [B Hk, N] of D
// components, row n of key head hk being token n / G of head hk G + n % G.
// Blocks of y = 1 take the second tensor.
struct SumArgs {
  const float *part[2];
  Tokens out[2];
  int64_t rows;  // B Hk N
  int parts, N, G, Hk, D;
};

template <class Tag, bool VEC>
__global__ __launch_bounds__(256) void attn_sum_kernel(SumArgs a) {
  constexpr int V = kJoin<VEC>;
  const uint32_t e = blockIdx.x * 256 + threadIdx.x, per = (uint32_t)a.D / V, row = e / per;  // (rows D is at most 2^31)
  if (row >= (uint32_t)a.rows) return;
  const int d = (int)(e - row * per) * V;
  const float *part = a.part[blockIdx.y] + (int64_t)row * a.D + d;
  const Tokens &t = a.out[blockIdx.y];
  const int64_t step = a.rows * a.D;
  float sum[V] = {};
  for (int p0 = 0; p0 < a.parts; p0 += 8) {
    float v[8][V] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (p0 + i < a.parts) load_part<VEC>(part + (p0 + i) * step, v[i]);
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int k = 0; k < V; ++k) sum[k] += v[i][k];
  }
  const uint32_t bh = row / (uint32_t)a.N, b = bh / (uint32_t)a.Hk;
  const int r = (int)(row - bh * a.N), hk = (int)(bh - b * a.Hk), s = r / a.G, g = r - s * a.G;
  store_part<Tag, VEC>(t.p + (int64_t)b * t.b + s * t.s + (int64_t)(hk * a.G + g) * t.h, d, sum);
}

// Workgroups that join rows of D components.
template <bool VEC> int64_t joiners(int64_t rows, int D) { return (rows * (D / kJoin<VEC>) + 255) / 256; }

// ---------------------------------------------------------------- launchers

// (the front end has checked the grids, attn_grids_fit)
#define WBMM_ATTN_LAUNCH(kernel, n, lds, args)                               \
  do {                                                                       \
    kernel<<<dim3((unsigned)(n)), dim3(256), (lds), stream>>>(args);         \
    const hipError_t e_ = hipGetLastError();                                 \
    if (e_ != hipSuccess) return e_;                                         \
  } while (0)

template <class Tag, int DP, bool VEC>
hipError_t launch_fwd(const AttnArgs &a, hipStream_t stream) {
  const int64_t bh = a.B * a.Hk;
  if (a.tile_rows == 32) {
    WBMM_ATTN_LAUNCH((attn_few_kernel<Tag, DP, VEC>), bh * ((a.R + 31) / 32) * a.splits, (FewShape<Tag, DP>::lds(a.R)), a);
    if (a.splits > 1) WBMM_ATTN_LAUNCH((attn_join_kernel<Tag, VEC>), joiners<VEC>(bh * a.R, a.D), 0, a);
  } else if (a.tile_rows == 64) {
    WBMM_ATTN_LAUNCH((attn_fwd_kernel<Tag, DP, 2, VEC, false>), bh * ((a.R + 63) / 64), (FwdShape<Tag, DP, 2>::LDS), a);
  } else if (VEC && a.D == DP && !a.mask) {
    WBMM_ATTN_LAUNCH((attn_fwd_kernel<Tag, DP, 1, VEC, VEC>), bh * ((a.R + 127) / 128), (FwdShape<Tag, DP, 1>::LDS), a);
  } else {
    WBMM_ATTN_LAUNCH((attn_fwd_kernel<Tag, DP, 1, VEC, false>), bh * ((a.R + 127) / 128), (FwdShape<Tag, DP, 1>::LDS), a);
  }
  return hipSuccess;
}

template <class Tag, int DP, int WK, bool VEC, bool PLAIN>
void launch_grads(const AttnArgs &a, int dq_lds, hipStream_t stream) {
  const int64_t bh = a.B * a.Hk, tile = a.tile_rows;
  const int n_dq = (int)(bh * ((a.R + tile - 1) / tile) * a.splits);
  const int n_dkv = (int)(bh * ((a.Sk + 127) / 128) * a.row_parts), dkv_lds = DkvShape<Tag, DP>::LDS;
  // (three products of a tile with all states, four with all rows)
  const bool dq_first = 3 * tile * (a.Sk / a.splits) > 4 * 128 * (int64_t)(a.R / a.row_parts);
  attn_grads_kernel<Tag, DP, WK, VEC, PLAIN>
      <<<dim3((unsigned)(n_dq + n_dkv)), dim3(256), dq_lds > dkv_lds ? dq_lds : dkv_lds, stream>>>(a, n_dq, n_dkv, dq_first);
}

template <class Tag, int DP, bool VEC>
hipError_t launch_bwd(const AttnArgs &a, hipStream_t stream) {
  const int64_t bh = a.B * a.Hk;
  if constexpr (Tag::W16) {
    if (a.one_pass) {
      // (blocks of 32 rows: as the registers allow, one_pass_rows)
      constexpr int NRB = one_pass_rows(DP) / 32;
      bool half = false;
      if constexpr (NRB == 4) {
        half = a.R <= 64;
        if (half) WBMM_ATTN_LAUNCH((attn_rows_bwd_kernel<Tag, DP, 2, VEC>), bh * a.splits, (RowsShape<Tag, DP, 2>::LDS), a);
      }
      if (!half) WBMM_ATTN_LAUNCH((attn_rows_bwd_kernel<Tag, DP, NRB, VEC>), bh * a.splits, (RowsShape<Tag, DP, NRB>::LDS), a);
      if (a.splits > 1) {
        const SumArgs s = {{a.part_o}, {a.dq}, bh * a.R, a.splits, a.R, a.G, a.Hk, a.D};
        WBMM_ATTN_LAUNCH((attn_sum_kernel<Tag, VEC>), joiners<VEC>(bh * a.R, a.D), 0, s);
      }
      return hipSuccess;
    }
  }
  const int64_t rows = bh * a.R;
  if (rows > 0) {
    const int64_t of_v = kPower<Tag> ? bh * ((a.Sk + 127) / 128) : 0;
    attn_stat_kernel<Tag, VEC><<<dim3((unsigned)(of_v + (rows + 15) / 16)), dim3(256), 0, stream>>>(a, (uint32_t)of_v);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.tile_rows == 32)
    launch_grads<Tag, DP, 0, VEC, false>(a, FewShape<Tag, DP>::lds(a.R), stream);
  else if (a.tile_rows == 64)
    launch_grads<Tag, DP, 2, VEC, false>(a, FwdShape<Tag, DP, 2>::LDS, stream);
  else if (VEC && a.D == DP && !a.mask)
    launch_grads<Tag, DP, 1, VEC, VEC>(a, FwdShape<Tag, DP, 1>::LDS, stream);
  else
    launch_grads<Tag, DP, 1, VEC, false>(a, FwdShape<Tag, DP, 1>::LDS, stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.splits > 1) {
    const SumArgs s = {{a.part_o}, {a.dq}, rows, a.splits, a.R, a.G, a.Hk, a.D};
    WBMM_ATTN_LAUNCH((attn_sum_kernel<Tag, VEC>), joiners<VEC>(rows, a.D), 0, s);
  }
  if (a.row_parts > 1 && a.Sk > 0) {
    const SumArgs s = {{a.part_dk, a.part_dv}, {a.dk, a.dv}, bh * a.Sk, a.row_parts, a.Sk, 1, a.Hk, a.D};
    attn_sum_kernel<Tag, VEC><<<dim3((unsigned)joiners<VEC>(bh * a.Sk, a.D), 2), dim3(256), 0, stream>>>(s);
    return hipGetLastError();
  }
  return hipSuccess;
}

#undef WBMM_ATTN_LAUNCH

}  // namespace

template <class Tag>
template <bool VEC>
hipError_t AttnEntry<Tag>::forward(const AttnArgs &a, hipStream_t stream) {
  if (a.D <= 32) return launch_fwd<Tag, 32, VEC>(a, stream);
  if (a.D <= 64) return launch_fwd<Tag, 64, VEC>(a, stream);
  if (a.D <= 96) return launch_fwd<Tag, 96, VEC>(a, stream);
  return launch_fwd<Tag, 128, VEC>(a, stream);
}

template <class Tag>
template <bool VEC>
hipError_t AttnEntry<Tag>::backward(const AttnArgs &a, hipStream_t stream) {
  if (a.D <= 32) return launch_bwd<Tag, 32, VEC>(a, stream);
  if (a.D <= 64) return launch_bwd<Tag, 64, VEC>(a, stream);
  if (a.D <= 96) return launch_bwd<Tag, 96, VEC>(a, stream);
  return launch_bwd<Tag, 128, VEC>(a, stream);
}

}  // namespace wbmm
