// Rotary positions with several axes.
//
// Pair i of a head belongs to one axis a(i); a token at positions
// pos[0..axes) turns it by the angle pos[a(i)] * freqs[i]:
//   lo' = lo cos - hi sin,  hi' = lo sin + hi cos
// and the gradient turns back.  The pairs are components (i, i + P), or
// neighbours (2i, 2i + 1); components from 2 P on are copied.
//
// The operator is a copy with a handful of products: it is bound by device
// memory, or by the launch for a few tokens.  A workgroup takes a run of
// tokens.  It computes each (token, pair)'s cosine and sine once, into LDS,
// for all heads; then its threads stream the heads' components in 16-byte
// pieces.  The angle is taken in 64 bits and reduced to a fraction of a turn
// there, since in 32 bits a position of 2^20 leaves no more than 2^-4 radians.
// Cosine and sine are taken in float32, of the fraction rounded to float32, and
// turned by what that left: float32 results are off by 0.69 x 2^-24 of themselves
// (root mean square), without it by 0.90, from cosines and sines of 64 bits that
// are rounded once by 0.71.
// Measured: 12544 x 40 x 128 bfloat16 40.7 us (6.3 TB/s); eight tokens 4 us.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "wbmm_attn_internal.h"
#include "wbmm_kernels.h"

namespace wbmm {

namespace {

constexpr int kRotThreads = 256;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <class Tag> __device__ inline void unpack(u32x4 v, float *f);
template <> __device__ inline void unpack<TagF32>(u32x4 v, float *f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
}
template <class Tag> __device__ inline void unpack16(u32x4 v, float *f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = to_f32<Tag>((u16)(v[i] & 0xffff));
    f[2 * i + 1] = to_f32<Tag>((u16)(v[i] >> 16));
  }
}
template <> __device__ inline void unpack<TagBF16>(u32x4 v, float *f) { unpack16<TagBF16>(v, f); }
template <> __device__ inline void unpack<TagF16>(u32x4 v, float *f) { unpack16<TagF16>(v, f); }

template <class Tag> __device__ inline u32x4 repack(const float *f) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (Tag::W16)
      v[i] = pack2<Tag>(f[2 * i], f[2 * i + 1]);
    else
      v[i] = __builtin_bit_cast(uint32_t, f[i]);
  }
  return v;
}

template <class Tag> __device__ inline void store1(char *p, float v) {
  if constexpr (Tag::W16)
    *(u16 *)p = (u16)pack2<Tag>(v, 0.f);
  else
    *(float *)p = v;
}

// Items of a token, per head: VEC: 16-byte pieces (paired ones carry two
// pieces in the half layout), then the pieces behind the pairs; else pairs,
// then single components.
struct RotPlan {
  int tok;        // tokens of a workgroup
  int heads;      // heads of a workgroup (grid dimension y counts the runs)
  int turn, per;  // turning items of a head, all items of a head
  int small;      // tokens are counted in 32 bits
  uint32_t magic, magic_tok;  // ceil(2^32 / per), ceil(2^32 / items of a token); 0 for 1
};

// e / d by d's rounded-up reciprocal in 2^-32 (exact while e d < 2^32).
__device__ inline int quotient(int e, uint32_t magic) { return magic ? (int)__umulhi((uint32_t)e, magic) : e; }
inline uint32_t reciprocal(int64_t d) { return d == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + d - 1) / d); }

// (Written out as fused products, so that every layout gives the same bits.)
__device__ inline void rotate(float *lo, float *hi, float2 r) {
  const float u = *lo, w = *hi;
  *lo = __builtin_fmaf(-w, r.y, u * r.x);
  *hi = __builtin_fmaf(u, r.y, w * r.x);
}

// Results are not read again here; kept out of the caches' way they leave
// faster: 12544 x 40 x 128 bfloat16 44.8 -> 40.0 us, 16000 x 24 x 128 float32
// 77 -> 60 us (6.6 TB/s).
__device__ inline void store16(char *p, u32x4 v) { __builtin_nontemporal_store(v, (u32x4 *)p); }

// Where an item's components lie in its row: up to two pieces of a head.
struct RotItem {
  int t, pos;        // token of the workgroup; first pair, or -1: copied
  int64_t x, y;      // bytes from the token's first component
  int64_t next;      // the second piece of a pair, behind the first (half layout)
};

template <class Tag, bool VEC, bool ADJ>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotaryArgs a, RotPlan pl) {
  constexpr int V = VEC ? 16 / Tag::ES : 1;  // components of a piece
  constexpr int U = 2;                       // items whose loads leave together
  extern __shared__ __align__(16) float2 cs[];  // [tok][P], then the tokens' x and y
  int64_t *const at = (int64_t *)(cs + pl.tok * a.P);
  const int tid = threadIdx.x;
  const int64_t n0 = (int64_t)blockIdx.x * pl.tok;
  const int64_t left = a.B * a.S - n0;
  const int ntok = left < pl.tok ? (int)left : pl.tok;
  const int h0 = blockIdx.y * pl.heads;
  const int nh = a.H - h0 < pl.heads ? a.H - h0 : pl.heads;
  for (int t = tid; t < ntok; t += kRotThreads) {  // (up to 1024 tokens of one pair)
    const int64_t n = n0 + t, b = pl.small ? (int64_t)((uint32_t)n / (uint32_t)a.S) : n / a.S, s = n - b * a.S;
    at[2 * t] = b * a.x.b + s * a.x.s;
    at[2 * t + 1] = b * a.y.b + s * a.y.s;
  }
  __syncthreads();
  const int per_token = nh * pl.per, items = ntok * per_token;
  auto item = [&](int g) {
    // (several tokens only with all heads in one run, so that per_token is the plan's)
    RotItem r;
    r.t = pl.tok == 1 ? 0 : quotient(g, pl.magic_tok);
    const int e = g - r.t * per_token;
    const int hd = quotient(e, pl.magic), i = e - hd * pl.per;
    const bool turn = i < pl.turn;
    const int piece = turn ? (ADJ && !VEC ? 2 * i : i * V) : 2 * a.P + (i - pl.turn) * V;
    r.pos = turn ? (ADJ && VEC ? i * V / 2 : i * V) : -1;
    r.x = at[2 * r.t] + (int64_t)(h0 + hd) * a.x.h + piece * Tag::ES;
    r.y = at[2 * r.t + 1] + (int64_t)(h0 + hd) * a.y.h + piece * Tag::ES;
    r.next = (ADJ ? (VEC ? 0 : 1) : a.P) * Tag::ES;
    return r;
  };
  // the first items' loads are under way while the angles are computed
  u32x4 lo[U], hi[U];
  RotItem it[U];
  auto load = [&](int g0) {
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int g = g0 + j * kRotThreads;
      it[j].t = -1;
      if (g >= items) continue;
      it[j] = item(g);
      const char *p = a.x.p + it[j].x;
      if constexpr (VEC) {
        lo[j] = *(const u32x4 *)p;
        if (!ADJ && it[j].pos >= 0) hi[j] = *(const u32x4 *)(p + it[j].next);
      } else if constexpr (Tag::W16) {
        lo[j][0] = *(const u16 *)p;
        if (it[j].pos >= 0) hi[j][0] = *(const u16 *)(p + it[j].next);
      } else {
        lo[j][0] = *(const uint32_t *)p;
        if (it[j].pos >= 0) hi[j][0] = *(const uint32_t *)(p + it[j].next);
      }
    }
  };
  load(tid);
  for (int e = tid; e < ntok * a.P; e += kRotThreads) {
    const int t = e / a.P, i = e - t * a.P;
    const int64_t n = n0 + t, b = pl.small ? (int64_t)((uint32_t)n / (uint32_t)a.S) : n / a.S, s = n - b * a.S;
    int axis = 0;
#pragma unroll
    for (int j = 0; j + 1 < kMaxAxes; ++j) axis += j + 1 < a.axes && i >= a.first[j];
    const int64_t pa = axis * a.pos_a + b * a.pos_b + s * a.pos_s;
    const double p = a.pos64 ? (double)((const int64_t *)a.pos)[pa] : (double)((const int32_t *)a.pos)[pa];
    const double turns = p * (double)a.freqs[i] * 0.15915494309189533577;
    const double exact = 2.0 * (turns - rint(turns));  // half turns, -1 .. 1
    const float half = (float)exact, rest = (float)((exact - (double)half) * 3.14159265358979323846);
    float sn, cn;
    sincospif(half, &sn, &cn);
    const float s1 = __builtin_fmaf(cn, rest, sn);  // (|rest| < 2^-23)
    cn = __builtin_fmaf(-sn, rest, cn);
    cs[e] = make_float2(cn, a.reverse ? -s1 : s1);
  }
  __syncthreads();
  for (int g0 = tid; g0 < items; g0 += U * kRotThreads) {
    if (g0 != tid) load(g0);
#pragma unroll
    for (int j = 0; j < U; ++j) {
      if (it[j].t < 0) continue;
      char *q = a.y.p + it[j].y;
      const float2 *ct = cs + it[j].t * a.P + it[j].pos;
      if constexpr (VEC) {
        if (it[j].pos < 0) {
          store16(q, lo[j]);
        } else if constexpr (ADJ) {
          float f[V];
          unpack<Tag>(lo[j], f);
#pragma unroll
          for (int k = 0; k < V; k += 2) {
            const float2 r = ct[k / 2];
            rotate(&f[k], &f[k + 1], r);
          }
          store16(q, repack<Tag>(f));
        } else {
          float fl[V], fh[V];
          unpack<Tag>(lo[j], fl);
          unpack<Tag>(hi[j], fh);
#pragma unroll
          for (int k = 0; k < V; ++k) {
            const float2 r = ct[k];
            rotate(&fl[k], &fh[k], r);
          }
          store16(q, repack<Tag>(fl));
          store16(q + it[j].next, repack<Tag>(fh));
        }
      } else {
        const uint32_t l = lo[j][0], m = hi[j][0];
        if (it[j].pos < 0) {
          if constexpr (Tag::W16)
            *(u16 *)q = (u16)l;
          else
            *(uint32_t *)q = l;
        } else {
          float u, w;
          if constexpr (Tag::W16)
            u = to_f32<Tag>((u16)l), w = to_f32<Tag>((u16)m);
          else
            u = __uint_as_float(l), w = __uint_as_float(m);
          const float2 r = *ct;
          rotate(&u, &w, r);
          store1<Tag>(q, u);
          store1<Tag>(q + it[j].next, w);
        }
      }
    }
  }
}

template <class Tag>
hipError_t launch(const RotaryArgs &a, hipStream_t stream) {
  constexpr int V = 16 / Tag::ES;
  const Tokens *t[2] = {&a.x, &a.y};
  bool vec = a.D % V == 0 && (a.adjacent ? 2 * a.P : a.P) % V == 0;
  for (const Tokens *k : t) vec = vec && ((uintptr_t)k->p | k->b | k->s | k->h) % 16 == 0;
  RotPlan pl;
  pl.turn = vec ? (a.adjacent ? 2 * a.P : a.P) / V : a.P;
  pl.per = pl.turn + (vec ? (a.D - 2 * a.P) / V : a.D - 2 * a.P);
  const int64_t most = ((int64_t)1 << 31) / ((int64_t)pl.per * pl.per);
  pl.heads = (int)(a.H < most ? a.H : most);
  const int64_t n = a.B * a.S, items = (int64_t)pl.heads * pl.per;
  const int64_t runs = (a.H + pl.heads - 1) / pl.heads;
  pl.tok = 1;
  while (runs == 1 && items * pl.tok < 4 * kRotThreads && 2 * pl.tok * a.P <= 2048 && n / (2 * pl.tok) >= 1024)
    pl.tok *= 2;
  pl.magic = reciprocal(pl.per);
  pl.magic_tok = reciprocal(items);
  const int64_t blocks = (n + pl.tok - 1) / pl.tok;
  if (blocks > (1 << 23) || runs > 65535) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)blocks, (unsigned)runs);
  pl.small = n < ((int64_t)1 << 31);
  const size_t lds = (size_t)pl.tok * (a.P * sizeof(float2) + 16);
  if (vec) {
    if (a.adjacent)
      rotary_kernel<Tag, true, true><<<grid, kRotThreads, lds, stream>>>(a, pl);
    else
      rotary_kernel<Tag, true, false><<<grid, kRotThreads, lds, stream>>>(a, pl);
  } else {
    if (a.adjacent)
      rotary_kernel<Tag, false, true><<<grid, kRotThreads, lds, stream>>>(a, pl);
    else
      rotary_kernel<Tag, false, false><<<grid, kRotThreads, lds, stream>>>(a, pl);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(Dt dt, const RotaryArgs &a, hipStream_t stream) {
  switch (dt) {
    case Dt::F32: return launch<TagF32>(a, stream);
    case Dt::BF16: return launch<TagBF16>(a, stream);
    case Dt::F16: return launch<TagF16>(a, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace wbmm
