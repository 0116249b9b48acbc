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

template <class Tag> __device__ inline float load1(const char *p) {
  if constexpr (Tag::W16)
    return to_f32<Tag>(*(const u16 *)p);
  else
    return *(const float *)p;
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
  uint32_t magic, magic_tok;  // ceil(2^32 / per), ceil(2^32 / items of a token); 0 for 1
};

// e / d by d's rounded-up reciprocal in 2^-32 (exact while e d < 2^32).
__device__ inline int quotient(int e, uint32_t magic) { return magic ? (int)__umulhi((uint32_t)e, magic) : e; }
inline uint32_t reciprocal(int64_t d) { return d == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + d - 1) / d); }

template <class Tag, bool VEC>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotaryArgs a, RotPlan pl) {
  constexpr int V = 16 / Tag::ES;
  extern __shared__ __align__(16) float2 cs[];  // [tok][P]
  const int tid = threadIdx.x;
  const int64_t n0 = (int64_t)blockIdx.x * pl.tok;
  const int64_t left = a.B * a.S - n0;
  const int ntok = left < pl.tok ? (int)left : pl.tok;
  const int h0 = blockIdx.y * pl.heads;
  const int nh = a.H - h0 < pl.heads ? a.H - h0 : pl.heads;
  for (int e = tid; e < ntok * a.P; e += kRotThreads) {
    const int t = e / a.P, i = e - t * a.P;
    const int64_t n = n0 + t, b = n / a.S, s = n - b * a.S;
    int axis = 0;
#pragma unroll
    for (int j = 0; j + 1 < kMaxAxes; ++j) axis += j + 1 < a.axes && i >= a.first[j];
    const int64_t at = axis * a.pos_a + b * a.pos_b + s * a.pos_s;
    const double p = a.pos64 ? (double)((const int64_t *)a.pos)[at] : (double)((const int32_t *)a.pos)[at];
    const double turns = p * (double)a.freqs[i] * 0.15915494309189533577;
    const float half = (float)(2.0 * (turns - rint(turns)));  // half turns, -1 .. 1
    float sn, cn;
    sincospif(half, &sn, &cn);
    cs[e] = make_float2(cn, a.reverse ? -sn : sn);
  }
  __syncthreads();
  const int per_token = nh * pl.per, items = ntok * per_token;
  for (int g = tid; g < items; g += kRotThreads) {
    // (several tokens only with all heads in one run, so that per_token is the plan's)
    const int t = pl.tok == 1 ? 0 : quotient(g, pl.magic_tok);
    const int e = g - t * per_token;
    const int hd = quotient(e, pl.magic), i = e - hd * pl.per;
    const int64_t n = n0 + t, b = n / a.S, s = n - b * a.S;
    const float2 *ct = cs + t * a.P;
    {
      const char *xr = a.x.p + b * a.x.b + s * a.x.s;
      char *yr = a.y.p + b * a.y.b + s * a.y.s;
      const char *xh = xr + (int64_t)(h0 + hd) * a.x.h;
      char *yh = yr + (int64_t)(h0 + hd) * a.y.h;
      if constexpr (VEC) {
        if (i < pl.turn && !a.adjacent) {
          const int o = i * 16, o2 = o + a.P * Tag::ES;
          const u32x4 lo = *(const u32x4 *)(xh + o), hi = *(const u32x4 *)(xh + o2);
          float fl[V], fh[V];
          unpack<Tag>(lo, fl);
          unpack<Tag>(hi, fh);
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const float2 r = ct[i * V + j];
            const float u = fl[j], w = fh[j];
            fl[j] = u * r.x - w * r.y;
            fh[j] = u * r.y + w * r.x;
          }
          *(u32x4 *)(yh + o) = repack<Tag>(fl);
          *(u32x4 *)(yh + o2) = repack<Tag>(fh);
        } else if (i < pl.turn) {
          float f[V];
          unpack<Tag>(*(const u32x4 *)(xh + i * 16), f);
#pragma unroll
          for (int j = 0; j < V; j += 2) {
            const float2 r = ct[(i * V + j) / 2];
            const float u = f[j], w = f[j + 1];
            f[j] = u * r.x - w * r.y;
            f[j + 1] = u * r.y + w * r.x;
          }
          *(u32x4 *)(yh + i * 16) = repack<Tag>(f);
        } else {
          const int o = 2 * a.P * Tag::ES + (i - pl.turn) * 16;
          *(u32x4 *)(yh + o) = *(const u32x4 *)(xh + o);
        }
      } else {
        if (i < pl.turn) {
          const int o = (a.adjacent ? 2 * i : i) * Tag::ES, o2 = o + (a.adjacent ? 1 : a.P) * Tag::ES;
          const float2 r = ct[i];
          const float u = load1<Tag>(xh + o), w = load1<Tag>(xh + o2);
          store1<Tag>(yh + o, u * r.x - w * r.y);
          store1<Tag>(yh + o2, u * r.y + w * r.x);
        } else {
          const int o = (2 * a.P + i - pl.turn) * Tag::ES;
          if constexpr (Tag::W16)
            *(u16 *)(yh + o) = *(const u16 *)(xh + o);
          else
            *(float *)(yh + o) = *(const float *)(xh + o);
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
  const size_t lds = (size_t)pl.tok * a.P * sizeof(float2);
  if (vec)
    rotary_kernel<Tag, true><<<grid, kRotThreads, lds, stream>>>(a, pl);
  else
    rotary_kernel<Tag, false><<<grid, kRotThreads, lds, stream>>>(a, pl);
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
