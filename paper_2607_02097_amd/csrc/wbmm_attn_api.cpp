// C-ABI front end of the rotary positions and the cross attention: argument
// validation, status codes and dispatch.  As in wbmm_api.cpp, every check runs
// on the host before any GPU work is enqueued; nothing here allocates, prints
// or aborts.
#include <math.h>
#include <stdint.h>

#include "wbmm.h"
#include "wbmm_attn_internal.h"

namespace {

using wbmm::AttnArgs;
using wbmm::AttnEntry;
using wbmm::Dt;
using wbmm::RotaryArgs;
using wbmm::Tokens;

int64_t elem_size(int64_t dtype) { return dtype == WBMM_F32 ? 4 : dtype == WBMM_BF16 || dtype == WBMM_F16 ? 2 : 0; }

bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }

wbmm_status from_hip(hipError_t e) {
  // a grid past the launch limits is a shape without a kernel
  return e == hipSuccess ? WBMM_OK : e == hipErrorInvalidConfiguration ? WBMM_ERR_UNSUPPORTED : WBMM_ERR_HIP;
}

// Addresses that a strided [B, S, H, D] tensor reaches, in bytes.
struct Span {
  uintptr_t at;
  int64_t bytes;                // of the whole range
  int64_t row;                  // of one row of components
  int64_t stride[3], n[3];      // entries, tokens, heads (stride 0: one of them)
};

constexpr int64_t kFar = (int64_t)1 << 46;  // bytes; keeps every offset far from overflow

// Checks a tensor of n elements in each dimension and describes it.
bool describe(const wbmm_tokens &t, int64_t B, int64_t S, int64_t H, int64_t D, int64_t es, Tokens *out, Span *sp) {
  const int64_t st[3] = {t.stride_b, t.stride_s, t.stride_h}, n[3] = {B, S, H};
  int64_t far = D;
  for (int i = 0; i < 3; ++i) {
    if (st[i] < 0) return false;
    if (n[i] > 1) {
      if (st[i] > kFar / (n[i] - 1)) return false;
      far += st[i] * (n[i] - 1);
    }
    if (far > kFar) return false;
  }
  const bool empty = B == 0 || S == 0;
  if (!empty && (!t.data || !aligned(t.data, (size_t)es))) return false;
  // a stride over a single element is never taken
  *out = {(char *)t.data, B > 1 ? st[0] * es : 0, S > 1 ? st[1] * es : 0, H > 1 ? st[2] * es : 0};
  *sp = {(uintptr_t)t.data, empty ? 0 : far * es, D * es, {out->b, out->s, out->h}, {B, S, H}};
  return true;
}

// An output's elements must not share an address.
bool folds(const Tokens &t, int64_t B, int64_t S, int64_t H, int64_t D, int64_t es) {
  if (B == 0 || S == 0) return false;
  // dimensions in the order of their strides, each past the whole of the ones below
  int64_t st[3] = {t.b, t.s, t.h}, n[3] = {B, S, H}, reach = D * es;
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (st[j] < st[i]) {
        const int64_t a = st[i], c = n[i];
        st[i] = st[j], n[i] = n[j], st[j] = a, n[j] = c;
      }
  for (int i = 0; i < 3; ++i) {
    if (n[i] <= 1) continue;
    if (st[i] < reach) return true;
    reach += st[i] * (n[i] - 1);
  }
  return false;
}

// What lies below the period p: the range of the dimensions with smaller
// strides; -1 if a larger stride is not a multiple of p.
int64_t within(const Span &x, int64_t p) {
  int64_t r = x.row;
  for (int i = 0; i < 3; ++i) {
    if (x.stride[i] >= p && x.stride[i] % p != 0) return -1;
    if (x.stride[i] < p) r += x.stride[i] * (x.n[i] - 1);
  }
  return r;
}

bool clash(const Span &a, const Span &b) {
  if (a.bytes == 0 || b.bytes == 0) return false;
  if (a.at + (uintptr_t)a.bytes <= b.at || b.at + (uintptr_t)b.bytes <= a.at) return false;
  // slices of one joint tensor: apart within a period that both repeat by
  for (int i = 0; i < 6; ++i) {
    const int64_t p = i < 3 ? a.stride[i] : b.stride[i - 3];
    if (p <= 0) continue;
    const int64_t ra = within(a, p), rb = within(b, p);
    if (ra < 0 || rb < 0) continue;
    const int64_t m = b.at >= a.at ? (int64_t)((b.at - a.at) % (uintptr_t)p) : (int64_t)((a.at - b.at) % (uintptr_t)p);
    const int64_t shift = b.at >= a.at || m == 0 ? m : p - m;  // of b behind a
    if (shift >= ra && shift + rb <= p) return false;
  }
  return true;
}

wbmm_status rotary(const wbmm_rotary_args *g, void *stream, int reverse) {
  if (!g) return WBMM_ERR_INVALID_ARG;
  const int64_t es = elem_size(g->dtype);
  if (!es) return WBMM_ERR_UNSUPPORTED;
  if (g->B < 0 || g->S < 0 || g->H <= 0 || g->D <= 0 || g->axes <= 0) return WBMM_ERR_INVALID_ARG;
  if (g->axes > wbmm::kMaxAxes || g->D > wbmm::kMaxRotaryDim || g->H > INT32_MAX / g->D) return WBMM_ERR_UNSUPPORTED;
  if (g->position_bytes != 4 && g->position_bytes != 8) return WBMM_ERR_INVALID_ARG;
  RotaryArgs a = {};
  int64_t pairs = 0;
  for (int i = 0; i < g->axes; ++i) {
    if (g->sections[i] < 0 || g->sections[i] > g->D) return WBMM_ERR_INVALID_ARG;
    pairs += g->sections[i];
    a.first[i] = (int)pairs;
  }
  if (pairs < 1 || 2 * pairs > g->D) return WBMM_ERR_INVALID_ARG;
  if (pairs > wbmm::kMaxPairs) return WBMM_ERR_UNSUPPORTED;
  if (g->pos_stride_a < 0 || g->pos_stride_b < 0 || g->pos_stride_s < 0) return WBMM_ERR_INVALID_ARG;
  Span x, y;
  if (!describe(g->x, g->B, g->S, g->H, g->D, es, &a.x, &x) || !describe(g->y, g->B, g->S, g->H, g->D, es, &a.y, &y))
    return WBMM_ERR_INVALID_ARG;
  if (folds(a.y, g->B, g->S, g->H, g->D, es)) return WBMM_ERR_INVALID_ARG;
  if (g->B == 0 || g->S == 0) return WBMM_OK;
  if (g->B > kFar / g->S) return WBMM_ERR_UNSUPPORTED;
  if (!g->positions || !g->freqs || !aligned(g->positions, (size_t)g->position_bytes) || !aligned(g->freqs, 4))
    return WBMM_ERR_INVALID_ARG;
  const bool in_place = a.x.p == a.y.p && a.x.b == a.y.b && a.x.s == a.y.s && a.x.h == a.y.h;
  if (!in_place && clash(x, y)) return WBMM_ERR_INVALID_ARG;
  const int64_t n[3] = {g->axes, g->B, g->S}, st[3] = {g->pos_stride_a, g->pos_stride_b, g->pos_stride_s};
  int64_t far = 1;
  for (int i = 0; i < 3; ++i) {
    if (n[i] > 1 && st[i] > kFar / (n[i] - 1)) return WBMM_ERR_INVALID_ARG;
    far += st[i] * (n[i] - 1);
  }
  const Span pos = {(uintptr_t)g->positions, far * g->position_bytes, far * g->position_bytes, {}, {}};
  const Span fr = {(uintptr_t)g->freqs, pairs * 4, pairs * 4, {}, {}};
  if (clash(y, pos) || clash(y, fr)) return WBMM_ERR_INVALID_ARG;
  a.pos = g->positions;
  a.pos_a = g->pos_stride_a, a.pos_b = g->pos_stride_b, a.pos_s = g->pos_stride_s;
  a.pos64 = g->position_bytes == 8;
  a.freqs = g->freqs;
  a.B = g->B, a.S = g->S;
  a.H = (int)g->H, a.D = (int)g->D, a.P = (int)pairs, a.axes = (int)g->axes;
  a.adjacent = g->adjacent != 0;
  a.reverse = reverse;
  return from_hip(wbmm::launch_rotary((Dt)g->dtype, a, (hipStream_t)stream));
}

// Sizes of an attention call; fills everything but the tensors.
wbmm_status attn_sizes(const wbmm_cross_attention_args *g, AttnArgs *a) {
  if (!g) return WBMM_ERR_INVALID_ARG;
  if (!elem_size(g->dtype)) return WBMM_ERR_UNSUPPORTED;
  if (g->B < 0 || g->Sq < 0 || g->Sk < 0 || g->Hq <= 0 || g->Hk <= 0 || g->D <= 0) return WBMM_ERR_INVALID_ARG;
  if (g->Hq % g->Hk != 0) return WBMM_ERR_INVALID_ARG;
  // (lse / scale has to be within float32's range)
  if (!(g->scale >= 1e-30) || !isfinite((float)g->scale)) return WBMM_ERR_INVALID_ARG;
  if (g->D > wbmm::kMaxHeadDim) return WBMM_ERR_UNSUPPORTED;
  // rows of a key head and states are counted in 32 bits, with room to spare
  const int64_t lim = (int64_t)1 << 30, G = g->Hq / g->Hk;
  if (g->B > lim || g->Hq > lim || g->Sk > lim || (g->Sq > 0 && G > lim / g->Sq)) return WBMM_ERR_UNSUPPORTED;
  if (g->B > 0 && g->Hq > lim / g->B) return WBMM_ERR_UNSUPPORTED;
  if (g->mask_stride_b < 0 || g->mask_stride_s < 0) return WBMM_ERR_INVALID_ARG;
  if (g->kv_lens && !aligned(g->kv_lens, 4)) return WBMM_ERR_INVALID_ARG;
  *a = AttnArgs{};
  a->B = g->B;
  a->Sq = (int)g->Sq, a->Sk = (int)g->Sk, a->Hq = (int)g->Hq, a->Hk = (int)g->Hk, a->G = (int)G, a->D = (int)g->D;
  a->R = (int)(g->Sq * G);
  a->scale = (float)g->scale;
  a->c = (float)(g->scale * 1.4426950408889634074);
  if (!isfinite(a->c)) return WBMM_ERR_INVALID_ARG;
  a->lens = g->kv_lens;
  a->mask = g->key_mask;
  a->mask_b = g->mask_stride_b, a->mask_s = g->mask_stride_s;
  return WBMM_OK;
}

int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

// Space of a planned call.
struct Space {
  int64_t sum_do, top_v, part_o, part_l, part_dk, part_dv, total;
};
Space forward_space(const AttnArgs &a) {
  Space w = {};
  if (a.splits > 1) {
    const int64_t rows = (int64_t)a.splits * a.B * a.Hk * a.R;
    w.part_l = up16(rows * a.D * 4);
    w.total = w.part_l + up16(rows * 4);
  }
  return w;
}
Space backward_space(const AttnArgs &a) {
  Space w = {};
  const int64_t bh = a.B * a.Hk;
  w.sum_do = a.one_pass ? 0 : up16(bh * a.R * 8);
  w.top_v = w.sum_do + (a.powers ? up16(bh * a.R * 4) : 0);
  w.part_o = w.top_v + (a.powers ? up16(bh * ((a.Sk + 31) / 32) * 4) : 0);
  const int64_t dq = a.splits > 1 ? up16((int64_t)a.splits * a.B * a.Hk * a.R * a.D * 4) : 0;
  const int64_t part = a.row_parts > 1 ? up16((int64_t)a.row_parts * a.B * a.Hk * a.Sk * a.D * 4) : 0;
  w.part_dk = w.part_o + dq;
  w.part_dv = w.part_dk + part;
  w.total = w.part_dv + part;
  return w;
}

bool rows16(const Tokens *const *t, int n, int64_t row) {
  bool ok = row % 16 == 0;
  for (int i = 0; i < n; ++i) ok = ok && ((uintptr_t)t[i]->p | t[i]->b | t[i]->s | t[i]->h) % 16 == 0;
  return ok;
}

// Offsets in a tile of states fit 32 bits (states further apart are moved
// element by element).
bool near(const AttnArgs &a) { return a.k.s < (1 << 24) && a.v.s < (1 << 24); }

bool clash_any(const Span &o, const Span *in, int n) {
  for (int i = 0; i < n; ++i)
    if (clash(o, in[i])) return true;
  return false;
}

Span flat(const void *p, int64_t bytes) { return {(uintptr_t)p, p ? bytes : 0, bytes, {}, {}}; }

// lens, mask and workspace as address ranges.
void side_spans(const wbmm_cross_attention_args *g, Span *sp) {
  sp[0] = flat(g->kv_lens, g->B * 4);
  sp[1] = flat(g->key_mask, g->B && g->Sk ? (g->B - 1) * g->mask_stride_b + (g->Sk - 1) * g->mask_stride_s + 1 : 0);
}

bool mask_far(const wbmm_cross_attention_args *g) {
  return (g->B > 1 && g->mask_stride_b > kFar / (g->B - 1)) || (g->Sk > 1 && g->mask_stride_s > kFar / (g->Sk - 1));
}

template <class Tag>
hipError_t run(const AttnArgs &a, bool vec, bool back, hipStream_t st) {
  if (back) return vec ? AttnEntry<Tag>::template backward<true>(a, st) : AttnEntry<Tag>::template backward<false>(a, st);
  return vec ? AttnEntry<Tag>::template forward<true>(a, st) : AttnEntry<Tag>::template forward<false>(a, st);
}

hipError_t run(int64_t dtype, const AttnArgs &a, bool vec, bool back, hipStream_t st) {
  return dtype == WBMM_F32    ? run<wbmm::TagF32>(a, vec, back, st)
         : dtype == WBMM_BF16 ? run<wbmm::TagBF16>(a, vec, back, st)
                              : run<wbmm::TagF16>(a, vec, back, st);
}

}  // namespace

extern "C" {

wbmm_status wbmm_rotary_forward(const wbmm_rotary_args *args, void *stream) { return rotary(args, stream, 0); }

wbmm_status wbmm_rotary_backward(const wbmm_rotary_args *args, void *stream) { return rotary(args, stream, 1); }

size_t wbmm_cross_attention_forward_workspace_bytes(const wbmm_cross_attention_args *g) {
  AttnArgs a;
  if (attn_sizes(g, &a) != WBMM_OK) return 0;
  wbmm::attn_plan_forward((Dt)g->dtype, &a);
  return wbmm::attn_grids_fit(a, false) ? (size_t)forward_space(a).total : 0;
}

wbmm_status wbmm_cross_attention_forward(const wbmm_cross_attention_args *g, void *stream) {
  AttnArgs a;
  wbmm_status s = attn_sizes(g, &a);
  if (s != WBMM_OK) return s;
  const int64_t es = elem_size(g->dtype);
  Span in[5], out;
  if (!describe(g->q, g->B, g->Sq, g->Hq, g->D, es, &a.q, &in[0]) ||
      !describe(g->k, g->B, g->Sk, g->Hk, g->D, es, &a.k, &in[1]) ||
      !describe(g->v, g->B, g->Sk, g->Hk, g->D, es, &a.v, &in[2]) ||
      !describe(g->out, g->B, g->Sq, g->Hq, g->D, es, &a.o, &out) || mask_far(g))
    return WBMM_ERR_INVALID_ARG;
  side_spans(g, in + 3);
  const Span lse = flat(g->lse, g->B * g->Hq * g->Sq * 4);
  if (g->lse && !aligned(g->lse, 4)) return WBMM_ERR_INVALID_ARG;
  if (folds(a.o, g->B, g->Sq, g->Hq, g->D, es) || clash_any(out, in, 5) || clash_any(lse, in, 5) || clash(out, lse))
    return WBMM_ERR_INVALID_ARG;
  if (g->B == 0 || g->Sq == 0) return WBMM_OK;
  wbmm::attn_plan_forward((Dt)g->dtype, &a);
  if (!wbmm::attn_grids_fit(a, false)) return WBMM_ERR_UNSUPPORTED;
  const Space w = forward_space(a);
  if (w.total > 0) {
    const Span ws = flat(g->workspace, w.total);
    if (!g->workspace || g->workspace_bytes < w.total || !aligned(g->workspace, 16) || clash_any(ws, in, 5) ||
        clash(ws, out) || clash(ws, lse))
      return WBMM_ERR_INVALID_ARG;
    a.part_o = (float *)((char *)g->workspace + w.part_o);
    a.part_l = (float *)((char *)g->workspace + w.part_l);
  }
  a.lse = g->lse;
  const Tokens *t[] = {&a.q, &a.k, &a.v, &a.o};
  return from_hip(run(g->dtype, a, rows16(t, 4, g->D * es) && near(a), false, (hipStream_t)stream));
}

size_t wbmm_cross_attention_backward_workspace_bytes(const wbmm_cross_attention_args *g) {
  AttnArgs a;
  if (attn_sizes(g, &a) != WBMM_OK) return 0;
  wbmm::attn_plan_backward((Dt)g->dtype, &a);
  return wbmm::attn_grids_fit(a, true) ? (size_t)backward_space(a).total : 0;
}

wbmm_status wbmm_cross_attention_backward(const wbmm_cross_attention_args *g, void *stream) {
  AttnArgs a;
  wbmm_status s = attn_sizes(g, &a);
  if (s != WBMM_OK) return s;
  const int64_t es = elem_size(g->dtype);
  Span in[8], out[3];
  if (!describe(g->q, g->B, g->Sq, g->Hq, g->D, es, &a.q, &in[0]) ||
      !describe(g->k, g->B, g->Sk, g->Hk, g->D, es, &a.k, &in[1]) ||
      !describe(g->v, g->B, g->Sk, g->Hk, g->D, es, &a.v, &in[2]) ||
      !describe(g->out, g->B, g->Sq, g->Hq, g->D, es, &a.o, &in[3]) ||
      !describe(g->dout, g->B, g->Sq, g->Hq, g->D, es, &a.dout, &in[4]) ||
      !describe(g->dq, g->B, g->Sq, g->Hq, g->D, es, &a.dq, &out[0]) ||
      !describe(g->dk, g->B, g->Sk, g->Hk, g->D, es, &a.dk, &out[1]) ||
      !describe(g->dv, g->B, g->Sk, g->Hk, g->D, es, &a.dv, &out[2]) || mask_far(g))
    return WBMM_ERR_INVALID_ARG;
  side_spans(g, in + 5);
  in[7] = flat(g->lse, g->B * g->Hq * g->Sq * 4);
  if (g->B > 0 && g->Sq > 0 && (!g->lse || !aligned(g->lse, 4))) return WBMM_ERR_INVALID_ARG;
  if (folds(a.dq, g->B, g->Sq, g->Hq, g->D, es) || folds(a.dk, g->B, g->Sk, g->Hk, g->D, es) ||
      folds(a.dv, g->B, g->Sk, g->Hk, g->D, es))
    return WBMM_ERR_INVALID_ARG;
  for (const Span &o : out)
    if (clash_any(o, in, 8)) return WBMM_ERR_INVALID_ARG;
  if (clash(out[0], out[1]) || clash(out[0], out[2]) || clash(out[1], out[2])) return WBMM_ERR_INVALID_ARG;
  if (g->B == 0 || (g->Sq == 0 && g->Sk == 0)) return WBMM_OK;
  wbmm::attn_plan_backward((Dt)g->dtype, &a);
  if (!wbmm::attn_grids_fit(a, true)) return WBMM_ERR_UNSUPPORTED;
  const Space w = backward_space(a);
  if (w.total > 0) {
    const Span ws = flat(g->workspace, w.total);
    if (!g->workspace || g->workspace_bytes < w.total || !aligned(g->workspace, 16) || clash_any(ws, in, 8) ||
        clash_any(ws, out, 3))
      return WBMM_ERR_INVALID_ARG;
    a.rowstat = (float2 *)g->workspace;
    a.sum_do = (float *)((char *)g->workspace + w.sum_do);
    a.top_v = (float *)((char *)g->workspace + w.top_v);
    a.part_o = (float *)((char *)g->workspace + w.part_o);
    a.part_dk = (float *)((char *)g->workspace + w.part_dk);
    a.part_dv = (float *)((char *)g->workspace + w.part_dv);
  }
  a.lse = g->lse;
  const Tokens *t[] = {&a.q, &a.k, &a.v, &a.o, &a.dout, &a.dq, &a.dk, &a.dv};
  return from_hip(run(g->dtype, a, rows16(t, 8, g->D * es) && near(a), true, (hipStream_t)stream));
}

}  // extern "C"

namespace wbmm {

namespace {

constexpr int64_t kUnits = 256;  // compute units

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t clamp(int64_t n, int64_t lo, int64_t hi) { return n < lo ? lo : n > hi ? hi : n; }

// By the number of workgroups.  Larger tiles of rows read the states less often
// and feed the matrix cores better, but need one for three compute units in
// four.  Tiles of 32 rows can take the states in parts, for a workgroup on every
// compute unit (one unit reads about 50 GB/s, whatever its waves), of 96 states
// at least, since the parts are joined by a launch of its own; single tokens
// over long sequences in up to eight workgroups a unit, so that unequal lengths
// even out.  One token, 8 key heads of 128 components: 196 states 6.4 us in one
// part, 8.1 in two; 784 states 11.7 us in one part, 9.1 in four, 8.2 in eight;
// 12544 states 129 us in one, 25 in 8, 17 in 24 to 32.  32 tokens over 12544
// states each: 294 us in one part, 285 in eight, 306 in 32.
void plan_by_count(AttnArgs *a) {
  const int64_t bh = a->B * a->Hk, enough = kUnits * 3 / 4;
  a->splits = 1;
  if (a->R > 64 && bh * cdiv(a->R, 128) >= enough) {
    a->tile_rows = 128;
  } else if (a->R > 32 && bh * cdiv(a->R, 64) >= enough) {
    a->tile_rows = 64;
  } else {
    a->tile_rows = 32;
    const int64_t wgs = bh * cdiv(a->R, 32);
    int64_t n = wgs > 0 ? kUnits / wgs : 1;
    if (a->R <= 32 && wgs > 0) n = n > a->Sk / 1536 ? n : clamp(8 * kUnits / wgs, 1, a->Sk / 1536);
    a->splits = a->Sk > 384 ? (int)clamp(n, 1, clamp(a->Sk / 96, 1, 64)) : 1;
  }
}

// An account of a launch's time.  Workgroups that own rows, and for gradients
// others that own states, run through products of 32 x 32 blocks, one wave's
// after the other; the launch takes the root of the sum of the squares of the
// longest of them and of all of them spread over the chip.  Larger tiles of rows
// read the states less often.  Parts take a launch more, and their sums are
// written and read.
struct Account {
  int products;          // of a block, for owners of rows
  double start;          // of a workgroup, in products
  double few;            // a block in tiles of 32 rows, whose states come from memory
  double spread[3];      // what shares a unit, in tiles of 128, 64 and 32 rows
  double block, launch;  // us
};
constexpr double kPartRate = 2.2e6;  // bytes of partial sums, written and read, a us

// Tiles and parts that take the least time by an account.
void plan_by(const Account &c, bool grads, AttnArgs *a) {
  const double bh = (double)(a->B * a->Hk), states = (double)cdiv(a->Sk, 32), rows = (double)cdiv(a->R, 32);
  const double n_states = grads ? bh * cdiv(a->Sk, 128) : 0;
  constexpr int counts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
  double best = INFINITY;
  for (int i = 0, tile = 128; i < 3; ++i, tile /= 2) {
    if (tile > 32 && a->R <= tile / 2) continue;
    const double n_rows = bh * cdiv(a->R, tile);
    for (int s : counts) {
      if (s > 1 && (tile > 32 || s > a->Sk / 96 || n_rows * s > 4 * kUnits)) break;
      const double by_rows = c.start + c.products * states * tile / 128 / s * (tile == 32 ? c.few : 1);
      for (int p : counts) {
        if (p > 1 && (p > a->R / 64 || !grads || n_states * p > 4 * kUnits)) break;
        const double by_states = grads ? c.start + 3.6 * rows / p : 0, longest = by_rows > by_states ? by_rows : by_states;
        const double all = (n_rows * s * by_rows * c.spread[i] + n_states * p * by_states * c.spread[0]) / kUnits;
        double t = c.block * sqrt(longest * longest + all * all);
        if (s > 1) t += c.launch + bh * a->R * a->D * 8 * s / kPartRate;
        if (p > 1) t += c.launch + bh * a->Sk * a->D * 16 * p / kPartRate;
        if (t < best) best = t, a->tile_rows = tile, a->splits = s, a->row_parts = p;
      }
    }
  }
}

}  // namespace

// The constants of the accounts are fitted to 184 (forward) and 200 sizes (4 to
// 192 heads, 33 to 4000 rows, 48 to 8000 states, 32 to 128 components), each in up
// to 30 arrangements.  What they choose takes 3.5 % more than the best of them on
// average (the gradients 2 %, in float32 5 %), where limits on the numbers of
// workgroups took 6 % (13 %, 10 %); in float32 the forward, at 5 % by either, goes
// by the limits.  bfloat16, forward: 16 heads of 590 rows over 51 states in tiles
// of 128 rows, not 32: 12.2 -> 6.6 us.  Gradients: 16 heads of 600 rows, 784
// states of 128 components: 128 rows a tile, no parts, 32 us (in tiles of 64 rows
// 35, of 32 rows 40, rows in two parts 46); 8 heads of 800 rows, 196 states: rows
// in 6 parts, 23 us (one part 37).  They also lose, at most a quarter of the time
// by limits: float32 gradients, 24 key heads of 588 rows, 236 states of 128
// components 103 -> 131 us; float16 forward, 2 key heads of 2744 rows, 507 masked
// states of 64 9.0 -> 11.3; bfloat16 forward, 16 heads of 88 rows, 2340 masked
// states of 72 16.3 -> 19.4; bfloat16 gradients, 24 heads of 149 rows, 2251 states
// of 72 37.8 -> 44.7.  Lengths and masks, which lie on the device, are not in them.
void attn_plan_forward(Dt dt, AttnArgs *a) {
  const int wide = (a->D + 31) / 32 * 32;  // components, as they are multiplied
  a->row_parts = 1;
  if (a->R <= 32 || dt == Dt::F32)
    plan_by_count(a);
  else
    plan_by({2, 8.5, 1.2, {0.96, 1.63, 1.84}, 4.75e-3 * (wide + 64), 2.5}, false, a);
}

// Few rows (16-bit): all gradients in one pass over the states, in parts for a
// workgroup on every unit: 64 key heads of 128 components over 3136 states
// 114 us in one part, 49 in four (one workgroup a unit), 60 in eight.
void attn_plan_backward(Dt dt, AttnArgs *a) {
  const int64_t bh = a->B * a->Hk;
  if (dt != Dt::F32 && a->R > 0 && a->R <= one_pass_rows(a->D) && a->Sk > 0) {
    a->tile_rows = 32;
    a->one_pass = a->row_parts = 1;
    a->splits = (int)clamp(bh > 0 ? kUnits / bh : 1, 1, clamp(a->Sk / 96, 1, 64));
    return;
  }
  a->powers = dt == Dt::F16;
  const int wide = (a->D + 31) / 32 * 32;
  if (dt == Dt::F32)
    plan_by({3, 7.4, 0.98, {1.13, 1.37, 1.13}, 50e-3 * (wide + 16), 5}, true, a);
  else
    plan_by({3, 16.5, 2, {0.62, 0.92, 1.24}, 5.75e-3 * (wide + 64), 5}, true, a);
}

bool attn_grids_fit(const AttnArgs &a, bool back) {
  constexpr int64_t most = 1 << 23;  // workgroups of 256 threads in a launch
  const int64_t bh = a.B * a.Hk, rows = bh * a.R;
  // (bh is at most 2^30, the tiles of a head fewer: no overflow)
  const int64_t of_rows = bh * cdiv(a.R, a.one_pass ? 1 << 30 : a.tile_rows) * a.splits;
  if (of_rows > most) return false;
  if (a.splits > 1 && rows > most * 256 / a.D) return false;
  if (!back) return true;
  if (!a.one_pass && (rows > most * 16 || bh * cdiv(a.Sk, 128) * a.row_parts > most - of_rows)) return false;
  return a.row_parts == 1 || bh * a.Sk <= most * 256 / a.D;
}

}  // namespace wbmm
