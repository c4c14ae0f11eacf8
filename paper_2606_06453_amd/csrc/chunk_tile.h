// Matrix operands of 16 cache tokens, from any cache type, and the online softmax that the tile kernels
// share.
//
// S^T = K Q^T is a 16x16x32 product: operand A is 16 tokens (row = lane & 15), operand B 16 query rows.  Lane
// (grp, col) then holds S[token 4 grp + i][row col], which, as bf16, is operand B of O^T = V^T P^T if the
// contraction's slot (grp, j) is token 4 grp + j of the first 16 tokens (j < 4) or of the second: no value
// changes lanes between the two products.  Operands straight from the cache (RawV): row `col` of V^T operand j is channel
// col * D / 16 + j, so that a lane's channels are neighbours in a V row.
#pragma once
#include "chunk_common.h"

namespace vx {
namespace chunk {

typedef __bf16 bf16x2v_t __attribute__((ext_vector_type(2)));

template <int KT, bool HI>
__device__ __forceinline__ uint32_t fp8_pair(uint32_t w) {
  bf16x2v_t r;
  if constexpr (KT == kKvFp8E4M3) r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, HI);
  else r = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8((int)w, 1.0f, HI);
  return __builtin_bit_cast(uint32_t, r);
}

// Two floats as a bf16 pair, to nearest even.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const bf16x2v_t v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}

// Channels of a lane's k-step kk of a K row (and of the query): 8 from here.  Types below 16 bits take D / 4
// consecutive channels a lane, so that they arrive in 16-byte loads.
template <int D, int KT>
__device__ __forceinline__ int k_channel(int kk, int grp) {
  return KT == kKvBf16 ? 32 * kk + 8 * grp : D / 4 * grp + 8 * kk;
}

// 16 tokens of K, and of V, as loaded: fp8 or mxfp4.
template <int D, int KT>
struct RawK {
  static constexpr int W = KT == kKvMxFp4 ? D / 32 : D / 16;     // words of a lane's part
  uint32_t w[W], scale;                    // scale: mxfp4
};
template <int D, int KT>
struct RawV {
  static constexpr int W = D / 64;         // words of an fp8 row's part
  static constexpr int N = KT == kKvMxFp4 ? D / 32 : 4 * W;
  uint32_t w[N], scale;
};

// Loads go through buffer resources of the page's slices: a base that all lanes share, lane offsets that stay the same
// for the whole kernel, and zeros for what lies behind the last token that any row attends, which may hold
// anything.
struct Slices {
  __amdgpu_buffer_rsrc_t k, v, k_scale, v_scale;         // scales: mxfp4
};
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const uint8_t* base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, bytes, 0x00020000);
}

// Tokens t .. t + 15 (t a multiple of 16, the same in all lanes) of a page, the first n of which are looked at (0 to 16).
template <int D, int KT>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const uint8_t* slice, int t, int n) {
  constexpr int kRow = KT == kKvMxFp4 ? D / 2 : D;
  // mxfp4: four tokens of V share their codes' bytes; what is not looked at goes by its scale
  return rsrc(slice + t * kRow, (KT == kKvMxFp4 ? 16 : n) * kRow);
}
template <int D>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t scales_of(const ChunkArgs& a, const uint8_t* slice, int t) {
  return rsrc(slice + mx::codes_bytes(a.ps, D) + t * (D / 32), 16 * (D / 32));
}

template <int N>
__device__ __forceinline__ void load_words(__amdgpu_buffer_rsrc_t r, int off, uint32_t* w) {
  if constexpr (N >= 4) {
#pragma unroll
    for (int x = 0; x < N; x += 4) {
      const u32x4_t y = __builtin_amdgcn_raw_buffer_load_b128(r, off + 4 * x, 0, 0);
      w[x] = y.x;
      w[x + 1] = y.y;
      w[x + 2] = y.z;
      w[x + 3] = y.w;
    }
  } else if constexpr (N == 2) {
    const u32x2_t y = __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0);
    w[0] = y.x;
    w[1] = y.y;
  } else {
    w[0] = __builtin_amdgcn_raw_buffer_load_b32(r, off, 0, 0);
  }
}

// n: tokens of the run that some row may attend.
template <int D, int KT>
__device__ __forceinline__ void load_k(const ChunkArgs& a, const uint8_t* slice, int t, int n, int col, int grp, RawK<D, KT>& r) {
  const __amdgpu_buffer_rsrc_t k = rows_of<D, KT>(slice, t, n);
  if constexpr (KT == kKvMxFp4) {
    load_words<D / 32>(k, col * (D / 2) + D / 8 * grp, r.w);
    r.scale = __builtin_amdgcn_raw_buffer_load_b8(scales_of<D>(a, slice, t), col * (D / 32) + D / 4 * grp / 32, 0, 0);
  } else {
    load_words<D / 16>(k, col * D + D / 4 * grp, r.w);
  }
}
template <int D, int KT>
__device__ __forceinline__ void load_v(const ChunkArgs& a, const uint8_t* slice, int t, int n, int col, int grp, RawV<D, KT>& r) {
  const __amdgpu_buffer_rsrc_t v = rows_of<D, KT>(slice, t, n);
  if constexpr (KT == kKvMxFp4) {
    load_words<D / 32>(v, (grp * 16 + col) * (D / 8), r.w);
    r.scale = __builtin_amdgcn_raw_buffer_load_b32(scales_of<D>(a, slice, t), (grp * (D / 32) + col * (D / 16) / 32) * 4, 0, 0);
    const int left = n - 4 * grp;                        // byte x: token 4 grp + x; a scale of 0 is 2^-127
    r.scale &= left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << (8 * left)) - 1;
  } else {
    constexpr int W = RawV<D, KT>::W;
#pragma unroll
    for (int x = 0; x < 4; x++) load_words<W>(v, (4 * grp + x) * D + col * (D / 16), r.w + x * W);
  }
}

// Operand A of k-step kk.
template <int D, int KT>
__device__ __forceinline__ bf16x8_t k_operand(const RawK<D, KT>& r, int kk) {
  u32x4_t w;
  if constexpr (KT == kKvMxFp4) {
    const float s = mx::scale_operand(r.scale);
    const uint32_t c = r.w[kk];
    w = u32x4_t{mx::pair_bf16<0>(c, s), mx::pair_bf16<1>(c, s), mx::pair_bf16<2>(c, s), mx::pair_bf16<3>(c, s)};
  } else {
    const uint32_t lo = r.w[2 * kk], hi = r.w[2 * kk + 1];
    w = u32x4_t{fp8_pair<KT, false>(lo), fp8_pair<KT, true>(lo), fp8_pair<KT, false>(hi), fp8_pair<KT, true>(hi)};
  }
  return __builtin_bit_cast(bf16x8_t, w);
}

// Rows 4 grp + x of V as bf16 words: channels col * D / 16 ..
template <int D, int KT>
__device__ __forceinline__ void v_rows(const RawV<D, KT>& r, uint32_t (&v)[4][D / 32]) {
#pragma unroll
  for (int x = 0; x < 4; x++) {
    if constexpr (KT == kKvMxFp4) {
      const float s = mx::scale_operand((r.scale >> (8 * x)) & 255);
      if constexpr (D == 128) {
        v[x][0] = mx::pair_bf16<0>(r.w[x], s);
        v[x][1] = mx::pair_bf16<1>(r.w[x], s);
        v[x][2] = mx::pair_bf16<2>(r.w[x], s);
        v[x][3] = mx::pair_bf16<3>(r.w[x], s);
      } else {
        const uint32_t c = r.w[x >> 1];
        v[x][0] = (x & 1) ? mx::pair_bf16<2>(c, s) : mx::pair_bf16<0>(c, s);
        v[x][1] = (x & 1) ? mx::pair_bf16<3>(c, s) : mx::pair_bf16<1>(c, s);
      }
    } else {
#pragma unroll
      for (int w = 0; w < D / 64; w++) {
        v[x][2 * w] = fp8_pair<KT, false>(r.w[x * (D / 64) + w]);
        v[x][2 * w + 1] = fp8_pair<KT, true>(r.w[x * (D / 64) + w]);
      }
    }
  }
}

// Operand A of O^T for output channels col * D / 16 + j, from the rows of two runs of 16 tokens.
template <int W>
__device__ __forceinline__ bf16x8_t v_operand(const uint32_t (&v0)[4][W], const uint32_t (&v1)[4][W], int j) {
  const uint32_t sel = (j & 1) ? 0x07060302u : 0x05040100u;
  const int w = j >> 1;
  const u32x4_t o = {__builtin_amdgcn_perm(v0[1][w], v0[0][w], sel), __builtin_amdgcn_perm(v0[3][w], v0[2][w], sel),
                     __builtin_amdgcn_perm(v1[1][w], v1[0][w], sel), __builtin_amdgcn_perm(v1[3][w], v1[2][w], sel)};
  return __builtin_bit_cast(bf16x8_t, o);
}

// Largest over the four lanes of a column (lanes 16 and 32 apart), and sum.
__device__ __forceinline__ float column_max(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float column_sum(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The weights' reference: 2^kAhead past the score that moved it, so that it moves seldom and weights stay
// below 2.
constexpr float kAhead = 8.f;
constexpr float kNoScore = -3.0e38f;       // the reference before the first score

// The rows of a wave: operand B, what each attends, and the state of their softmax.
template <int D, int DV, int RT>
struct Rows {
  static constexpr int KS = D / 32, NJ = DV / 16;
  bf16x8_t q[RT][KS];
  int from[RT], to[RT], bit[RT];
  int all_from, all_to;                    // tokens that every row attends (uniform)
  f32x4_t acc[RT][NJ];
  float m[RT], l[RT];
};

template <int D, int DV, int KT, int RT>
__device__ __forceinline__ void begin_rows(const ChunkArgs& a, const Tile& t, int h, int r0, int col, int grp,
                                           Rows<D, DV, RT>& w) {
  const int rows = t.n * a.g;
#pragma unroll
  for (int rt = 0; rt < RT; rt++) {
    const int r = r0 + 16 * rt + col, x = r / a.g, head = r - x * a.g;
    const bool there = r < rows;
    const uint16_t* src = a.q + (t.row0 + (there ? x : 0)) * a.q_row + (int64_t)(h * a.g + (there ? head : 0)) * a.q_head;
#pragma unroll
    for (int kk = 0; kk < D / 32; kk++) {
      w.q[rt][kk] = *reinterpret_cast<const bf16x8_t*>(src + k_channel<D, KT>(kk, grp));
      if (!there) w.q[rt][kk] = bf16x8_t{};
    }
    w.from[rt] = first_key(a, t.p0 + x);
    w.to[rt] = there ? end_key(a, t, t.p0 + x) : 0;
    w.bit[rt] = x & 15;
    w.m[rt] = kNoScore;
    w.l[rt] = 0.f;
#pragma unroll
    for (int j = 0; j < DV / 16; j++) w.acc[rt][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  w.all_from = first_key(a, t.p0 + t.n - 1);
  w.all_to = end_key(a, t, t.p0);
}

// Scores of tokens that a row does not attend: s holds 16 tokens from tok0 and 16 from tok1.  Few steps need it: the
// statement without instructions keeps its comparisons, which the compiler would make ahead of the branch around
// it for every step, inside.
template <int D, int DV, int RT>
__device__ __forceinline__ void mask_scores(f32x4_t (&s)[RT][2], int tok0, int tok1, int grp, const Rows<D, DV, RT>& w) {
  asm volatile("" : "+s"(tok0), "+s"(tok1));
  const int t0 = tok0 + 4 * grp, t1 = tok1 + 4 * grp;
#pragma unroll
  for (int rt = 0; rt < RT; rt++)
#pragma unroll
    for (int i = 0; i < 4; i++) {
      s[rt][0][i] = t0 + i < w.to[rt] && t0 + i >= w.from[rt] ? s[rt][0][i] : -INFINITY;
      s[rt][1][i] = t1 + i < w.to[rt] && t1 + i >= w.from[rt] ? s[rt][1][i] : -INFINITY;
    }
}

// One step of the softmax: the scores s of 32 tokens become weights p, operand B of O^T = V^T P^T.  The weights are
// taken at the present references first and seldom reach 2 (bit 14 of a bf16 number; infinities and NaN have it too);
// only then the references move.  A weight is the sum of two bf16 parts, p[.][0] and what it leaves, p[.][1], each to
// the nearest: 2^-16 of it at most, as in the decode step.  One part alone (2^-8) would be as large an error as the
// rounding of the output.  The sum takes the weights before their rounding.
// LISTED: mask0 and mask1 hold the tile tokens that list the first and the last 16 tokens; another's reference for
// them is infinite, and their weights are zero.
template <int D, int DV, int RT, bool LISTED>
__device__ __forceinline__ void softmax_step(float scale_log2, const f32x4_t (&s)[RT][2], int mask0, int mask1,
                                             Rows<D, DV, RT>& w, uint32_t (&p)[RT][2][4]) {
  float x[RT][8];
  auto on = [&](int rt, int e) { return !LISTED || ((e ? mask1 : mask0) >> w.bit[rt] & 1) != 0; };
  auto weigh = [&](int rt) {
    const float m[2] = {on(rt, 0) ? w.m[rt] : INFINITY, on(rt, 1) ? w.m[rt] : INFINITY};
#pragma unroll
    for (int i = 0; i < 8; i++) x[rt][i] = __builtin_amdgcn_exp2f(fmaf(s[rt][i >> 2][i & 3], scale_log2, -m[i >> 2]));
#pragma unroll
    for (int i = 0; i < 4; i++) p[rt][0][i] = pack_bf16(x[rt][2 * i], x[rt][2 * i + 1]);
  };
  uint32_t seen = 0;
#pragma unroll
  for (int rt = 0; rt < RT; rt++) {
    weigh(rt);
    seen |= (p[rt][0][0] | p[rt][0][1]) | (p[rt][0][2] | p[rt][0][3]);
  }
  if (__builtin_expect(__any((seen & 0x40004000u) != 0), 0)) {
#pragma unroll
    for (int rt = 0; rt < RT; rt++) {
      float top = -INFINITY;
#pragma unroll
      for (int e = 0; e < 2; e++)
        if (on(rt, e)) top = fmaxf(top, fmaxf(fmaxf(s[rt][e][0], s[rt][e][1]), fmaxf(s[rt][e][2], s[rt][e][3])) * scale_log2);
      const float c = column_max(top), next = c > w.m[rt] ? c + kAhead : w.m[rt];
      const float alpha = __builtin_amdgcn_exp2f(w.m[rt] - next);
      w.m[rt] = next;
      w.l[rt] *= alpha;
#pragma unroll
      for (int j = 0; j < DV / 16; j++)
#pragma unroll
        for (int i = 0; i < 4; i++) w.acc[rt][j][i] *= alpha;
      weigh(rt);
    }
  }
#pragma unroll
  for (int rt = 0; rt < RT; rt++) {
#pragma unroll
    for (int i = 0; i < 4; i++)
      p[rt][1][i] = pack_bf16(x[rt][2 * i] - bf16lo(p[rt][0][i]), x[rt][2 * i + 1] - bf16hi(p[rt][0][i]));
    w.l[rt] += ((x[rt][0] + x[rt][1]) + (x[rt][2] + x[rt][3])) + ((x[rt][4] + x[rt][5]) + (x[rt][6] + x[rt][7]));
  }
}

__device__ __forceinline__ bf16x8_t p_operand(const uint32_t (&p)[4]) {
  const u32x4_t w = {p[0], p[1], p[2], p[3]};
  return __builtin_bit_cast(bf16x8_t, w);
}

}  // namespace chunk
}  // namespace vx
