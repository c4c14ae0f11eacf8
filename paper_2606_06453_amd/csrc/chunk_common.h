// What the kernels over a chunk of new tokens share: their arguments, the way from a workgroup to its tokens,
// values of single cache rows, and the attention of one row token by token.
#pragma once
#include "mxfp4.h"
#include "vx_device.h"
#include "vx_internal.h"

namespace vx {
namespace chunk {

struct ChunkArgs {
  const uint16_t* q;
  int64_t q_row, q_head;                   // strides in elements
  const int32_t* q_indptr;
  const int32_t* q_lens;
  int num_rows;
  const void* k;
  const void* v;
  const int32_t* indptr;
  const int32_t* indices;
  const int32_t* seq_lens;
  int batch, max_pages, H, g, Hq, ps, ps_shift, num_phys;
  int bs, bs_shift;                        // selection unit in tokens
  const int32_t* sel_pages;
  const int32_t* sel_count;
  int max_sel;
  int max_blocks;                          // blocks per request bound (selections)
  int window;                              // 0: none
  int causal;
  float scale_log2;                        // sm_scale * log2(e) * K scale
  float v_scale;
  uint16_t* out;
  float* lse;
  int tokens;                              // tokens of a tile
  int splits;
  float* part_o;                           // [row][Hq][splits][Dv] weighted means
  float2* part_ml;                         // [row][Hq][splits]: reference (log2) and sum
};

// A workgroup's tokens: n of request i, from its chunk's token t0 on.
struct Tile {
  int i, n;
  int64_t row0;                            // row of the first
  int p0;                                  // its position (negative: before the request's first token)
  int len;                                 // tokens of the request that its page list holds
  const int32_t* pages;                    // the list
};

// A request's rows in q.
__device__ __forceinline__ void rows_of_request(const ChunkArgs& a, int i, int& q0, int& n) {
  q0 = min(max(a.q_indptr[i], 0), a.num_rows);
  n = min(max(a.q_indptr[i + 1], q0), a.num_rows) - q0;
  if (a.q_lens) n = min(max(a.q_lens[i], 0), n);
}

// Tile x of the grid, or false for one with no token.  No plan is made first:
//   up to 64 requests   lane i counts the tiles of request i, and the requests take the grid in the order of their
//                       lengths, the longest first (the last workgroups to start are then the shortest: 48 requests
//                       of up to 12000 tokens, a quarter of them prompts, 1078 -> 894 us);
//   more                request i owns the tiles from floor(q_indptr[i] / T) + i on, at least as many as its rows need;
//                       its request is the last one that starts at or before x, found 64 requests at a time.
// Within a request the last tile, whose tokens attend most, comes first.
__device__ __forceinline__ bool find_tile(const ChunkArgs& a, int x, Tile& t) {
  const int T = a.tokens, lane = lane_id();
  int i, q0, n, y;
  if (a.batch <= kWave) {
    int tiles = 0, len = 0;
    if (lane < a.batch) {
      rows_of_request(a, lane, q0, n);
      len = a.seq_lens[lane];
      tiles = (n + T - 1) / T;
    }
    int start = 0;
    for (int j = 0; j < a.batch; j++) {
      const int other = __builtin_amdgcn_readlane(len, j), c = __builtin_amdgcn_readlane(tiles, j);
      if (other > len || (other == len && j < lane)) start += c;
    }
    const uint64_t mine = __ballot(lane < a.batch && x >= start && x < start + tiles);
    if (!mine) return false;
    i = __builtin_ctzll(mine);
    q0 = __builtin_amdgcn_readlane(q0, i);
    n = __builtin_amdgcn_readlane(n, i);
    y = x - __builtin_amdgcn_readlane(start, i);
  } else {
    int lo = 0, hi = a.batch;
    while (hi - lo > 1) {
      const int step = (hi - lo + kWave - 1) / kWave;
      const int at = lo + lane * step;
      const bool below = at < hi && min(max(a.q_indptr[min(at, hi - 1)], 0), a.num_rows) / T + at <= x;
      const int c = max(__popcll(__ballot(below)), 1);
      hi = min(hi, lo + c * step);
      lo += (c - 1) * step;
    }
    i = __builtin_amdgcn_readfirstlane(lo);
    rows_of_request(a, i, q0, n);
    y = x - q0 / T - i;
    if (y < 0 || y >= (n + T - 1) / T) return false;
  }
  const int t0 = ((n + T - 1) / T - 1 - y) * T;
  const int L = max(a.seq_lens[i], 0), base = a.indptr[i];
  t.i = i;
  t.n = min(T, n - t0);
  t.row0 = q0 + t0;
  t.p0 = L - n + t0;
  t.pages = a.indices + base;
  const int P = num_pages(L, a.ps, a.indptr[i + 1] - base, a.max_pages);
  t.len = (int)min((int64_t)L, (int64_t)P * a.ps);
  return true;
}

// Tiles that n rows of a batch can have: the grid of find_tile.
inline int64_t most_tiles(int64_t n, int tokens, int64_t batch) {
  return batch <= kWave ? (n + batch * (tokens - 1)) / tokens : (n + tokens - 1) / tokens + batch - 1;
}

// The tokens [lo, hi) that the token at position p attends.
__device__ __forceinline__ int first_key(const ChunkArgs& a, int p) {
  return a.window > 0 ? max(p - a.window + 1, 0) : 0;
}
__device__ __forceinline__ int end_key(const ChunkArgs& a, const Tile& t, int p) {
  return p < 0 ? 0 : a.causal ? min(p + 1, t.len) : t.len;
}

// ---- single rows of the cache ------------------------------------------------------------------
// Slice of (page, head): K or V of ps tokens.
template <int D, int KT>
__device__ __forceinline__ const uint8_t* slice_of(const ChunkArgs& a, const void* base, int64_t page, int h) {
  const int64_t s = page * a.H + h;
  if constexpr (KT == kKvMxFp4) return static_cast<const uint8_t*>(base) + s * mx::slice_bytes(a.ps, D);
  return static_cast<const uint8_t*>(base) + s * a.ps * D * (KT == kKvBf16 ? 2 : 1);
}

// 8 values (without an fp8 cache's scale) of chunk c8 of token t of a slice.
template <int D, int KT>
__device__ __forceinline__ void chunk_of(const ChunkArgs& a, const uint8_t* s, bool v, int t, int c8, float (&x)[8]) {
  if constexpr (KT == kKvBf16) {
    const uint4 w = *reinterpret_cast<const uint4*>(s + 2 * ((int64_t)t * D + 8 * c8));
    const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; e++) {
      x[2 * e] = bf16lo(ws[e]);
      x[2 * e + 1] = bf16hi(ws[e]);
    }
  } else if constexpr (KT == kKvMxFp4) {
    const uint32_t w = v ? mx::get_v_codes(s, t, c8, D) : *reinterpret_cast<const uint32_t*>(s + mx::k_code(t, c8, D));
    const uint32_t e =
        s[mx::codes_bytes(a.ps, D) + (v ? mx::v_scale(t, c8 >> 2, D) : mx::k_scale(t, c8 >> 2, D))];
    const float f = mx::scale_operand(e);
    const float2_t p[4] = {mx::pair_f32<0>(w, f), mx::pair_f32<1>(w, f), mx::pair_f32<2>(w, f), mx::pair_f32<3>(w, f)};
#pragma unroll
    for (int e2 = 0; e2 < 4; e2++) {
      x[2 * e2] = p[e2][0];
      x[2 * e2 + 1] = p[e2][1];
    }
  } else {
    const uint2 w = *reinterpret_cast<const uint2*>(s + (int64_t)t * D + 8 * c8);
    const int ws[2] = {(int)w.x, (int)w.y};
#pragma unroll
    for (int e = 0; e < 2; e++) {
      float2_t lo, hi;
      if constexpr (KT == kKvFp8E4M3) {
        lo = __builtin_amdgcn_cvt_pk_f32_fp8(ws[e], false);
        hi = __builtin_amdgcn_cvt_pk_f32_fp8(ws[e], true);
      } else {
        lo = __builtin_amdgcn_cvt_pk_f32_bf8(ws[e], false);
        hi = __builtin_amdgcn_cvt_pk_f32_bf8(ws[e], true);
      }
      x[4 * e] = lo[0];
      x[4 * e + 1] = lo[1];
      x[4 * e + 2] = hi[0];
      x[4 * e + 3] = hi[1];
    }
  }
}

// ---- one row, token by token --------------------------------------------------------------------
// The entries of a list of token runs: run e is tokens first + e * len .. (ids == nullptr) or block ids[e],
// and belongs to token x of the tile where bit x of its mask is set.
struct Runs {
  int lo, hi;                              // entries
  const uint16_t* ids;
  const uint16_t* masks;                   // by block id
  int shift;                               // log2 tokens of a run (at most 6)
};

// State of a row: reference and sum of the weights in the log2 domain, channels 8 c8 + j of the weighted mean in the
// lanes c8 = lane, lane + 64 below DV / 8, and whether the row attends a token at all.
template <int DV>
struct RowState {
  static constexpr int N = (DV / 8 + kWave - 1) / kWave;
  float m, l, o[N][8];
  bool any;
};
// The reference of a part whose tokens all score -inf (a part without a token: -inf).  A row of such parts alone has no
// weights, 0 / 0, and gives NaN; a row without a token gives zeros.
constexpr float kNoWeight = -3.0e38f;

// A wave's attention of query head r of tile token x over the runs, without matrix operands: a token that
// the row does not attend is not multiplied by a zero weight but left out, so that its infinities and NaN
// do not reach the row; and the mean is kept instead of the sum, which may pass the largest float where the
// mean does not.  Lanes hold a token each for the scores and a chunk of channels each for the mean.
template <int D, int DV, int KT>
__device__ void attend_row(const ChunkArgs& a, const Tile& t, int h, int r, int x, const Runs& runs,
                           RowState<DV>& st) {
  const int lane = lane_id();
  const int p = t.p0 + x, from = first_key(a, p), to = end_key(a, t, p);
  const uint16_t* q = a.q + (t.row0 + x) * a.q_row + (int64_t)(h * a.g + r) * a.q_head;
  const void* vbase = a.v ? a.v : a.k;
  st.m = -INFINITY;
  st.l = 0.f;
  st.any = false;
#pragma unroll
  for (int u = 0; u < RowState<DV>::N; u++)
#pragma unroll
    for (int e = 0; e < 8; e++) st.o[u][e] = 0.f;
  const int per = kWave >> runs.shift;     // runs a step
  for (int e0 = runs.lo; e0 < runs.hi; e0 += per) {
    const int e = e0 + (lane >> runs.shift);
    int tok = 0;
    bool ok = e < runs.hi;
    if (ok) {
      const int id = runs.ids ? runs.ids[e] : e;
      if (runs.ids) ok = (runs.masks[id] >> x) & 1;
      tok = (id << runs.shift) + (lane & ((1 << runs.shift) - 1));
      ok = ok && tok >= from && tok < to;
    }
    const uint64_t some = __ballot(ok);
    if (!some) continue;
    st.any = true;
    int page = 0;
    float z = -INFINITY;
    const int at = tok & (a.ps - 1);
    if (ok) {
      page = (int)clamp_page(t.pages[tok >> a.ps_shift], a.num_phys);
      const uint8_t* s = slice_of<D, KT>(a, a.k, page, h);
      float dot = 0.f;
      for (int c8 = 0; c8 < D / 8; c8++) {
        float kx[8];
        chunk_of<D, KT>(a, s, false, at, c8, kx);
#pragma unroll
        for (int j = 0; j < 8; j++) dot = fmaf(bf16_to_f32(q[8 * c8 + j]), kx[j], dot);
      }
      z = dot * a.scale_log2;
    }
    float mx_ = z != z ? -INFINITY : z;
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) mx_ = fmaxf(mx_, xor_shfl(mx_, s));
    const float m_new = fmaxf(st.m, mx_);
    const float alpha = st.m == -INFINITY ? 0.f : exp2f(st.m - m_new);
    const float w = !ok || (z == -INFINITY) ? 0.f : exp2f(z - m_new);
    float sum = w;
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) sum += xor_shfl(sum, s);
    const float l_new = st.l * alpha + sum, inv = l_new != 0.f ? 1.f / l_new : 0.f;   // NaN stays NaN
    const float shrink = st.l * alpha * inv;
    st.l = l_new;
    st.m = m_new;
#pragma unroll
    for (int u = 0; u < RowState<DV>::N; u++)
#pragma unroll
      for (int j = 0; j < 8; j++) st.o[u][j] *= shrink;
    for (uint64_t left = some; left; left &= left - 1) {
      const int src = __builtin_ctzll(left);
      const float ws = __shfl(w, src, kWave) * inv;
      const int pg = __builtin_amdgcn_readlane(page, src), ta = __builtin_amdgcn_readlane(at, src);
      const uint8_t* s = a.v ? slice_of<DV, KT>(a, vbase, pg, h) : slice_of<D, KT>(a, vbase, pg, h);
#pragma unroll
      for (int u = 0; u < RowState<DV>::N; u++) {
        const int c8 = lane + kWave * u;
        if (c8 < DV / 8) {
          float vx_[8];
          if (a.v) chunk_of<DV, KT>(a, s, true, ta, c8, vx_);
          else chunk_of<D, KT>(a, s, false, ta, c8, vx_);
#pragma unroll
          for (int j = 0; j < 8; j++) st.o[u][j] = fmaf(ws, vx_[j], st.o[u][j]);
        }
      }
    }
  }
}

// The row's result, or its part of it (split s).
template <int DV>
__device__ __forceinline__ void store_row(const ChunkArgs& a, int64_t row, int head, int s, const RowState<DV>& st) {
  const int lane = lane_id();
  const int64_t at = row * a.Hq + head;
  const bool parts = a.splits > 1, bare = st.any && st.l == 0.f;
#pragma unroll
  for (int u = 0; u < RowState<DV>::N; u++) {
    const int c8 = lane + kWave * u;
    if (c8 >= DV / 8) continue;
    if (parts) {
      float4* dst = reinterpret_cast<float4*>(a.part_o + (at * a.splits + s) * DV + 8 * c8);
      dst[0] = make_float4(st.o[u][0], st.o[u][1], st.o[u][2], st.o[u][3]);
      dst[1] = make_float4(st.o[u][4], st.o[u][5], st.o[u][6], st.o[u][7]);
    } else {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; e++)
        w[e] = bare ? 0x7fc07fc0u : f32_to_bf16_rne(st.o[u][2 * e] * a.v_scale) | (f32_to_bf16_rne(st.o[u][2 * e + 1] * a.v_scale) << 16);
      *reinterpret_cast<uint4*>(a.out + at * DV + 8 * c8) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  if (lane == 0) {
    if (parts) a.part_ml[at * a.splits + s] = make_float2(bare ? kNoWeight : st.m, st.l);
    else if (a.lse) a.lse[at] = st.l > 0.f ? (st.m + log2f(st.l)) * 0.693147180559945309f : st.l == 0.f ? -INFINITY : st.l;
  }
}

}  // namespace chunk
}  // namespace vx
