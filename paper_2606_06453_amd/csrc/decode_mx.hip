// Sparse paged attention over an mxfp4 cache (GQA geometry): the split kernel of decode.hip's work
// plan for slices of E2M1 codes and E8M0 scales.
//
// A (page of 16, KV head) is 1088 bytes of K and of V at D = 128, a quarter of bf16, so the time per
// byte is a quarter and the vector instructions per token decide.  A wave takes two 16-token tiles
// per round, 32 tokens:
//   S^T = K Q^T   MFMA 16x16x32 per tile: a lane's K codes are D/4 consecutive channels of one token
//                 (one load), widened with their scale by the E2M1 conversion (a code times a power
//                 of two is a bf16 value, so nothing is rounded)
//   softmax       log2 domain, against a running bound of a head's scores instead of their maximum.  A score
//                 that passes it moves it 2^8 past that score; until the next one does, a round needs no
//                 exchange between lanes.  Weights are at most 1, as against the maximum (2^-8 for the score
//                 that moved the bound: fp32 sums and the two bf16 parts carry those as exactly)
//   O^T += V^T P^T  MFMA 16x16x32 over the 32 tokens: a lane's V codes are one piece (D/16 channels) of
//                 four tokens side by side, widened and paired by tokens (v_perm).  P's layout is that
//                 of S^T, 4 tokens of each tile per lane, and V^T's rows follow it.
// P is the sum of two bf16 parts, hi = p and lo = p - hi, each to the nearest: 2^-17 of p, unbiased as the
// weights' sum needs (parts cut to 8 bits are up to 0.5% faster, but 2^-15 too small: 0.6% of the outputs
// were not the nearest bf16, now 0.2%).  With at most 8 query heads per KV head the 16 columns hold every
// head twice, the hi parts in columns 0 to 7 and the lo parts in 8 to 15, so one MFMA per operand does
// both; else two.
//
// D = 128, 8 KV heads: 64 requests of 128 selected pages of 16 and 32 query heads take 29.2 us (4.9 TB/s
// of the cache; the launches' start and the merge are the rest), 128 requests of 256 blocks of 32 and 48
// query heads 180 us (6.0 TB/s, a long read's rate being 6.3), one request 8.4 us.  Vector instructions take
// 55% and 65% of the CU cycles of the first two.  With 16 query heads per KV head, two MFMAs per operand,
// 64 requests take 31.8 us instead of 30.1; 32 requests of 32768 tokens 197 us at 1 head, 205 at 4, 213 at 8, 228
// at 16 (floor 181).
#include <algorithm>

#include "decode_common.h"
#include "mxfp4.h"

namespace vx {
using namespace dec;
namespace {

constexpr int kMxWaves = 4;               // per workgroup
constexpr float kRoomLog2 = 8.f;
constexpr float kNoMax = -3.4028234e38f;  // running bound before the first token: no score is below it

template <int D>
struct MxTile {
  uint32_t k[D / 32], v[D / 32];          // codes: token col, channels D/4 * grp ..; tokens 4 grp .., piece col
  uint32_t ke, ve;                        // scale bytes: k's; v's four tokens
};

// Lane constants of a tile's loads, bytes from the tile's codes and scales.
struct MxLane {
  uint32_t kc, vc, ks, vs;
};

template <int D>
__device__ __forceinline__ MxLane mx_lane(int col, int grp) {
  return MxLane{(uint32_t)(col * (D / 2) + grp * (D / 8)), (uint32_t)(grp * (2 * D) + col * (D / 8)),
                (uint32_t)(col * (D / 32) + grp * D / 128), (uint32_t)(grp * (D / 8) + col / (512 / D) * 4)};
}

// The tile at token t0 of a slice.  Buffer loads: the slice's address is uniform and goes into the
// resource, the lane's part is the same for every tile, so a load costs no vector instruction and no
// access can leave the slice.
constexpr int kStreamLoad = 2;             // cache policy bits: nt
template <int D>
__device__ __forceinline__ void mx_load(const uint8_t* __restrict__ k, const uint8_t* __restrict__ v, int64_t slice,
                                        int slice_bytes, int t0, int ps, const MxLane& l, MxTile<D>& t) {
  const __amdgpu_buffer_rsrc_t kr = coherent_rsrc(k + slice, (uint32_t)slice_bytes);
  const __amdgpu_buffer_rsrc_t vr = coherent_rsrc(v + slice, (uint32_t)slice_bytes);
  const int codes = t0 * (D / 2), scales = ps * (D / 2) + t0 * (D / 32);
  if constexpr (D == 128) {
    const u32x4v_t a = __builtin_amdgcn_raw_buffer_load_b128(kr, (int)l.kc, codes, kStreamLoad);
    const u32x4v_t b = __builtin_amdgcn_raw_buffer_load_b128(vr, (int)l.vc, codes, kStreamLoad);
#pragma unroll
    for (int x = 0; x < 4; x++) {
      t.k[x] = a[x];
      t.v[x] = b[x];
    }
  } else {
    typedef unsigned int u32x2_load __attribute__((ext_vector_type(2)));
    const u32x2_load a = __builtin_amdgcn_raw_buffer_load_b64(kr, (int)l.kc, codes, kStreamLoad);
    const u32x2_load b = __builtin_amdgcn_raw_buffer_load_b64(vr, (int)l.vc, codes, kStreamLoad);
#pragma unroll
    for (int x = 0; x < 2; x++) {
      t.k[x] = a[x];
      t.v[x] = b[x];
    }
  }
  t.ke = __builtin_amdgcn_raw_buffer_load_b8(kr, (int)l.ks, scales, kStreamLoad);
  t.ve = __builtin_amdgcn_raw_buffer_load_b32(vr, (int)l.vs, scales, kStreamLoad);
}

// S^T of a tile: lane (grp, col) holds tokens 4 grp + i of query column col.
template <int D>
__device__ __forceinline__ f32x4_t mx_scores(const MxTile<D>& t, const bf16x8_t (&qv)[D / 32]) {
  const float s = mx::scale_operand(t.ke);
  f32x4_t st = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int kk = 0; kk < D / 32; kk++) {
    const u32x4_t w = {mx::pair_bf16<0>(t.k[kk], s), mx::pair_bf16<1>(t.k[kk], s), mx::pair_bf16<2>(t.k[kk], s),
                       mx::pair_bf16<3>(t.k[kk], s)};
    st = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, w), qv[kk], st, 0, 0, 0);
  }
  return st;
}

// Channels 2 x and 2 x + 1 of token row r of a tile's V.
template <int D>
__device__ __forceinline__ uint32_t mx_widen_v(const MxTile<D>& t, int r, int x) {
  // the conversion takes the exponent field alone: the byte of each row shifted there will do
  const float s = __uint_as_float(r == 0 ? t.ve << 23 : r == 1 ? t.ve << 15 : r == 2 ? t.ve << 7 : t.ve >> 1);
  const uint32_t c = D == 128 ? t.v[r] : t.v[r >> 1];
  switch (D == 128 ? x : 2 * (r & 1) + x) {                 // known once unrolled
    case 0: return mx::pair_bf16<0>(c, s);
    case 1: return mx::pair_bf16<1>(c, s);
    case 2: return mx::pair_bf16<2>(c, s);
    default: return mx::pair_bf16<3>(c, s);
  }
}

// Rows at and past `valid` (of 16) drop out: their scores to -inf, their V to code 0 at scale 1, so that
// no garbage or NaN meets their zero weight.
template <int D>
__device__ __forceinline__ void mx_mask(int valid, int grp, f32x4_t& st, MxTile<D>& t) {
#pragma unroll
  for (int r = 0; r < 4; r++) {
    if (4 * grp + r >= valid) {
      st[r] = -INFINITY;
      t.ve = (t.ve & ~(0xffu << (8 * r))) | (127u << (8 * r));
      if constexpr (D == 128) t.v[r] = 0u;
      else t.v[r >> 1] &= (r & 1) ? 0x0000ffffu : 0xffff0000u;
    }
  }
}

// Two floats as packed bf16, to the nearest even (one instruction).
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((float2_t{lo, hi}), mx::bf16x2_t));
}

// Which halves of a packed pair a lane takes off as floats: both in the columns of the lo parts (a v_perm
// selector and a mask), none in those of the hi parts.
struct LoPart {
  uint32_t low, high;
};

// A round of two tiles with va and vb valid tokens.  G8: at most 8 query heads, lo by the lane's column.
template <int D, bool G8>
__device__ __forceinline__ void mx_round(MxTile<D> (&t)[2], int va, int vb, const bf16x8_t (&qv)[D / 32], int grp,
                                         float scale_log2, const LoPart& lo, float& m, float& lsum,
                                         f32x4_t (&acc)[D / 16]) {
  f32x4_t sa = mx_scores<D>(t[0], qv), sb = mx_scores<D>(t[1], qv);
  if (va < 16) mx_mask<D>(va, grp, sa, t[0]);               // uniform
  if (vb < 16) mx_mask<D>(vb, grp, sb, t[1]);
  // Scaled and rounded before the bound is taken off (a fused form would leave the product's rounding
  // error in the exponent, which overflows for scores past 2^30).
  float z[8];
#pragma unroll
  for (int i = 0; i < 4; i++) {
#pragma clang fp contract(off)
    z[i] = sa[i] * scale_log2;
    z[4 + i] = sb[i] * scale_log2;
  }
  float mt = fmaxf(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])), fmaxf(fmaxf(z[4], z[5]), fmaxf(z[6], z[7])));
  if (__builtin_amdgcn_ballot_w64(mt > m) != 0) {
    mt = fmaxf(mt, xor_shfl(mt, 16));
    mt = fmaxf(mt, xor_shfl(mt, 32));
    const float m_new = fmaxf(m, mt + kRoomLog2);
    const float alpha = __builtin_amdgcn_exp2f(m - m_new);
    m = m_new;
    lsum *= alpha;
#pragma unroll
    for (int j = 0; j < D / 16; j++) {
      acc[j][0] *= alpha;
      acc[j][1] *= alpha;
      acc[j][2] *= alpha;
      acc[j][3] *= alpha;
    }
  }
  float p[8];
#pragma unroll
  for (int i = 0; i < 8; i++) {
#pragma clang fp contract(off)
    p[i] = __builtin_amdgcn_exp2f(z[i] - m);
  }
  lsum += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
  // the hi parts, and what is left of each p (G8: in the columns of the lo parts; p itself in the others)
  const u32x4_t hi = {pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7])};
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const uint32_t h = hi[i >> 1];
    x[i] = p[i] - __uint_as_float(G8 ? __builtin_amdgcn_perm(0u, h, lo.low) : h << 16);
    x[i + 1] = p[i + 1] - __uint_as_float(h & (G8 ? lo.high : 0xffff0000u));
  }
  const bf16x8_t left = __builtin_bit_cast(
      bf16x8_t, (u32x4_t{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])}));
  const bf16x8_t p0 = G8 ? left : __builtin_bit_cast(bf16x8_t, hi), p1 = left;
#pragma unroll
  for (int x = 0; x < D / 32; x++) {                        // channel pair x of every piece
    uint32_t wa[4], wb[4];
#pragma unroll
    for (int r = 0; r < 4; r++) {
      wa[r] = mx_widen_v<D>(t[0], r, x);
      wb[r] = mx_widen_v<D>(t[1], r, x);
    }
#pragma unroll
    for (int odd = 0; odd < 2; odd++) {
      // channel 2 x + odd: the tokens' halves side by side
      const uint32_t sel = odd ? 0x07060302u : 0x05040100u;
      const u32x4_t w = {__builtin_amdgcn_perm(wa[1], wa[0], sel), __builtin_amdgcn_perm(wa[3], wa[2], sel),
                         __builtin_amdgcn_perm(wb[1], wb[0], sel), __builtin_amdgcn_perm(wb[3], wb[2], sel)};
      const bf16x8_t a = __builtin_bit_cast(bf16x8_t, w);
      f32x4_t& o = acc[2 * x + odd];
      o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p0, o, 0, 0, 0);
      if constexpr (!G8) o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p1, o, 0, 0, 0);
    }
  }
}

// One wave's share of a split, as gqa_wave_slots of decode.hip: the slots lo + w, lo + w + U, .. below
// min(hi_fixed, cnt).
template <int D, bool G8>
__device__ __forceinline__ void mx_wave_slots(const DecodeArgs& a, int i, int h, int lo, int hi_fixed, int w, int U,
                                              int lane, float& m, float& lsum, f32x4_t (&acc)[D / 16], int& cnt_all) {
  const uint8_t* kbase = static_cast<const uint8_t*>(a.k);
  const uint8_t* vbase = static_cast<const uint8_t*>(a.v);
  constexpr int KS = D / 32;
  const int col = lane & 15, grp = lane >> 4;
  const int head = G8 ? (col & 7) : col;
  const LoPart part = G8 && col >= 8 ? LoPart{0x01000c0cu, 0xffff0000u} : LoPart{0x0c0c0c0cu, 0u};
#pragma unroll
  for (int j = 0; j < D / 16; j++) acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  m = kNoMax;
  lsum = 0.f;
  const int32_t* sel = a.sel_pages + ((int64_t)i * a.H + h) * a.max_sel;
  const int cnt_raw = a.sel_count[i];
  const int L = a.seq_lens[i];
  const int base = a.indptr[i];
  const int list_len = a.indptr[i + 1] - base;
  const int slot0 = lo + w + U * lane;
  const int j_first = slot0 < hi_fixed ? sel[slot0] : -1;
  bf16x8_t qv[KS];
  {
    const bool hv = head < a.g;
    const uint16_t* qp = a.q + ((int64_t)i * a.Hq + h * a.g + (hv ? head : 0)) * D + KS * 8 * grp;
#pragma unroll
    for (int kk = 0; kk < KS; kk++) {
      qv[kk] = *reinterpret_cast<const bf16x8_t*>(qp + 8 * kk);
      if (!hv) qv[kk] = bf16x8_t{};
    }
  }
  cnt_all = min(max(cnt_raw, 0), a.max_sel);
  const int cnt = min(cnt_all, hi_fixed);
  const int P = num_pages(L, a.bs, list_len * a.r, INT_MAX);
  const int tsh = __builtin_ctz((unsigned)a.bs) - 4;       // log2 of the tiles per slot
  const int64_t slice_bytes = mx::slice_bytes(a.ps, D);
  const MxLane ln = mx_lane<D>(col, grp);

  for (int w0 = 0; lo + w + U * w0 < cnt; w0 += kWave) {
    const int slot = slot0 + U * w0;
    const int j = w0 == 0 ? j_first : (slot < hi_fixed ? sel[slot] : -1);
    // lane: slice of its slot's block, and (first tile of the block in the page) << 16 | valid tokens
    // (0: an id outside the request, whose tiles weigh nothing)
    int64_t my_s = 0;
    int my_n = 0;
    if (slot < cnt && j >= 0 && j < P) {
      const int jp = j / a.r, blk = j - jp * a.r;
      my_s = (clamp_page(a.indices[base + jp], a.num_phys) * a.H + h) * slice_bytes;
      my_n = min(a.bs, L - j * a.bs) | ((blk << tsh) << 16);
    }
    const int tiles = min(kWave, (cnt - lo - w - U * w0 + U - 1) / U) << tsh;
    // Tile u of the window into t, the last one again past the end.
    auto load = [&](int u, MxTile<D>& t) {
      u = min(u, tiles - 1);
      const int ls = u >> tsh, tt = u - (ls << tsh);
      const uint32_t s_lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)my_s, ls);
      const uint32_t s_hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)my_s >> 32), ls);
      const int t0 = 16 * ((__builtin_amdgcn_readlane(my_n, ls) >> 16) + tt);
      mx_load<D>(kbase, vbase, (int64_t)(((uint64_t)s_hi << 32) | s_lo), (int)slice_bytes, t0, a.ps, ln, t);
    };
    auto valid = [&](int u) {
      if (u >= tiles) return 0;
      const int ls = u >> tsh, tt = u - (ls << tsh);
      return min(16, (__builtin_amdgcn_readlane(my_n, ls) & 0xffff) - 16 * tt);
    };
    // Two rounds' tiles in registers: one loads while the other computes.  The loads are unconditional
    // (past the end the last tile once more, a cache hit), so that no branch makes the compiler wait
    // for all of them.
    MxTile<D> t[2], n[2];
    load(0, t[0]);
    load(1, t[1]);
    for (int u = 0;; u += 4) {
      load(u + 2, n[0]);
      load(u + 3, n[1]);
      mx_round<D, G8>(t, valid(u), valid(u + 1), qv, grp, a.scale_log2, part, m, lsum, acc);
      if (u + 2 >= tiles) break;
      load(u + 4, t[0]);
      load(u + 5, t[1]);
      mx_round<D, G8>(n, valid(u + 2), valid(u + 3), qv, grp, a.scale_log2, part, m, lsum, acc);
      if (u + 4 >= tiles) break;
    }
  }
}

__device__ __forceinline__ void put_merged(uint16_t* dst, float W, const float4& o) {
  const float inv = W == 0.f ? 0.f : 1.f / W;
  *reinterpret_cast<uint2*>(dst) = make_uint2(f32_to_bf16_rne(o.x * inv) | (f32_to_bf16_rne(o.y * inv) << 16),
                                              f32_to_bf16_rne(o.z * inv) | (f32_to_bf16_rne(o.w * inv) << 16));
}

// A partial's running bound (no score is above it) and sum.  Their log-sum-exp in one float would round at
// the bound's magnitude: at scores of 2^24 a split's weight would be off by half.
typedef unsigned int u32x2v_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void put_state(__amdgpu_buffer_rsrc_t r, uint32_t row, float m, float l) {
  __builtin_amdgcn_raw_buffer_store_b64((u32x2v_t{__float_as_uint(m), __float_as_uint(l)}), r, (int)(row * 8u), 0,
                                        kAgentCoherent);
}
__device__ __forceinline__ float2_t get_state(__amdgpu_buffer_rsrc_t r, uint32_t row) {
  const u32x2v_t w = __builtin_amdgcn_raw_buffer_load_b64(r, (int)(row * 8u), 0, kAgentCoherent);
  return float2_t{__uint_as_float(w.x), __uint_as_float(w.y)};
}

// Merge of a split pair's S partials by the workgroup, each weighing its sum.  A slot is 4 channels of one head;
// with fewer slots than threads, G threads share one and take every G-th partial, kMergeBatch loads in
// flight each, and meet in LDS ([G][slots] of 6 floats): a pair cut into many splits (few requests)
// is merged in one or two round trips.
template <int D, int NT>
__device__ __forceinline__ void merge_pair(int S, int g, __amdgpu_buffer_rsrc_t o_rs, __amdgpu_buffer_rsrc_t l_rs,
                                           float* lds, uint16_t* out) {
  const int slots = g * D / 4;
  const int G = max(1, min(NT / slots, S));
  for (int y = (int)threadIdx.x; y < slots * G; y += NT) {   // one turn, unless there are more slots than threads
    const int k = y / slots, x = y - k * slots;
    const int c = (4 * x) / D, d = 4 * x - c * D;
    float M = kNoMax, W = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = k; s0 < S; s0 += G * kMergeBatch) {
      float2_t l[kMergeBatch];
      float4 p[kMergeBatch];
#pragma unroll
      for (int b = 0; b < kMergeBatch; b++) {
        const uint32_t row = (uint32_t)(min(s0 + G * b, S - 1) * g + c);
        l[b] = get_state(l_rs, row);
        p[b] = coherent_load4(o_rs, (row * D + d) * 4u);
      }
      float m_new = M;
#pragma unroll
      for (int b = 0; b < kMergeBatch; b++) {
        if (s0 + G * b >= S) l[b] = float2_t{kNoMax, 0.f};
        m_new = fmaxf(m_new, l[b][0]);
      }
      const float keep = __builtin_amdgcn_exp2f(M - m_new);
      W *= keep;
      o.x *= keep;
      o.y *= keep;
      o.z *= keep;
      o.w *= keep;
#pragma unroll
      for (int b = 0; b < kMergeBatch; b++) {
        const float wgt = __builtin_amdgcn_exp2f(l[b][0] - m_new) * l[b][1];
        W += wgt;
        o.x += wgt * p[b].x;
        o.y += wgt * p[b].y;
        o.z += wgt * p[b].z;
        o.w += wgt * p[b].w;
      }
      M = m_new;
    }
    if (G > 1) {
      float* q = lds + (size_t)y * 6;
      q[0] = M;
      q[1] = W;
      q[2] = o.x;
      q[3] = o.y;
      q[4] = o.z;
      q[5] = o.w;
    } else {
      put_merged(out + c * D + d, W, o);
    }
  }
  if (G == 1) return;                                        // uniform
  __syncthreads();
  if ((int)threadIdx.x >= slots) return;
  const int x = (int)threadIdx.x, c = (4 * x) / D, d = 4 * x - c * D;
  float M = kNoMax, W = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k = 0; k < G; k++) M = fmaxf(M, lds[(size_t)(k * slots + x) * 6]);
  for (int k = 0; k < G; k++) {
    const float* q = lds + (size_t)(k * slots + x) * 6;
    const float wgt = __builtin_amdgcn_exp2f(q[0] - M);
    W += wgt * q[1];
    o.x += wgt * q[2];
    o.y += wgt * q[3];
    o.z += wgt * q[4];
    o.w += wgt * q[5];
  }
  put_merged(out + c * D + d, W, o);
}

template <int D, bool G8, bool BAL>
__global__ __launch_bounds__(kMxWaves * kWave) __attribute__((amdgpu_waves_per_eu(3))) void decode_mx_kernel(
    const DecodeArgs a) {
  constexpr int DPL = D / 16, NW = kMxWaves;
  extern __shared__ __attribute__((aligned(16))) float mx_lds[];
  load_args(a);
  const int lane = lane_id(), wv = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int col = lane & 15, grp = lane >> 4;
  __shared__ int last;
  const int pairs = (int)gridDim.x / a.S;
  const int split = (int)blockIdx.x / pairs;
  int ui = ((int)blockIdx.x - split * pairs) / a.H;
  const int uh = (int)blockIdx.x - split * pairs - ui * a.H;
  if constexpr (BAL) ui = balanced_request(a, ui, pairs / a.H);
  const int T = a.T, pair = ui * a.H + uh, lo = split * T;

  f32x4_t acc[DPL];
  float m, lsum;
  int cnt;
  mx_wave_slots<D, G8>(a, ui, uh, lo, min(lo + T, a.max_sel), wv, NW, lane, m, lsum, acc, cnt);
  const int Sp = splits_of(cnt, T);                        // uniform: every wave loaded the count
  if (split >= Sp) return;
  float lt = lsum + xor_shfl(lsum, 16);
  lt += xor_shfl(lt, 32);
  if constexpr (G8) {                                      // hi and lo parts' columns, 8 lanes apart
#pragma unroll
    for (int j = 0; j < DPL; j++) {
#pragma unroll
      for (int r = 0; r < 4; r++) acc[j][r] += dpp_f32<0x128>(acc[j][r]);
    }
  }

  // the waves' states meet in LDS
  const int g = a.g;
  float* obuf = mx_lds;                                    // [wave][g][D]
  float* mbuf = obuf + NW * g * D;                         // [wave][g]
  float* lbuf = mbuf + NW * g;                             // [wave][g]
  if (col < g) {
    // lane (grp, col) holds channels (4*grp + r)*DPL + j of query head col
    float* dst = obuf + (wv * g + col) * D + 4 * grp * DPL;
#pragma unroll
    for (int r = 0; r < 4; r++) {
#pragma unroll
      for (int j = 0; j < DPL; j += 4)
        *reinterpret_cast<float4*>(dst + r * DPL + j) = make_float4(acc[j][r], acc[j + 1][r], acc[j + 2][r], acc[j + 3][r]);
    }
    if (grp == 0) {
      mbuf[wv * g + col] = m;
      lbuf[wv * g + col] = lt;
    }
  }
  __syncthreads();
  const uint32_t pair_rows = (uint32_t)(a.S * g);
  const __amdgpu_buffer_rsrc_t o_rs = coherent_rsrc(a.part_o + (int64_t)pair * pair_rows * D, pair_rows * D * 4u);
  const __amdgpu_buffer_rsrc_t l_rs = coherent_rsrc(a.part_lse + (int64_t)pair * pair_rows * 2, pair_rows * 8u);
  for (int x = (int)threadIdx.x; x < g * D / 4; x += NW * kWave) {
    const int c = (4 * x) / D, d = 4 * x - c * D;
    float M = kNoMax;
#pragma unroll
    for (int k = 0; k < NW; k++) M = fmaxf(M, mbuf[k * g + c]);
    float Ls = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < NW; k++) {
      const float wgt = __builtin_amdgcn_exp2f(mbuf[k * g + c] - M);      // a wave without a token has zeros
      const float4 v = *reinterpret_cast<const float4*>(obuf + (k * g + c) * D + d);
      Ls += wgt * lbuf[k * g + c];
      o.x += wgt * v.x;
      o.y += wgt * v.y;
      o.z += wgt * v.z;
      o.w += wgt * v.w;
    }
    const float inv = Ls == 0.f ? 0.f : 1.f / Ls;
    if (Sp == 1) {
      uint16_t* dst = a.out + ((int64_t)ui * a.Hq + uh * g + c) * D + d;
      *reinterpret_cast<uint2*>(dst) = make_uint2(f32_to_bf16_rne(o.x * inv) | (f32_to_bf16_rne(o.y * inv) << 16),
                                                  f32_to_bf16_rne(o.z * inv) | (f32_to_bf16_rne(o.w * inv) << 16));
    } else {
      const uint32_t row = (uint32_t)(split * g + c);
      coherent_store4(o_rs, (row * D + d) * 4u, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
      if (d == 0) put_state(l_rs, row, M, Ls);
    }
  }
  if (Sp > 1) {
    // split pair: the last split to arrive merges, as in decode.hip
    wait_vm_all();
    __syncthreads();
    if (threadIdx.x == 0)
      last = __builtin_amdgcn_atomic_inc32(a.ctr + pair, (uint32_t)(Sp - 1), __ATOMIC_RELAXED, "agent") ==
             (uint32_t)(Sp - 1);
    __syncthreads();
    if (last) merge_pair<D, NW * kWave>(Sp, g, o_rs, l_rs, mx_lds, a.out + ((int64_t)ui * a.Hq + uh * g) * D);
  }
}

template <int D>
void launch(const DecodeArgs& a, unsigned grid, hipStream_t stream) {
  // the waves' states, then merge_pair's
  const size_t lds = sizeof(float) * (size_t)kMxWaves * std::max(a.g * (D + 2), kWave * 6);
  const dim3 block(kMxWaves * kWave);
#define VX_MX(G8, BAL) hipLaunchKernelGGL((decode_mx_kernel<D, G8, BAL>), dim3(grid), block, lds, stream, a)
  if (a.g <= 8) {
    if (a.order_block > 0) VX_MX(true, true);
    else VX_MX(true, false);
  } else {
    if (a.order_block > 0) VX_MX(false, true);
    else VX_MX(false, false);
  }
#undef VX_MX
}

}  // namespace

void launch_decode_mx(const DecodeArgs& a, int D, unsigned grid, hipStream_t stream) {
  if (D == 128) launch<128>(a, grid, stream);
  else launch<64>(a, grid, stream);
}

}  // namespace vx
