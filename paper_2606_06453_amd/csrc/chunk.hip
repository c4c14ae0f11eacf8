// Attention of a chunk's tokens over the paged cache: all of it (vx_chunk_attention), or the blocks listed for
// each token (vx_sparse_chunk_attention).
//
// chunk_narrow_kernel  tiles of 16 query rows (token, head of the group) whose waves share out the tokens;
// chunk_wide_kernel    tiles of 64 or 128 rows whose waves share the rows, and the tokens through LDS;
// chunk_merge_kernel   joins the parts of a list that several workgroups took.
// A tile whose sums are not finite is done again row by row (attend_rows).
#include <algorithm>
#include <climits>

#include "chunk_common.h"
#include "chunk_tile.h"
#include "chunk_wide.h"

namespace vx {
using namespace chunk;
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kTileRows = 16;              // query rows (token, head of the group) of a matrix operand
constexpr int kNarrowTiles = 4;            // most narrow tiles of a request, on average
constexpr int kTargetWgs = 512;            // two workgroups a CU
constexpr int kMaxParts = 64;              // a merging wave's lanes
constexpr int kPartTokens = 512;           // least tokens of a part: four pairs of runs a wave
constexpr int kAtOnce = 4;                 // K operands of a run that are sent for together
constexpr float kLn2 = 0.693147180559945309f;

// The blocks listed for the tile's tokens: masks[id] holds a bit for each token that lists block id, ids the
// listed ones in ascending order; wave_total: kWaves words.  Returns their count.  Every thread of the workgroup takes
// part.
__device__ __forceinline__ int listed_blocks(const ChunkArgs& a, const Tile& t, int h, uint32_t* words, uint16_t* ids,
                                             int* wave_total) {
  const int tid = (int)threadIdx.x, lane = lane_id(), wave = tid >> 6;
  const int p_last = t.p0 + t.n - 1;
  const int nb = p_last < 0 ? 0 : min((min(p_last + 1, t.len) + a.bs - 1) >> a.bs_shift, a.max_blocks);
  for (int x = tid; x < (nb + 1) / 2; x += kThreads) words[x] = 0;
  __syncthreads();
  for (int x = 0; x < t.n; x++) {
    const int p = t.p0 + x, most = p < 0 ? 0 : min((p >> a.bs_shift) + 1, nb);
    const int cnt = min(max(a.sel_count[t.row0 + x], 0), a.max_sel);
    const int32_t* sel = a.sel_pages + ((t.row0 + x) * a.H + h) * a.max_sel;
    for (int s = tid; s < cnt; s += kThreads) {
      const int id = sel[s];
      if (id >= 0 && id < most) atomicOr(&words[id >> 1], 1u << (x + 16 * (id & 1)));
    }
  }
  __syncthreads();
  const uint16_t* masks = reinterpret_cast<const uint16_t*>(words);
  const int per = (nb + kThreads - 1) / kThreads, b0 = min(tid * per, nb), b1 = min(b0 + per, nb);
  int mine = 0;
  for (int b = b0; b < b1; b++) mine += masks[b] != 0;
  int before = mine;                                   // inclusive over the wave
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) {
    const int y = __shfl_up(before, s, kWave);
    if (lane >= s) before += y;
  }
  if (lane == kWave - 1) wave_total[wave] = before;
  __syncthreads();
  int total = 0;
  before -= mine;
#pragma unroll
  for (int w = 0; w < kWaves; w++) {
    if (w < wave) before += wave_total[w];
    total += wave_total[w];
  }
  for (int b = b0; b < b1; b++)
    if (masks[b]) ids[before++] = (uint16_t)b;
  __syncthreads();
  return total;
}

// Part s of [lo, hi), in parts of `per`.
__device__ __forceinline__ void part_of(int lo, int hi, int s, int per, int& plo, int& phi) {
  plo = min(lo + s * per, hi);
  phi = min(plo + per, hi);
}

// 16-token runs of a part: the longest list of the batch cut into a.splits, for every request, so that all parts
// take equally long (four contexts of 24000 to 32768 tokens: cut by their own lengths, the longest's parts end 15%
// after the mean).
__device__ __forceinline__ int part_runs16(const ChunkArgs& a) {
  if (a.splits == 1) return INT_MAX / 2;
  int most = 0;
  for (int i = lane_id(); i < a.batch; i += kWave) most = max(most, a.seq_lens[i]);
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) most = max(most, __shfl_xor(most, s, kWave));
  most = (int)min((int64_t)most, (int64_t)a.max_pages * a.ps);
  if (a.window > 0) most = (int)min((int64_t)most, (int64_t)a.window + a.tokens + 15 + (a.causal ? 0 : most));
  return ((most + 15) / 16 + a.splits) / a.splits;       // a window's ends may lie inside runs
}

// The tile's rows one by one: where a sum of the tile kernels is not finite.
template <int D, int DV, int KT>
__device__ __forceinline__ void attend_rows(const ChunkArgs& a, const Tile& t, int h, const Runs& runs, int split) {
  for (int x = (int)threadIdx.x >> 6; x < t.n * a.g; x += kWaves) {
    RowState<DV> st;
    attend_row<D, DV, KT>(a, t, h, x % a.g, x / a.g, runs, st);
    store_row<DV>(a, t.row0 + x / a.g, h * a.g + x % a.g, split, st);
  }
}

// A part with no token: its rows' sums are zero, and the join leaves it out.
__device__ __forceinline__ bool empty_part(const ChunkArgs& a, const Tile& t, int h, int split, const Runs& runs) {
  if (a.splits == 1 || runs.lo < runs.hi) return false;
  for (int r = (int)threadIdx.x; r < t.n * a.g; r += kThreads)
    a.part_ml[((t.row0 + r / a.g) * a.Hq + h * a.g + r % a.g) * a.splits + split] = make_float2(-INFINITY, 0.f);
  return true;
}

// The runs of a workgroup's part; shift16: log2 of the 16-token runs of an entry.  scratch: kWaves words.
template <bool SPARSE>
__device__ __forceinline__ Runs part_runs(const ChunkArgs& a, const Tile& t, int h, int split, uint32_t* lds, uint32_t* scratch,
                                          int& shift16) {
  Runs runs;
  if constexpr (SPARSE) {
    uint16_t* ids = reinterpret_cast<uint16_t*>(lds + (a.max_blocks + 1) / 2);
    const int all = __builtin_amdgcn_readfirstlane(listed_blocks(a, t, h, lds, ids, reinterpret_cast<int*>(scratch)));
    runs.ids = ids;
    runs.masks = reinterpret_cast<const uint16_t*>(lds);
    runs.shift = a.bs_shift;
    shift16 = a.bs_shift - 4;
    part_of(0, all, split, (all + a.splits - 1) / a.splits, runs.lo, runs.hi);
  } else {
    runs.ids = nullptr;
    runs.masks = nullptr;
    runs.shift = 4;
    shift16 = 0;
    const int lo = first_key(a, t.p0) >> 4, hi = (end_key(a, t, t.p0 + t.n - 1) + 15) >> 4;
    part_of(lo, hi, split, __builtin_amdgcn_readfirstlane(part_runs16(a)), runs.lo, runs.hi);
    if (split == a.splits - 1) runs.hi = hi;             // never less than the whole list
  }
  return runs;
}

// Four waves share a tile of 16 query rows; each takes every fourth pair of 16-token runs of the tile's list,
// straight from the cache into matrix operands, and the waves' states meet in LDS.  For few rows over fp8 or mxfp4 caches,
// which memory bounds: no barrier stands between loads and their use, and codes widen once for 16 rows (drafted tokens of
// 32 users over 64 listed blocks of 32 tokens, E4M3: 57 us, 6.3 TB/s of the 7.05 that a stream reads; in wide tiles 114).
// bf16 rows take wide tiles from the first row: straight to LDS they need no register on their way (4 users' drafted
// tokens 92 us, here 125).
template <int D, int KT, bool SPARSE>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2))) void chunk_narrow_kernel(const ChunkArgs a) {
  constexpr int KS = D / 32, NJ = D / 16, W = D / 32;
  extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
  const int tid = (int)threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, grp = lane >> 4;
  const int h = (int)blockIdx.x % a.H, split = (int)blockIdx.y;
  Tile t;
  if (!find_tile(a, (int)blockIdx.x / a.H, t)) return;
  int shift16;
  const Runs runs = part_runs<SPARSE>(a, t, h, split, lds, lds + 2 * ((a.max_blocks + 1) / 2), shift16);
  if (empty_part(a, t, h, split, runs)) return;
  const int rows = t.n * a.g, last = end_key(a, t, t.p0 + t.n - 1);        // past every row's tokens
  Rows<D, D, 1> w;
  begin_rows<D, D, KT, 1>(a, t, h, 0, col, grp, w);

  const int n16 = (runs.hi - runs.lo) << shift16, pairs = (n16 + 1) >> 1;
  int listed = 0;                                        // tile tokens that list one of the wave's runs
  // 32 pairs of the wave at a time: lane 2 u + e finds run e of its pair u
  for (int w0 = wave; w0 < pairs; w0 += 32 * kWaves) {
    int my_page = 0, my_tok = 0, my_mask = 0, my_n = 0;    // my_n: of its 16 tokens, those that some row may attend
    {
      const int x = 2 * (w0 + (lane >> 1) * kWaves) + (lane & 1), y = min(x, n16 - 1);
      if (y >= 0) {                                      // past the end: the last run again, for no row
        const int e = runs.lo + (y >> shift16);
        int id = e;
        my_mask = 0xffff;
        if constexpr (SPARSE) {
          id = runs.ids[e];
          my_mask = runs.masks[id];
        }
        if (x >= n16) my_mask = 0;
        my_tok = (id << runs.shift) + 16 * (y & ((1 << shift16) - 1));
        my_page = (int)clamp_page(t.pages[my_tok >> a.ps_shift], a.num_phys);
        my_n = min(max(last - my_tok, 0), 16);           // a listed block may end in runs behind the last token
      }
    }
    const int count = min(32, (pairs - w0 + kWaves - 1) / kWaves);
    // One buffer: a pair's K is sent for when the scores have taken the one before, its V when the sums have, so
    // that each travels through half a step and the registers leave room for three waves a SIMD.
    RawK<D, KT> k[2];
    RawV<D, KT> v[2];
    auto fetch_k = [&](int u) {
#pragma unroll
      for (int e = 0; e < 2; e++) {
        const int page = __builtin_amdgcn_readlane(my_page, 2 * u + e), tok = __builtin_amdgcn_readlane(my_tok, 2 * u + e);
        load_k<D, KT>(a, slice_of<D, KT>(a, a.k, page, h), tok & (a.ps - 1), __builtin_amdgcn_readlane(my_n, 2 * u + e), col, grp, k[e]);
      }
    };
    auto fetch_v = [&](int u) {
#pragma unroll
      for (int e = 0; e < 2; e++) {
        const int page = __builtin_amdgcn_readlane(my_page, 2 * u + e), tok = __builtin_amdgcn_readlane(my_tok, 2 * u + e);
        load_v<D, KT>(a, slice_of<D, KT>(a, a.v, page, h), tok & (a.ps - 1), __builtin_amdgcn_readlane(my_n, 2 * u + e), col, grp, v[e]);
      }
    };
    fetch_k(0);
    fetch_v(0);
    for (int u = 0; u < count; u++) {
      const int tok0 = __builtin_amdgcn_readlane(my_tok, 2 * u), tok1 = __builtin_amdgcn_readlane(my_tok, 2 * u + 1);
      const int mask0 = __builtin_amdgcn_readlane(my_mask, 2 * u), mask1 = __builtin_amdgcn_readlane(my_mask, 2 * u + 1);
      if constexpr (SPARSE) listed |= mask0 | mask1;
      const bool inner = min(tok0, tok1) >= w.all_from && max(tok0, tok1) + 16 <= w.all_to;
      const int next = min(u + 1, count - 1);
      f32x4_t s[1][2];
#pragma unroll
      for (int e = 0; e < 2; e++) {
        s[0][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < KS; kk++)
          s[0][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k_operand<D, KT>(k[e], kk), w.q[0][kk], s[0][e], 0, 0, 0);
      }
      fetch_k(next);
      if (!inner) mask_scores<D, D, 1>(s, tok0, tok1, grp, w);
      uint32_t p[1][2][4];
      softmax_step<D, D, 1, true>(a.scale_log2, s, mask0, mask1, w, p);
      uint32_t v0[4][W], v1[4][W];
      v_rows<D, KT>(v[0], v0);
      v_rows<D, KT>(v[1], v1);
#pragma unroll
      for (int j = 0; j < NJ; j++)
#pragma unroll
        for (int e = 0; e < 2; e++)
          w.acc[0][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v_operand<W>(v0, v1, j), p_operand(p[0][e]), w.acc[0][j], 0, 0, 0);
      fetch_v(next);
    }
  }

  // the waves' states meet: weighted means, references and sums
  constexpr int kRow = D + 4;                            // a row's floats in LDS
  float* obuf = reinterpret_cast<float*>(lds);           // the lists have been read
  float2* mbuf = reinterpret_cast<float2*>(obuf + kWaves * 16 * kRow);
  constexpr int CPT = 16 * D / kThreads;                 // channels of a thread
  const int orow = tid / (D / CPT), oc = (tid % (D / CPT)) * CPT;
  __syncthreads();
  const float sum = column_sum(w.l[0]);
  if (grp == 0) mbuf[wave * 16 + col] = make_float2(SPARSE && !(listed >> w.bit[0] & 1) ? -INFINITY : w.m[0], sum);
#pragma unroll
  for (int i = 0; i < 4; i++)
#pragma unroll
    for (int j = 0; j < NJ; j += 4)
      *reinterpret_cast<float4*>(obuf + (wave * 16 + col) * kRow + (4 * grp + i) * NJ + j) =
          make_float4(w.acc[0][j][i], w.acc[0][j + 1][i], w.acc[0][j + 2][i], w.acc[0][j + 3][i]);
  __syncthreads();
  float2 ml[kWaves];
  float top = kNoScore;
#pragma unroll
  for (int x = 0; x < kWaves; x++) {
    ml[x] = mbuf[x * 16 + orow];
    top = fmaxf(top, ml[x].x);
  }
  float total = 0.f, o[CPT];
#pragma unroll
  for (int c = 0; c < CPT; c++) o[c] = 0.f;
#pragma unroll
  for (int x = 0; x < kWaves; x++) {
    const float f = __builtin_amdgcn_exp2f(ml[x].x - top);
    total = fmaf(ml[x].y, f, total);
#pragma unroll
    for (int c = 0; c < CPT; c++) o[c] = fmaf(obuf[(x * 16 + orow) * kRow + oc + c], f, o[c]);
  }
  const float inv = total > 0.f ? 1.f / total : 0.f;
  bool fine = fabsf(total) < INFINITY;
  if (total == 0.f) {                                    // a row that attends tokens and has no weight: every score is -inf
    bool some = false;
    if constexpr (SPARSE) {
#pragma unroll
      for (int x = 0; x < kWaves; x++) some = some || ml[x].x > -INFINITY;
    } else if (orow < rows) {
      const int p = t.p0 + orow / a.g;
      some = max(first_key(a, p), runs.lo << 4) < min(end_key(a, t, p), min(runs.hi, INT_MAX >> 4) << 4);
    }
    fine = !some;
  }
#pragma unroll
  for (int c = 0; c < CPT; c++) {
    fine = fine && fabsf(o[c]) < INFINITY;
    o[c] *= inv;
  }
  if (orow < rows) {
    const int64_t at = (t.row0 + orow / a.g) * a.Hq + h * a.g + orow % a.g;
    if (a.splits > 1) {
      float* dst = a.part_o + (at * a.splits + split) * D + oc;
#pragma unroll
      for (int c = 0; c < CPT; c += 4) *reinterpret_cast<float4*>(dst + c) = make_float4(o[c], o[c + 1], o[c + 2], o[c + 3]);
      if (oc == 0) a.part_ml[at * a.splits + split] = make_float2(total > 0.f ? top : -INFINITY, total);
    } else {
#pragma unroll
      for (int c = 0; c < CPT; c += 4)
        *reinterpret_cast<uint2*>(a.out + at * D + oc + c) =
            make_uint2(pack_bf16(o[c] * a.v_scale, o[c + 1] * a.v_scale), pack_bf16(o[c + 2] * a.v_scale, o[c + 3] * a.v_scale));
      if (oc == 0 && a.lse) a.lse[at] = total > 0.f ? (top + log2f(total)) * kLn2 : -INFINITY;
    }
  }
  if (__syncthreads_or(orow < rows && !fine)) {
    if constexpr (SPARSE) listed_blocks(a, t, h, lds, const_cast<uint16_t*>(runs.ids), reinterpret_cast<int*>(lds + 2 * ((a.max_blocks + 1) / 2)));
    attend_rows<D, D, KT>(a, t, h, runs, split);
  }
}

// Tokens of a buffer.  Listed blocks are short runs in any place, which take longest to arrive: half the tokens let
// twice the workgroups wait side by side (4096 tokens over 128 blocks each 790 us, with 64 880).  Lists of everything
// want 64 (prompts: bf16 4380, with 32 and two waves a SIMD 4590, with 32 and three 4470; mxfp4 1000 and 1228).  The
// latent's rows are 4.5 times longer, and two workgroups of 72 KB share a CU.
template <int D, int DV, int KT, bool SPARSE>
constexpr int kTokens = SPARSE || D != DV ? 32 : 64;

// Four waves of 16 RT rows each share the tokens of their tile through LDS (chunk_wide.h).  A wave passes over
// runs that none of its rows attends.  Two operands of rows a wave halve the reads of LDS a product; one serves tiles of
// up to 64 rows, listed blocks (16 tokens a mask) and the latent, whose 512 output channels fill the registers.
//   a prompt's last 8192 of 32768 tokens, 32 heads over 8, bf16: 4420 us, 1300 TFLOP/s with the weights' second part
//     counted (a library product of 16384^3 1356); matrix instructions 61% and vector ones up to 55% of the cycles, at 1.9
//     to 2 GHz.  With weights in one part 3200 us at the same rate
//   prompts and drafts of 48 requests, mxfp4: 1000 us; 45% and up to 51%, and the widened rows' way to LDS
//   prompts under a window of 1000 tokens, 64 channels, E4M3: 118 us; 37% and 75%: the softmax, which D does not shorten
//   the latent, eight prompts' chunks: 348 us with the join; 51% and 24%, LDS 35%
//   4096 tokens over 128 listed blocks of 16 each: 790 us; 38% and 52%.  A wave's four tokens list 2.3 times the blocks
//     of one, and pairs of runs in the order of blocks make that 3.3
template <int D, int DV, int KT, int RT, bool SPARSE>
__device__ __forceinline__ void wide_tile(const ChunkArgs& a, const Tile& t, int h, int split, uint32_t* lds) {
  constexpr int TK = kTokens<D, DV, KT, SPARSE>;
  using G = Wide<D, DV, KT, TK>;
  constexpr int KS = D / 32, NJ = DV / 16;
  const int tid = (int)threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, grp = lane >> 4;
  uint8_t* bufs = reinterpret_cast<uint8_t*>(lds);
  uint32_t* lists = lds + 2 * G::BUF / sizeof(uint32_t);
  int shift16;
  const Runs runs = part_runs<SPARSE>(a, t, h, split, lists, lds, shift16);
  if (empty_part(a, t, h, split, runs)) return;
  const int rows = t.n * a.g, last = end_key(a, t, t.p0 + t.n - 1);
  const int r0 = wave * 16 * RT;
  Rows<D, DV, RT> w;
  begin_rows<D, DV, kKvBf16, RT>(a, t, h, r0, col, grp, w);
  // the tile tokens of this wave's rows, and what they attend between them
  const int x0 = min(r0 / a.g, t.n), x1 = min((r0 + 16 * RT - 1) / a.g, t.n - 1);
  const int wave_from = first_key(a, t.p0 + x0);
  int wave_to = r0 < rows ? end_key(a, t, t.p0 + x1) : 0;
  if constexpr (!SPARSE) {                               // what lies behind the part is for the others
    const int end = min(runs.hi, INT_MAX >> 4) << 4;
    wave_to = min(wave_to, end);
    w.all_to = min(w.all_to, end);
#pragma unroll
    for (int rt = 0; rt < RT; rt++) w.to[rt] = min(w.to[rt], end);
  }
  const int wave_mask = SPARSE && r0 < rows ? (2 << x1) - (1 << x0) : 0;

  const int n16 = (runs.hi - runs.lo) << shift16, steps = (n16 + G::UNITS - 1) / G::UNITS;
  // The runs that a lane looks up for all (listed blocks), or for its wave (a range): first token, page, and the tile
  // tokens that list it.  Listed: lane u holds run 64 w + u, the next 64 are on their way meanwhile.  A range: lane u
  // holds the run that this wave loads in step 64 w + u.
  struct Found {
    int tok, page, mask;
  };
  const int unit = wave / G::WPU;
  auto look_up = [&](int w) {
    Found f{0, 0, 0};
    const int x = SPARSE ? 64 * w + lane : G::UNITS * (64 * w + lane) + unit, y = min(x, n16 - 1);
    if (y >= 0) {                                        // past the end: the last run again, for no row
      const int e = runs.lo + (y >> shift16);
      int id = e;
      if constexpr (SPARSE) {
        id = runs.ids[e];
        f.mask = x < n16 ? runs.masks[id] : 0;
      }
      f.tok = (id << runs.shift) + 16 * (y & ((1 << shift16) - 1));
      f.page = (int)clamp_page(t.pages[f.tok >> a.ps_shift], a.num_phys);
    }
    return f;
  };
  Found now = look_up(0), after = now;
  if constexpr (SPARSE) after = look_up(1);
  Travel<D, DV, KT, TK> travel;
  // runs of the step that is on its way: first tokens and masks
  int toks[G::UNITS], masks[G::UNITS], mine = 0;
  auto send = [&](int s) {
    int page;
    if constexpr (SPARSE) {
      const int at = G::UNITS * s & 63;
      if (at == 0 && s > 0) {
        now = after;
        after = look_up(G::UNITS * s / 64 + 1);
      }
#pragma unroll
      for (int u = 0; u < G::UNITS; u++) {
        toks[u] = __builtin_amdgcn_readlane(now.tok, at + u);
        masks[u] = __builtin_amdgcn_readlane(now.mask, at + u);
      }
      page = __builtin_amdgcn_readlane(now.page, at + unit);
      mine = __builtin_amdgcn_readlane(now.tok, at + unit);
    } else {
      if ((s & 63) == 0 && s > 0) now = look_up(s / 64);
      page = __builtin_amdgcn_readlane(now.page, s & 63);
      mine = __builtin_amdgcn_readlane(now.tok, s & 63);
    }
    const uint8_t* ks = slice_of<D, KT>(a, a.k, page, h);
    send_run<D, DV, KT, TK>(a, ks, G::kAlias ? ks : slice_of<D, KT>(a, a.v, page, h), mine & (a.ps - 1),
                            SPARSE ? max(last - mine, 0) : last - mine, wave, lane, bufs + (s & 1) * G::BUF, travel);
  };
  int listed = 0;                                        // tile tokens that list a run of the part
  if (steps > 0) send(0);
  for (int s = 0; s < steps; s++) {
    uint8_t* buf = bufs + (s & 1) * G::BUF;
    land_run<D, DV, KT, TK>(wave, lane, last - mine, buf, travel);
    lds_barrier();                                       // every wave's part is there, and the other buffer is free
    int tok[G::UNITS], mask[G::UNITS];
#pragma unroll
    for (int u = 0; u < G::UNITS; u++) {
      tok[u] = SPARSE ? toks[u] : (runs.lo + G::UNITS * s + u) << 4;
      mask[u] = SPARSE ? masks[u] : 0xffff;
    }
    if (s + 1 < steps) send(s + 1);
    const uint8_t* vt = G::kAlias ? buf : buf + G::TILE;
#pragma unroll
    for (int y = 0; y < G::UNITS; y += 2) {
      const int tok0 = tok[y], tok1 = tok[y + 1], mask0 = mask[y], mask1 = mask[y + 1];
      if constexpr (SPARSE) listed |= mask0 | mask1;
      const bool some = SPARSE ? ((mask0 | mask1) & wave_mask) != 0 : tok0 < wave_to && tok0 + 32 > wave_from;
      if (some) {
        // of a list the last blocks alone may reach past a row's own token
        const bool inner = SPARSE ? max(tok0, tok1) + 16 <= w.all_to : tok0 >= w.all_from && tok0 + 32 <= w.all_to;
        f32x4_t sc[RT][2];
#pragma unroll
        for (int rt = 0; rt < RT; rt++) sc[rt][0] = sc[rt][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k0 = 0; k0 < KS; k0 += kAtOnce) {       // a few operands at a time, sent for together
          bf16x8_t k[kAtOnce][2];
#pragma unroll
          for (int kk = 0; kk < kAtOnce; kk++)
#pragma unroll
            for (int e = 0; e < 2; e++)
              if (k0 + kk < KS) k[kk][e] = k_from_lds<G::PLANE>(buf, 16 * (y + e), k0 + kk, col, grp);
#pragma unroll
          for (int kk = 0; kk < kAtOnce; kk++)
#pragma unroll
            for (int e = 0; e < 2; e++)
#pragma unroll
              for (int rt = 0; rt < RT; rt++)
                if (k0 + kk < KS)
                  sc[rt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[kk][e], w.q[rt][k0 + kk], sc[rt][e], 0, 0, 0);
        }
        if (!inner) mask_scores<D, DV, RT>(sc, tok0, tok1, grp, w);
        uint32_t p[RT][2][4];
        softmax_step<D, DV, RT, SPARSE>(a.scale_log2, sc, mask0, mask1, w, p);
        // bf16: the waves that add values go first, the others meanwhile weigh theirs (prompt 4500 -> 4470 us, listed
        // blocks 796 -> 785, the latent 346 -> 351; mxfp4, whose waves also widen, 1000 -> 1046 us with it)
        if constexpr (KT == kKvBf16) __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int j = 0; j < NJ; j += 2) {                // two channels' operands: a weight's parts add to one sum in turn
          if (KT == kKvBf16 && j == NJ - 2) __builtin_amdgcn_s_setprio(0);
          const bf16x8_t v[2] = {v_from_lds<G::PLANE>(vt, 16 * y, j, col, grp), v_from_lds<G::PLANE>(vt, 16 * y, j + 1, col, grp)};
#pragma unroll
          for (int e = 0; e < 2; e++)
#pragma unroll
            for (int rt = 0; rt < RT; rt++)
#pragma unroll
              for (int x = 0; x < 2; x++)
                w.acc[rt][j + x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[x], p_operand(p[rt][e]), w.acc[rt][j + x], 0, 0, 0);
        }
      }
    }
  }

  bool bad = false;
#pragma unroll
  for (int rt = 0; rt < RT; rt++) {
    const float total = column_sum(w.l[rt]);
    const float inv = total > 0.f ? 1.f / total : 0.f;
    const int r = r0 + 16 * rt + col;
    const bool there = r < rows;
    const int64_t at = (t.row0 + (there ? r / a.g : 0)) * a.Hq + h * a.g + (there ? r % a.g : 0);
    // a row that attends tokens and has no weight: every score is -inf
    const bool some = SPARSE ? (listed >> w.bit[rt] & 1) != 0 : max(w.from[rt], runs.lo << 4) < w.to[rt];
    bool fine = fabsf(total) < INFINITY && !(total == 0.f && some);
#pragma unroll
    for (int j = 0; j < NJ; j++) {
      float o[4];
#pragma unroll
      for (int i = 0; i < 4; i++) {
        fine = fine && fabsf(w.acc[rt][j][i]) < INFINITY;
        o[i] = w.acc[rt][j][i] * inv;
      }
      if (!there) continue;
      if (a.splits > 1)
        *reinterpret_cast<float4*>(a.part_o + (at * a.splits + split) * DV + 16 * j + 4 * grp) = make_float4(o[0], o[1], o[2], o[3]);
      else
        *reinterpret_cast<uint2*>(a.out + at * DV + 16 * j + 4 * grp) =
            make_uint2(pack_bf16(o[0] * a.v_scale, o[1] * a.v_scale), pack_bf16(o[2] * a.v_scale, o[3] * a.v_scale));
    }
    if (there && grp == 0) {
      if (a.splits > 1) a.part_ml[at * a.splits + split] = make_float2(total > 0.f ? w.m[rt] : -INFINITY, total);
      else if (a.lse) a.lse[at] = total > 0.f ? (w.m[rt] + log2f(total)) * kLn2 : -INFINITY;
    }
    bad = bad || (there && !fine);
  }
  if (__syncthreads_or(bad)) attend_rows<D, DV, KT>(a, t, h, runs, split);
}

// The latent's rows just fit two waves a SIMD, with some words in scratch (15, as fp8 50); one wave takes longer (44
// requests' drafted tokens 280 and 399 us, 440 and 432 with one).
template <int D, int DV, int KT, int RT, bool SPARSE>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2))) void chunk_wide_kernel(const ChunkArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
  const int h = (int)blockIdx.x % a.H, split = (int)blockIdx.y;
  Tile t;
  if (!find_tile(a, (int)blockIdx.x / a.H, t)) return;
  if constexpr (RT > 1) {
    if (t.n * a.g <= 4 * kTileRows) {                    // a short request among long ones
      wide_tile<D, DV, KT, 1, SPARSE>(a, t, h, split, lds);
      return;
    }
  }
  wide_tile<D, DV, KT, RT, SPARSE>(a, t, h, split, lds);
}

// Joins the parts of every row, a wave a row and a token a workgroup (a.tokens is 1): each part's weight is its
// sum at the row's largest reference.  Memory bounds it: 16 heads of 1241 tokens in two parts of 512 channels 23 us
// (4.5 TB/s), 16 parts of drafted tokens 6 us.
template <int DV>
__global__ __launch_bounds__(kThreads) void chunk_merge_kernel(const ChunkArgs a) {
  constexpr int N = DV / kWave, kBatch = 8;              // channels of a lane; parts on their way at a time
  const int lane = lane_id(), h = (int)blockIdx.x % a.H, S = a.splits;
  Tile t;
  if (!find_tile(a, (int)blockIdx.x / a.H, t)) return;
  for (int x = (int)threadIdx.x >> 6; x < a.g; x += kWaves) {
    const int64_t at = t.row0 * a.Hq + h * a.g + x;
    const float2 ml = lane < S ? a.part_ml[at * S + lane] : make_float2(-INFINITY, 0.f);
    float top = ml.y != 0.f ? ml.x : -INFINITY;
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) top = fmaxf(top, xor_shfl(top, s));
    float w = ml.y == 0.f ? 0.f : ml.y * __builtin_amdgcn_exp2f(ml.x - top);   // NaN stays NaN
    float total = w;
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) total += xor_shfl(total, s);
    w = total != 0.f ? w / total : 0.f;
    const bool bare = total == 0.f && __any(ml.x > -INFINITY);           // tokens, and no weight
    float o[N];
#pragma unroll
    for (int c = 0; c < N; c++) o[c] = bare ? NAN : 0.f;
    const float* src = a.part_o + at * S * DV + N * lane;
    for (int s0 = 0; s0 < S; s0 += kBatch) {
      float v[kBatch][N];
#pragma unroll
      for (int y = 0; y < kBatch; y++) {
        const float* p = src + (int64_t)min(s0 + y, S - 1) * DV;
        if constexpr (N == 1) {
          v[y][0] = p[0];
        } else if constexpr (N == 2) {
          const float2 u = *reinterpret_cast<const float2*>(p);
          v[y][0] = u.x;
          v[y][1] = u.y;
        } else {
#pragma unroll
          for (int c = 0; c < N; c += 4) {
            const float4 u = *reinterpret_cast<const float4*>(p + c);
            v[y][c] = u.x;
            v[y][c + 1] = u.y;
            v[y][c + 2] = u.z;
            v[y][c + 3] = u.w;
          }
        }
      }
#pragma unroll
      for (int y = 0; y < kBatch; y++) {
        const float f = s0 + y < S ? __shfl(w, min(s0 + y, S - 1), kWave) : 0.f;
        if (f != 0.f)                                    // a part with no token is not written
#pragma unroll
          for (int c = 0; c < N; c++) o[c] = fmaf(v[y][c], f, o[c]);
      }
    }
    uint16_t* dst = a.out + at * DV + N * lane;
#pragma unroll
    for (int c = 0; c < N; c++) dst[c] = (uint16_t)f32_to_bf16_rne(o[c] * a.v_scale);
    if (lane == 0 && a.lse) a.lse[at] = total > 0.f ? (top + log2f(total)) * kLn2 : total == 0.f ? -INFINITY : total;
  }
}

// Rows of a wave's operand, tokens of a tile and parts of its list.
struct Plan {
  int operands;                            // of 16 rows a wave (wide), 0: narrow
  int tokens, splits;
  size_t o_bytes, bytes;
};
int tile_tokens(int operands, int group, bool sparse) {
  const int rows = operands == 0 ? kTileRows : 4 * kTileRows * operands;
  return std::max(1, sparse ? std::min(16, rows / group) : rows / group);
}
int64_t most_parts(const Geometry& g, int tokens, bool sparse, int max_sel) {
  const int64_t list = std::min<int64_t>((int64_t)g.max_pages * g.bs, sparse ? (int64_t)max_sel * tokens * g.bs : INT64_MAX);
  return std::min<int64_t>(kMaxParts, (list + kPartTokens - 1) / kPartTokens);
}
size_t part_bytes(const Geometry& g) { return g.Dv * sizeof(float) + sizeof(float2); }
constexpr int kHalvesFrom = kTargetWgs / 2, kHalvesTo = kTargetWgs * 3 / 4;        // tiles of the latent: see plan_of
Plan plan_of(const Geometry& g, int n, int Hq, bool sparse, int max_sel) {
  Plan p{};
  const int group = Hq / g.H;
  const bool latent = g.Dqk != g.Dv;
  const int64_t batch = std::max(g.batch, 1);
  if (!latent && g.kv_dtype != kKvBf16 && (int64_t)n <= batch * kNarrowTiles * (kTileRows / group)) p.operands = 0;
  else p.operands = sparse || latent || (int64_t)n * group <= batch * 4 * kTileRows ? 1 : 2;
  p.tokens = tile_tokens(p.operands, group, sparse);
  const int64_t tiles = std::max<int64_t>(batch, (n + p.tokens - 1) / p.tokens) * g.H;
  const int64_t most = most_parts(g, p.tokens, sparse, max_sel);
  // A little more than one tile of the latent a CU: as halves, which are cut from the longest list and so spare the short
  // ones, the long lists end earlier.  40 batches of 260 to 384 tiles with contexts of 0-2048 to 16000-30000 tokens take
  // 0.62 to 1.10 times as long as wholes, 0.83 on average (8 requests of 2048-8192: 350 and 493 us), 8 batches of equal
  // contexts 1.07 to 1.33 times; how even a batch is the host does not know.  Where memory bounds, as for drafted tokens,
  // halves cost more than they bring (58 -> 70 us).
  const bool halves = latent && tiles > kHalvesFrom && tiles <= kHalvesTo;
  p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(most, halves ? 2 : kTargetWgs / tiles));
  if (p.splits > 1) {
    p.o_bytes = (size_t)n * Hq * p.splits * g.Dv * sizeof(float);
    p.bytes = (size_t)n * Hq * p.splits * part_bytes(g);
  }
  p.bytes = std::max<size_t>(p.bytes, 16);
  return p;
}

template <int D, int KT, bool SPARSE>
void launch_narrow(const ChunkArgs& a, dim3 grid, size_t lists, hipStream_t stream) {
  const size_t states = sizeof(float) * kWaves * 16 * (D + 4) + sizeof(float2) * kWaves * 16;
  hipLaunchKernelGGL((chunk_narrow_kernel<D, KT, SPARSE>), grid, dim3(kThreads), std::max(lists + kWaves * sizeof(int), states), stream, a);
}
template <int D, int DV, int KT, int RT, bool SPARSE>
void launch_wide(const ChunkArgs& a, dim3 grid, size_t lists, hipStream_t stream) {
  const size_t lds = 2 * (size_t)Wide<D, DV, KT, kTokens<D, DV, KT, SPARSE>>::BUF + lists;
  hipLaunchKernelGGL((chunk_wide_kernel<D, DV, KT, RT, SPARSE>), grid, dim3(kThreads), lds, stream, a);
}

template <int D, int DV, int KT>
void launch_tiles(const ChunkArgs& a, int operands, dim3 grid, hipStream_t stream) {
  if constexpr (D == DV) {
    const size_t lists = a.sel_pages ? 2 * sizeof(uint32_t) * ((a.max_blocks + 1) / 2) : 0;    // at most 64 KiB
    if constexpr (KT != kKvBf16) {
      if (operands == 0) {
        if (a.sel_pages) launch_narrow<D, KT, true>(a, grid, lists, stream);
        else launch_narrow<D, KT, false>(a, grid, 0, stream);
        return;
      }
    }
    if (a.sel_pages) {
      launch_wide<D, DV, KT, 1, true>(a, grid, lists, stream);
      return;
    }
    if (operands == 2) {
      launch_wide<D, DV, KT, 2, false>(a, grid, 0, stream);
      return;
    }
  }
  launch_wide<D, DV, KT, 1, false>(a, grid, 0, stream);
}

template <int D, int DV, int KT>
hipError_t launch_kt(const ChunkArgs& a, int operands, hipStream_t stream) {
  const int64_t tiles = most_tiles(a.num_rows, a.tokens, a.batch);
  launch_tiles<D, DV, KT>(a, operands, dim3((unsigned)(tiles * a.H), (unsigned)a.splits), stream);
  if (a.splits > 1) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    ChunkArgs m = a;
    m.tokens = 1;
    const int64_t rows = most_tiles(a.num_rows, 1, a.batch);
    hipLaunchKernelGGL((chunk_merge_kernel<DV>), dim3((unsigned)(rows * a.H)), dim3(kThreads), 0, stream, m);
  }
  return hipGetLastError();
}

template <int D, int DV>
hipError_t launch_d(const ChunkArgs& a, int kt, int operands, hipStream_t stream) {
  if (kt == kKvFp8E4M3) return launch_kt<D, DV, kKvFp8E4M3>(a, operands, stream);
  if (kt == kKvFp8E5M2) return launch_kt<D, DV, kKvFp8E5M2>(a, operands, stream);
  if constexpr (D == DV) {
    if (kt == kKvMxFp4) return launch_kt<D, DV, kKvMxFp4>(a, operands, stream);
  }
  return launch_kt<D, DV, kKvBf16>(a, operands, stream);
}

}  // namespace

size_t chunk_attention_workspace(const Geometry& g, int n, int Hq, bool sparse, int max_sel) {
  return plan_of(g, n, Hq, sparse, max_sel).bytes;
}

// The same for any call of at most n rows, g.batch requests and max_sel blocks a list.  Tiles of T tokens and H heads number at
// least rows H / T, so that rows times parts is at most T kTargetWgs / H (or rows times `most`), and of halves 2 T kHalvesTo / H.
size_t chunk_attention_workspace_up_to(const Geometry& g, int n, int Hq, bool sparse, int max_sel) {
  const int group = Hq / g.H;
  const bool latent = g.Dqk != g.Dv;
  int64_t most = 0;
  for (int operands = 0; operands <= 2; operands++) {
    if ((operands == 0 && (latent || g.kv_dtype == kKvBf16)) || (operands == 2 && (latent || sparse))) continue;
    const int T = tile_tokens(operands, group, sparse);
    const int64_t parts = most_parts(g, T, sparse, max_sel);
    if (parts <= 1) continue;
    most = std::max(most, std::min<int64_t>(n * parts, (int64_t)T * kTargetWgs / g.H));
    if (latent) most = std::max(most, 2 * std::min<int64_t>(n, (int64_t)T * kHalvesTo / g.H));
  }
  return std::max<size_t>((size_t)most * Hq * part_bytes(g), 16);
}

hipError_t launch_chunk_attention(const Geometry& g, const ChunkRows& rows, const ChunkSelection& sel, int window,
                                  bool causal, float sm_scale, uint16_t* out, float* lse, void* ws, hipStream_t stream) {
  if (g.batch == 0 || rows.n == 0) return hipSuccess;
  ChunkArgs a{};
  a.q = rows.q;
  a.q_row = rows.row_stride;
  a.q_head = rows.head_stride;
  a.q_indptr = rows.indptr;
  a.q_lens = rows.lens;
  a.num_rows = rows.n;
  a.k = g.k;
  a.v = g.v;
  a.indptr = g.indptr;
  a.indices = g.indices;
  a.seq_lens = g.seq_lens;
  a.batch = g.batch;
  a.max_pages = g.max_pages / g.r;
  a.H = g.H;
  a.Hq = rows.Hq;
  a.g = rows.Hq / g.H;
  a.ps = g.ps;
  a.ps_shift = __builtin_ctz((unsigned)g.ps);
  a.num_phys = g.num_phys_pages;
  a.bs = g.bs;
  a.bs_shift = __builtin_ctz((unsigned)g.bs);
  a.sel_pages = sel.pages;
  a.sel_count = sel.count;
  a.max_sel = sel.max_sel;
  a.max_blocks = g.max_pages;
  a.window = std::min(window, 1 << 30);
  a.causal = causal ? 1 : 0;
  a.scale_log2 = sm_scale * 1.44269504088896341f * g.k_scale;
  a.v_scale = g.v ? g.v_scale : g.k_scale;
  a.out = out;
  a.lse = lse;
  const Plan p = plan_of(g, rows.n, rows.Hq, sel.pages != nullptr, sel.max_sel);
  a.tokens = p.tokens;
  a.splits = p.splits;
  a.part_o = static_cast<float*>(ws);
  a.part_ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + p.o_bytes);
  if (g.Dqk == 128) return launch_d<128, 128>(a, g.kv_dtype, p.operands, stream);
  if (g.Dqk == 64) return launch_d<64, 64>(a, g.kv_dtype, p.operands, stream);
  return launch_d<576, 512>(a, g.kv_dtype, p.operands, stream);
}

}  // namespace vx
