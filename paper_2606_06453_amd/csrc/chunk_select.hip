// The blocks that each token of a chunk attends (vx_chunk_score_topk): block-mean scores of every block before
// its own, then the sink and local blocks and the best others.
//
// A score is sum_c qbar_c mean_jc in fp64, rounded to fp32 (qbar: the mean of the group's queries), and the
// selection is by these scores exactly.  Few of them are computed so:
//   1. A workgroup takes up to 32 tokens and one KV head.  Scores s' come from matrix products of bf16 parts,
//      qbar = qh + ql and mean = mh + ml (s' = qh mh + ql mh + qh ml in fp32), and stay in LDS as bf16 numbers f.
//   2. |s - f| <= B = kBound |qbar| max_j |mean_j| + 2^-8 max_j |f_j|: the parts leave 2^-16 of a channel each
//      and the product of the low ones, 3 D additions 2^-23 of their sum each, together below 2^-13 of the
//      norms' product (Cauchy-Schwarz); bf16 rounds by 2^-8 of a value.  The norms of the means are the diagonal of a
//      matrix product too.
//   3. A wave finds the K-th largest f of a row (histograms that narrow down on it) to lie within [lo, hi].  Blocks
//      with f - 2 B > hi have fewer than K others at or above them: in.  Blocks with f + 2 B < lo: out.
//   4. The others, a dozen or so, are scored in fp64 and ranked, ties to the lower block.
// Rows with more than kMostOpen of them (many equal scores), and rows where a norm is not finite or so small that
// its square is lost, select by digits of the exact scores alone, which they compute anew for every digit.
#include <algorithm>

#include "chunk_tile.h"

namespace vx {
using namespace chunk;
namespace {

constexpr int kThreads = 512, kWaves = kThreads / kWave;
constexpr int kBins = 256;
constexpr int kMostOpen = 128;
constexpr float kBound = 1.f / 4096.f;                   // twice the bound above
constexpr float kTinySquare = 7.9e-31f;                  // 2^-100

struct SelectArgs {
  const float* mean;
  const int32_t* budget;
  int n_sink, n_local, r, stride;          // stride: scores of a token in LDS
  int32_t* sel_pages;
  int32_t* sel_count;
};

// A wave's own LDS: a histogram, then the row's query.
struct WaveLds {
  union {
    uint32_t hist[kBins];
    double qbar[128];
  };
  uint32_t key[kMostOpen];
  uint16_t id[kMostOpen];
};

// LDS of a wave is written and read in order; the compiler keeps the order too.
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) x = fmaxf(x, xor_shfl(x, s));
  return x;
}
__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) x += __shfl_xor(x, s, kWave);
  return x;
}

// Keys of the exact scores of 8 blocks: block j8 of lane / 8 (below 0: none), qbar in LDS.  Every lane of the 8 gets
// its block's key.
template <int D>
__device__ __forceinline__ uint32_t exact_keys(const ChunkArgs& a, const SelectArgs& s, const Tile& t, int h, int j8,
                                               const double* qbar) {
  const int x = lane_id() & 7;
  double dot = 0.0;
  if (j8 >= 0) {
    const float* m = s.mean + (block_row(t.pages, j8, s.r, a.num_phys) * a.H + h) * D;
    float4 v[D / 32];
#pragma unroll
    for (int c = 0; c < D / 32; c++) v[c] = *reinterpret_cast<const float4*>(m + 32 * c + 4 * x);
#pragma unroll
    for (int c = 0; c < D / 32; c++) {
      const double* q = qbar + 32 * c + 4 * x;
      dot = fma(q[0], (double)v[c].x, dot);
      dot = fma(q[1], (double)v[c].y, dot);
      dot = fma(q[2], (double)v[c].z, dot);
      dot = fma(q[3], (double)v[c].w, dot);
    }
  }
#pragma unroll
  for (int y = 1; y < 8; y <<= 1) dot += __shfl_xor(dot, y, kWave);
  return float_key((float)dot);
}

// The row's K best candidates of [c0, c1) by their exact scores alone: flags[j] = 1 or 0.
template <int D>
__device__ __forceinline__ void select_by_digits(const ChunkArgs& a, const SelectArgs& s, const Tile& t, int h, int c0,
                                                 int c1, int want, const double* qbar, uint16_t* flags) {
  const int lane = lane_id(), sub = lane >> 3;
  uint32_t T = 0;
  int ties = want;
  for (int bit = 31; bit >= 0; bit -= 4) {               // 16 bins a digit, a lane each
    const int shift = bit - 3;
    const uint32_t above = shift == 28 ? 0u : ~0u << (shift + 4);
    int bin = 0;                                         // lane d < 16: candidates of digit d
    for (int j0 = c0; j0 < c1; j0 += 8) {
      const int j = j0 + sub;
      const uint32_t k = exact_keys<D>(a, s, t, h, j < c1 ? j : -1, qbar);
      const bool on = j < c1 && (lane & 7) == 0 && (k & above) == T;
      const int d = (int)(k >> shift) & 15;
#pragma unroll
      for (int x = 0; x < 16; x++) {
        const int c = __popcll(__ballot(on && d == x));
        if (lane == x) bin += c;
      }
    }
    int d = 15;
    for (; d > 0; d--) {
      const int c = __builtin_amdgcn_readlane(bin, d);
      if (c >= ties) break;
      ties -= c;
    }
    T |= (uint32_t)d << shift;
  }
  int seen = 0;
  for (int j0 = c0; j0 < c1; j0 += 8) {
    const int j = j0 + sub;
    const uint32_t k = exact_keys<D>(a, s, t, h, j < c1 ? j : -1, qbar);
    const uint64_t eq = __ballot(j < c1 && (lane & 7) == 0 && k == T);
    const int before = seen + __popcll(eq & ((1ull << (lane & 56)) - 1));
    seen += __popcll(eq);
    if (j < c1 && (lane & 7) == 0) flags[j] = k > T || (k == T && before < ties) ? 1 : 0;
  }
}

template <int D, int CG>
__global__ __launch_bounds__(kThreads) void chunk_select_kernel(const ChunkArgs a, const SelectArgs s) {
  constexpr int KS = D / 32, TOK = 16 * CG;
  extern __shared__ __attribute__((aligned(16))) uint16_t slab[];          // [token][stride]
  __shared__ WaveLds wave_lds[kWaves];
  __shared__ uint32_t key_lo[TOK], key_hi[TOK], norm_q[TOK], norm_m;       // ordered bits of floats
  const int tid = (int)threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, grp = lane >> 4;
  const int h = (int)blockIdx.x % a.H;
  Tile t;
  if (!find_tile(a, (int)blockIdx.x / a.H, t)) return;
  const int total = min(max(s.budget[t.i], 0), a.max_sel);
  const int nb_all = min((t.len + a.bs - 1) >> a.bs_shift, a.max_blocks);
  auto blocks_of = [&](int x) { return t.p0 + x < 0 ? 0 : min(((t.p0 + x) >> a.bs_shift) + 1, nb_all); };
  const int nb_last = blocks_of(t.n - 1);
  const int c0 = min(s.n_sink, nb_last), c1_last = max(nb_last - s.n_local, c0);       // candidates of the last token
  const bool scored = total < nb_last && total > 0 && c1_last > c0;

  if (tid < TOK) {
    key_lo[tid] = 0xffffffffu;
    key_hi[tid] = 0u;
    norm_q[tid] = 0u;
  }
  if (tid == 0) norm_m = 0u;
  __syncthreads();
  if (scored) {
    bf16x8_t qh[CG][KS], ql[CG][KS];
    int c1[CG];
#pragma unroll
    for (int y = 0; y < CG; y++) {
      const int x = 16 * y + col;
      const bool there = x < t.n;
      c1[y] = there ? max(blocks_of(x) - s.n_local, 0) : 0;
      const uint16_t* q = a.q + (t.row0 + (there ? x : 0)) * a.q_row + (int64_t)h * a.g * a.q_head;
      float square = 0.f;
#pragma unroll
      for (int kk = 0; kk < KS; kk++) {
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int g = 0; g < a.g; g++) {
          const uint4 w = *reinterpret_cast<const uint4*>(q + g * a.q_head + 32 * kk + 8 * grp);
          const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int e = 0; e < 4; e++) {
            v[2 * e] += bf16lo(ws[e]);
            v[2 * e + 1] += bf16hi(ws[e]);
          }
        }
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const float u = v[2 * e] / a.g, z = v[2 * e + 1] / a.g;
          square = fmaf(u, u, fmaf(z, z, square));
          hi[e] = pack_bf16(u, z);
          lo[e] = pack_bf16(u - bf16lo(hi[e]), z - bf16hi(hi[e]));
        }
        qh[y][kk] = __builtin_bit_cast(bf16x8_t, u32x4_t{hi[0], hi[1], hi[2], hi[3]});
        ql[y][kk] = __builtin_bit_cast(bf16x8_t, u32x4_t{lo[0], lo[1], lo[2], lo[3]});
      }
      square = column_sum(square);
      if (wave == 0 && grp == 0) norm_q[x] = __float_as_uint(square);
    }
    float least[CG], most[CG], norm = 0.f;
#pragma unroll
    for (int y = 0; y < CG; y++) {
      least[y] = INFINITY;
      most[y] = -INFINITY;
    }
    bool odd = false;                                    // a score that is not finite
    struct Means {
      float4 v[KS][2];
    };
    auto fetch = [&](int j0, Means& m) {                 // this lane: block j0 + col
      const int j = min(max(j0 + col, c0), c1_last - 1);
      const float* src = s.mean + (block_row(t.pages, j, s.r, a.num_phys) * a.H + h) * D + 8 * grp;
#pragma unroll
      for (int kk = 0; kk < KS; kk++) {
        m.v[kk][0] = *reinterpret_cast<const float4*>(src + 32 * kk);
        m.v[kk][1] = *reinterpret_cast<const float4*>(src + 32 * kk + 4);
      }
    };
    auto score = [&](int j0, const Means& m) {
      f32x4_t sc[CG], gram = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int y = 0; y < CG; y++) sc[y] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < KS; kk++) {
        const float v[8] = {m.v[kk][0].x, m.v[kk][0].y, m.v[kk][0].z, m.v[kk][0].w,
                            m.v[kk][1].x, m.v[kk][1].y, m.v[kk][1].z, m.v[kk][1].w};
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int e = 0; e < 4; e++) {
          hi[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
          lo[e] = pack_bf16(v[2 * e] - bf16lo(hi[e]), v[2 * e + 1] - bf16hi(hi[e]));
        }
        const bf16x8_t mh = __builtin_bit_cast(bf16x8_t, u32x4_t{hi[0], hi[1], hi[2], hi[3]});
        const bf16x8_t ml = __builtin_bit_cast(bf16x8_t, u32x4_t{lo[0], lo[1], lo[2], lo[3]});
        gram = __builtin_amdgcn_mfma_f32_16x16x32_bf16(mh, mh, gram, 0, 0, 0);
#pragma unroll
        for (int y = 0; y < CG; y++) {
          sc[y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ml, qh[y][kk], sc[y], 0, 0, 0);
          sc[y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(mh, ql[y][kk], sc[y], 0, 0, 0);
          sc[y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(mh, qh[y][kk], sc[y], 0, 0, 0);
        }
      }
      // lane (grp, col): scores of blocks j0 + 4 grp + i and token 16 y + col; blocks' own products on the diagonal
      if ((col >> 2) == grp && j0 + col >= c0 && j0 + col < c1_last) {
        const float d = (col & 2) ? ((col & 1) ? gram[3] : gram[2]) : ((col & 1) ? gram[1] : gram[0]);
        norm = d != d ? INFINITY : fmaxf(norm, d);
      }
#pragma unroll
      for (int y = 0; y < CG; y++) {
        const uint2 w = make_uint2(pack_bf16(sc[y][0], sc[y][1]), pack_bf16(sc[y][2], sc[y][3]));
        if (CG > 1 || col < a.tokens) *reinterpret_cast<uint2*>(slab + (16 * y + col) * s.stride + j0 + 4 * grp) = w;
        const float f[4] = {bf16lo(w.x), bf16hi(w.x), bf16lo(w.y), bf16hi(w.y)};
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const int j = j0 + 4 * grp + i;
          const bool on = j >= c0 && j < c1[y];
          least[y] = on ? fminf(least[y], f[i]) : least[y];
          most[y] = on ? fmaxf(most[y], f[i]) : most[y];
          odd = odd || (on && !(fabsf(f[i]) < INFINITY));
        }
      }
    };
    const int g0 = c0 >> 4, g1 = (c1_last + 15) >> 4;    // groups of 16 blocks
    Means ma, mb;
    int g = g0 + wave;
    if (g < g1) fetch(16 * g, ma);
    for (; g < g1; g += 2 * kWaves) {
      fetch(16 * min(g + kWaves, g1 - 1), mb);
      score(16 * g, ma);
      if (g + kWaves >= g1) break;
      fetch(16 * min(g + 2 * kWaves, g1 - 1), ma);
      score(16 * (g + kWaves), mb);
    }
    norm = __any(odd) ? INFINITY : wave_max(norm);
    if (lane == 0) atomicMax(&norm_m, __float_as_uint(norm));              // not negative: ordered as its bits
#pragma unroll
    for (int y = 0; y < CG; y++) {
      const float hi = column_max(most[y]), lo = -column_max(-least[y]);
      if (grp == 0 && hi >= lo) {
        atomicMax(&key_hi[16 * y + col], float_key(hi));
        atomicMin(&key_lo[16 * y + col], float_key(lo));
      }
    }
  }
  __syncthreads();

  auto from_key = [](uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k); };
  WaveLds& mine = wave_lds[wave];
  for (int x = wave; x < t.n; x += kWaves) {
    const int64_t row = t.row0 + x;
    const int nb = blocks_of(x), forced = min(nb, s.n_sink + s.n_local);
    const int k0 = min(s.n_sink, nb), k1 = max(nb - s.n_local, k0);        // the row's candidates
    const bool all = total >= nb;
    const int want = all ? k1 - k0 : min(max(total - forced, 0), k1 - k0);
    uint16_t* f16 = slab + x * s.stride;
    const bool choose = want > 0 && want < k1 - k0;
    if (choose) {
      const float square = __uint_as_float(norm_q[x]), norm = __uint_as_float(norm_m);
      float lo = from_key(key_lo[x]), hi = from_key(key_hi[x]);
      bool exact = !(square < INFINITY) || !(norm < INFINITY) || square < kTinySquare || norm < kTinySquare;
      int open = 0, in = 0;
      if (!exact) {
        const float bound = 2.f * (kBound * sqrtf(square) * sqrtf(norm) + 0.00392f * fmaxf(fabsf(lo), fabsf(hi)));
        // narrow [lo, hi] down around the K-th largest
        int left = want;
        for (int level = 0; level < 4 && hi > lo; level++) {
          const float scale = kBins / (hi - lo);
          for (int b = lane; b < kBins; b += kWave) mine.hist[b] = 0;
          wave_fence();
          auto bin_of = [&](float f) { return min(max((int)((f - lo) * scale), 0), kBins - 1); };
          for (int p = lane; 2 * p < k1; p += kWave) {
            const uint32_t w = reinterpret_cast<const uint32_t*>(f16)[p];
            const float f0 = bf16lo(w), f1 = bf16hi(w);
            if (2 * p >= k0 && f0 >= lo && f0 <= hi) atomicAdd(&mine.hist[bin_of(f0)], 1u);
            if (2 * p + 1 >= k0 && 2 * p + 1 < k1 && f1 >= lo && f1 <= hi) atomicAdd(&mine.hist[bin_of(f1)], 1u);
          }
          wave_fence();
          // lane y: bins 255 - 4 y .. 252 - 4 y, from the top
          int c[4], sum = 0;
#pragma unroll
          for (int e = 0; e < 4; e++) sum += c[e] = (int)mine.hist[kBins - 1 - 4 * lane - e];
          int upto = sum;
#pragma unroll
          for (int y = 1; y < kWave; y <<= 1) {
            const int z = __shfl_up(upto, y, kWave);
            if (lane >= y) upto += z;
          }
          const int src = __builtin_ctzll(__ballot(upto >= left) | (1ull << 63));
          int before = upto - sum, bin = kBins - 1 - 4 * lane;
#pragma unroll
          for (int e = 0; e < 3; e++)
            if (before + c[e] < left && bin == kBins - 1 - 4 * lane - e) {
              before += c[e];
              bin--;
            }
          bin = __builtin_amdgcn_readlane(bin, src);
          before = __builtin_amdgcn_readlane(before, src);
          const int here = (int)mine.hist[bin];
          float top = -INFINITY, low = INFINITY;
          for (int p = lane; 2 * p < k1; p += kWave) {
            const uint32_t w = reinterpret_cast<const uint32_t*>(f16)[p];
            const float f0 = bf16lo(w), f1 = bf16hi(w);
            if (2 * p >= k0 && f0 >= lo && f0 <= hi && bin_of(f0) == bin) {
              top = fmaxf(top, f0);
              low = fminf(low, f0);
            }
            if (2 * p + 1 >= k0 && 2 * p + 1 < k1 && f1 >= lo && f1 <= hi && bin_of(f1) == bin) {
              top = fmaxf(top, f1);
              low = fminf(low, f1);
            }
          }
          hi = wave_max(top);
          lo = -wave_max(-low);
          left -= before;
          if (here <= 16) break;
        }
        // in, out, or open
        for (int j0 = 0; j0 < k1; j0 += kWave) {
          const int j = j0 + lane;
          const bool cand = j >= k0 && j < k1;
          const float f = cand ? __uint_as_float((uint32_t)f16[j] << 16) : 0.f;
          const bool yes = cand && f - bound > hi, no = f + bound < lo;
          const bool ask = cand && !yes && !no;
          int n;
          const int at = open + wave_excl_count(ask, &n);
          if (ask && at < kMostOpen) mine.id[at] = (uint16_t)j;
          if (cand) f16[j] = yes ? 1 : 0;
          open += n;
          in += __popcll(__ballot(yes));
        }
        exact = open > kMostOpen;
      }
      wave_fence();
      // the row's query in fp64
      for (int c = lane; c < D; c += kWave) {
        double sum = 0.0;
        for (int g = 0; g < a.g; g++)
          sum += (double)bf16_to_f32(a.q[row * a.q_row + (int64_t)(h * a.g + g) * a.q_head + c]);
        mine.qbar[c] = sum / a.g;
      }
      wave_fence();
      if (exact) {
        select_by_digits<D>(a, s, t, h, k0, k1, want, mine.qbar, f16);
      } else {
        for (int u = 0; u < open; u += 8) {
          const int y = u + (lane >> 3);
          const uint32_t k = exact_keys<D>(a, s, t, h, y < open ? (int)mine.id[y] : -1, mine.qbar);
          if (y < open && (lane & 7) == 0) mine.key[y] = k;
        }
        wave_fence();
        for (int u = lane; u < open; u += kWave) {       // ids ascend: of equal scores the earlier entry
          const uint32_t k = mine.key[u];
          int rank = 0;
          for (int y = 0; y < open; y++) rank += mine.key[y] > k || (mine.key[y] == k && y < u);
          if (rank < want - in) f16[mine.id[u]] = 1;
        }
      }
      wave_fence();
    }
    // the list, ascending
    int32_t* sel = s.sel_pages + (row * a.H + h) * a.max_sel;
    int at = 0;
    for (int j0 = 0; j0 < nb; j0 += kWave) {
      const int j = j0 + lane;
      const bool must = j < s.n_sink || j >= nb - s.n_local;
      const bool take = j < nb && (must || want == k1 - k0 || (choose && f16[j] == 1));
      int n;
      const int place = at + wave_excl_count(take, &n);
      if (take && place < a.max_sel) sel[place] = j;
      at += n;
    }
    for (int y = at + lane; y < a.max_sel; y += kWave) sel[y] = -1;
    if (h == 0 && lane == 0) s.sel_count[row] = at;
  }
}

template <int D>
hipError_t launch(ChunkArgs& a, SelectArgs& s, hipStream_t stream) {
  // tokens of a workgroup: as many as leave their scores room in LDS.  Rows are 16 bytes past a multiple of 64, so
  // that the 16 tokens of a store spread over the banks.
  s.stride = ((a.max_blocks + 31) & ~31) + 8;
  int tokens = 32;
  while (tokens > 4 && (size_t)tokens * s.stride * sizeof(uint16_t) > 136 * 1024) tokens /= 2;
  a.tokens = tokens;
  const int64_t tiles = (int64_t)a.num_rows / tokens + a.batch;
  const dim3 grid((unsigned)(tiles * a.H));
  const size_t lds = sizeof(uint16_t) * (size_t)tokens * s.stride;
  if (tokens == 32) hipLaunchKernelGGL((chunk_select_kernel<D, 2>), grid, dim3(kThreads), lds, stream, a, s);
  else hipLaunchKernelGGL((chunk_select_kernel<D, 1>), grid, dim3(kThreads), lds, stream, a, s);
  return hipGetLastError();
}

}  // namespace

size_t chunk_select_workspace(const Geometry& g, int n, int Hq) { return 16; }

hipError_t launch_chunk_select(const Geometry& g, const ChunkRows& rows, const float* mean, const int32_t* budget,
                               int n_sink, int n_local, int max_sel, int32_t* sel_pages, int32_t* sel_count, void* ws,
                               hipStream_t stream) {
  if (g.batch == 0 || rows.n == 0) return hipSuccess;
  ChunkArgs a{};
  a.q = rows.q;
  a.q_row = rows.row_stride;
  a.q_head = rows.head_stride;
  a.q_indptr = rows.indptr;
  a.q_lens = rows.lens;
  a.num_rows = rows.n;
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
  a.max_sel = max_sel;
  a.max_blocks = g.max_pages;
  SelectArgs s{mean, budget, n_sink, n_local, g.r, 0, sel_pages, sel_count};
  return g.Dqk == 128 ? launch<128>(a, s, stream) : launch<64>(a, s, stream);
}

}  // namespace vx
