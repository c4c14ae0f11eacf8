// The blocks that each token of a chunk attends (vx_chunk_score_topk): block-mean scores of every block before
// its own, then the sink and local blocks and the best others.
//
// A score is sum_c qbar_c mean_jc in fp64, rounded to fp32 (qbar: the mean of the group's queries, summed in fp64), and the
// selection is by these scores exactly.  Few of them are computed so:
//   1. chunk_score_kernel: scores s' from matrix products of bf16 parts, qbar = qh + ql and mean = mh + ml
//      (s' = qh mh + ql mh + qh ml in fp32), kept as bf16 numbers f in the workspace.  A workgroup takes up to 64
//      tokens, one KV head and a part of the blocks; a wave splits 16 means into their parts once for all tokens.
//   2. |s - f| <= B = kBound |qbar| max_j |mean_j| + 2^-8 max_j |f_j|: the parts leave 2^-16 of a channel each
//      (of qbar itself, however its heads cancel) and the product of the low ones, 3 D additions 2^-23 of their sum
//      each, together below 2^-13 of the norms' product (Cauchy-Schwarz); bf16 rounds by 2^-8 of a value.  The
//      norms of the means are the diagonal of a matrix product too.
//   3. chunk_choose_kernel, a wave a row and KV head: the K-th largest f (histograms that narrow down on it) lies
//      within [lo, hi].  Blocks with f - 2 B > hi have fewer than K others at or above them: in.  Blocks with
//      f + 2 B < lo: out.
//   4. The others, two dozen or so, are scored in fp64 and ranked, ties to the lower block.
// Rows with more than kMostOpen of them (many equal scores), and rows where a norm is not finite or so small that
// its square is lost, select by digits of the exact scores alone, which they compute anew for every digit.
// One kernel that kept the scores of 32 tokens in LDS took 388 us for 4096 tokens over 2048 blocks and 55 us for a few
// users' drafted tokens: a row's passes waited with two waves a SIMD, and few tokens left most of the chip idle.
// Now 231 and 37 us: 4096 tokens take 95 us of scores and 123 us of choosing, which vector instructions bound (2200 a
// row); eight users' 4 tokens each 17 us and 17 us, which are the latencies of a few dependent passes.  With equal means
// every row selects by digits: 17 ms and 2 ms.
#include <algorithm>

#include "chunk_tile.h"

namespace vx {
using namespace chunk;
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kBins = 256;
constexpr int kMostOpen = 128;
constexpr int kFewInBin = 32;
constexpr int kTogether = 2;               // times 8 open blocks whose means travel together
constexpr int kScoreWgs = 512;             // workgroups of the scores that fill the chip (1024: 234 and 38 us where 230 and 36 are, at the top)
constexpr int kUnit = 32;                  // blocks that a wave looks up at a time
constexpr size_t kScoreBytes = (size_t)128 << 20;        // of scores at a time: half of the last cache
constexpr float kBound = 1.f / 4096.f;                   // twice the bound above
constexpr float kTinySquare = 7.9e-31f;                  // 2^-100

struct SelectArgs {
  const float* mean;
  const int32_t* budget;
  int n_sink, n_local, r;
  int32_t* sel_pages;
  int32_t* sel_count;
  uint16_t* scores;                        // [tile][H][tokens][stride]
  float* norms;                            // [tile][H][parts]: largest square of the means' norms
  int stride, part, parts;                 // of a row; blocks of a part
  int tile0;                               // first tile of the launch
};

// What a tile's tokens select among.
struct Scope {
  int total;                               // the budget
  int nb_all;                              // blocks of the request
  int c0, c1;                              // candidates of the last token
  bool scored;
};
__device__ __forceinline__ int blocks_of(const ChunkArgs& a, const Tile& t, const Scope& c, int x) {
  return t.p0 + x < 0 ? 0 : min(((t.p0 + x) >> a.bs_shift) + 1, c.nb_all);
}
__device__ __forceinline__ Scope scope_of(const ChunkArgs& a, const SelectArgs& s, const Tile& t) {
  Scope c;
  c.total = min(max(s.budget[t.i], 0), a.max_sel);
  c.nb_all = min((t.len + a.bs - 1) >> a.bs_shift, a.max_blocks);
  const int nb = blocks_of(a, t, c, t.n - 1);
  c.c0 = min(s.n_sink, nb);
  c.c1 = max(nb - s.n_local, c.c0);
  c.scored = c.total < nb && c.total > 0 && c.c1 > c.c0;
  return c;
}

// A wave's own LDS: a histogram, then the row's query.
struct WaveLds {
  union {
    uint32_t hist[kBins];
    double qbar[128];
  };
  __attribute__((aligned(16))) uint32_t key[kMostOpen];
  uint16_t id[kMostOpen];
};

// LDS of a wave is written and read in order; the compiler keeps the order too.
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// Over the wave, in registers (row_ror within 16 lanes, then swaps of 16 and 32): a row takes a dozen of these one
// after the other, and each through LDS costs six of its round trips.
__device__ __forceinline__ float wave_max(float x) {
  x = fmaxf(x, dpp_f32<0x128>(x));
  x = fmaxf(x, dpp_f32<0x124>(x));
  x = fmaxf(x, dpp_f32<0x122>(x));
  x = fmaxf(x, dpp_f32<0x121>(x));
  return column_max(x);
}
// Sum over this lane and those below it: row_shr 1, 2, 4, 8, then the sums of the rows before (row_bcast 15 and 31).
__device__ __forceinline__ int wave_prefix(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}

// Keys of the exact scores of N times 8 blocks, qbar in LDS: row8[z] is the summary row of the block of this lane's 8
// (below 0: none), and every lane of the 8 gets its key.
template <int D, int N>
__device__ __forceinline__ void exact_keys(const ChunkArgs& a, const SelectArgs& s, int h, const int (&row8)[N],
                                           const double* qbar, uint32_t (&key)[N]) {
  const int x = lane_id() & 7;
  float4 v[N][D / 32];
#pragma unroll
  for (int z = 0; z < N; z++) {
    const float* m = s.mean + ((int64_t)max(row8[z], 0) * a.H + h) * D;
#pragma unroll
    for (int c = 0; c < D / 32; c++) v[z][c] = *reinterpret_cast<const float4*>(m + 32 * c + 4 * x);
  }
#pragma unroll
  for (int z = 0; z < N; z++) {
    double dot = 0.0;
#pragma unroll
    for (int c = 0; c < D / 32; c++) {
      const double* q = qbar + 32 * c + 4 * x;
      dot = fma(q[0], (double)v[z][c].x, dot);
      dot = fma(q[1], (double)v[z][c].y, dot);
      dot = fma(q[2], (double)v[z][c].z, dot);
      dot = fma(q[3], (double)v[z][c].w, dot);
    }
#pragma unroll
    for (int y = 1; y < 8; y <<= 1) dot += __shfl_xor(dot, y, kWave);
    key[z] = float_key((float)dot);
  }
}

// The row's K best candidates of [c0, c1) by their exact scores alone: flags[j] = 1 or 0.
template <int D>
__device__ __forceinline__ void select_by_digits(const ChunkArgs& a, const SelectArgs& s, const Tile& t, int h, int c0,
                                                 int c1, int want, const double* qbar, uint16_t* flags) {
  const int lane = lane_id(), sub = lane >> 3;
  auto key_of = [&](int j) {
    const int row8[1] = {(int)block_row(t.pages, min(j, c1 - 1), s.r, a.num_phys)};
    uint32_t k[1];
    exact_keys<D, 1>(a, s, h, row8, qbar, k);
    return k[0];
  };
  uint32_t T = 0;
  int ties = want;
  for (int bit = 31; bit >= 0; bit -= 4) {               // 16 bins a digit, a lane each
    const int shift = bit - 3;
    const uint32_t above = shift == 28 ? 0u : ~0u << (shift + 4);
    int bin = 0;                                         // lane d < 16: candidates of digit d
    for (int j0 = c0; j0 < c1; j0 += 8) {
      const int j = j0 + sub;
      const uint32_t k = key_of(j);
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
    const uint32_t k = key_of(j);
    const uint64_t eq = __ballot(j < c1 && (lane & 7) == 0 && k == T);
    const int before = seen + __popcll(eq & ((1ull << (lane & 56)) - 1));
    seen += __popcll(eq);
    if (j < c1 && (lane & 7) == 0) flags[j] = k > T || (k == T && before < ties) ? 1 : 0;
  }
}

// CG groups of 16 tokens, all of whose queries stay in registers, and a part of the blocks.  4096 tokens over 2048
// blocks of 8 heads, 95 us: matrix instructions 27% and vector ones, which split the means (once for 64 tokens), 34% of
// the time; the means come from the caches, 8 MB for every 64 tokens.
template <int D, int CG>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2))) void chunk_score_kernel(const ChunkArgs a, const SelectArgs s) {
  constexpr int KS = D / 32;
  __shared__ bf16x8_t parts[CG][KS][2][kWave];           // qh and ql, operand B
  __shared__ uint32_t norm_m;                            // of a float that is not negative: ordered as its bits
  const int tid = (int)threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, grp = lane >> 4;
  const int h = (int)blockIdx.x % a.H, xt = (int)blockIdx.x / a.H, part = (int)blockIdx.y;
  Tile t;
  if (!find_tile(a, s.tile0 + xt, t)) return;
  const Scope c = scope_of(a, s, t);
  const int j_lo = max(c.c0 & ~(kUnit - 1), part * s.part), j_hi = min((c.c1 + kUnit - 1) & ~(kUnit - 1), (part + 1) * s.part);
  if (tid == 0) norm_m = 0u;
  if (!c.scored) return;
  float* norm_out = s.norms + ((int64_t)xt * a.H + h) * s.parts + part;
  if (j_lo >= j_hi) {
    if (tid == 0) *norm_out = 0.f;
    return;
  }
  const double share = 1.0 / a.g;
  for (int y = wave; y < CG; y += kWaves) {
    const int x = 16 * y + col;
    const bool there = x < t.n;
    const uint16_t* q = a.q + (t.row0 + (there ? x : 0)) * a.q_row + (int64_t)h * a.g * a.q_head;
#pragma unroll
    for (int kk = 0; kk < KS; kk++) {
      // in fp64: where a group's queries cancel, an fp32 sum is off by more than the bound of what is left
      double v[8] = {0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0};
      for (int g = 0; g < a.g; g++) {
        const uint4 w = *reinterpret_cast<const uint4*>(q + g * a.q_head + 32 * kk + 8 * grp);
        const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; e++) {
          v[2 * e] += (double)bf16lo(ws[e]);
          v[2 * e + 1] += (double)bf16hi(ws[e]);
        }
      }
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const double u = v[2 * e] * share, z = v[2 * e + 1] * share;
        hi[e] = pack_bf16((float)u, (float)z);
        lo[e] = pack_bf16((float)(u - (double)bf16lo(hi[e])), (float)(z - (double)bf16hi(hi[e])));
      }
      parts[y][kk][0][lane] = __builtin_bit_cast(bf16x8_t, u32x4_t{hi[0], hi[1], hi[2], hi[3]});
      parts[y][kk][1][lane] = __builtin_bit_cast(bf16x8_t, u32x4_t{lo[0], lo[1], lo[2], lo[3]});
    }
  }
  __syncthreads();
  bf16x8_t qh[CG][KS], ql[CG][KS];
#pragma unroll
  for (int y = 0; y < CG; y++)
#pragma unroll
    for (int kk = 0; kk < KS; kk++) {
      qh[y][kk] = parts[y][kk][0][lane];
      ql[y][kk] = parts[y][kk][1][lane];
    }
  uint16_t* out = s.scores + (((int64_t)xt * a.H + h) * a.tokens) * s.stride;
  float norm = 0.f;
  struct Means {
    float4 v[KS][2];
  };
  // a lane finds the summary row of one of the unit's blocks, then two groups of 16 are scored
  auto find = [&](int j0) {
    const int j = min(max(j0 + (lane & (kUnit - 1)), c.c0), c.c1 - 1);
    return (int)block_row(t.pages, j, s.r, a.num_phys);
  };
  auto fetch = [&](int found, int q, Means& m) {         // this lane: block 16 q + col of the unit
    const float* src = s.mean + ((int64_t)__shfl(found, 16 * q + col, kWave) * a.H + h) * D + 8 * grp;
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
    if ((col >> 2) == grp && j0 + col >= c.c0 && j0 + col < c.c1) {
      const float d = (col & 2) ? ((col & 1) ? gram[3] : gram[2]) : ((col & 1) ? gram[1] : gram[0]);
      norm = d != d ? INFINITY : fmaxf(norm, d);
    }
#pragma unroll
    for (int y = 0; y < CG; y++) {
      if (16 * y + col < t.n)
        *reinterpret_cast<uint2*>(out + (int64_t)(16 * y + col) * s.stride + j0 + 4 * grp) =
            make_uint2(pack_bf16(sc[y][0], sc[y][1]), pack_bf16(sc[y][2], sc[y][3]));
    }
  };
  int j0 = j_lo + kUnit * wave;
  if (j0 < j_hi) {
    int found = find(j0);
    Means ma, mb;
    fetch(found, 0, ma);
    for (; j0 < j_hi; j0 += kUnit * kWaves) {
      const int next = find(min(j0 + kUnit * kWaves, j_hi - kUnit));
      fetch(found, 1, mb);
      score(j0, ma);
      fetch(next, 0, ma);
      score(j0 + 16, mb);
      found = next;
    }
  }
  norm = wave_max(norm);
  if (lane == 0) atomicMax(&norm_m, __float_as_uint(norm));
  __syncthreads();
  if (tid == 0) *norm_out = __uint_as_float(norm_m);
}

// A wave a row; six waves a SIMD, for a row's passes depend on one another (two: 264 -> 238 us for 4096 tokens,
// scores included).  Vector instructions bound it.
template <int D>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(6))) void chunk_choose_kernel(const ChunkArgs a, const SelectArgs s) {
  extern __shared__ __attribute__((aligned(16))) uint16_t slab[];          // [wave][stride]
  __shared__ WaveLds wave_lds[kWaves];
  const int tid = (int)threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int groups = (a.tokens + kWaves - 1) / kWaves;   // of a tile's rows, one a wave
  const int h = (int)blockIdx.x % a.H, xt = (int)blockIdx.x / a.H / groups;
  const int x = ((int)blockIdx.x / a.H - xt * groups) * kWaves + wave;
  Tile t;
  if (!find_tile(a, s.tile0 + xt, t) || x >= t.n) return;
  const Scope c = scope_of(a, s, t);
  const int total = c.total;
  WaveLds& mine = wave_lds[wave];
  {
    const int64_t row = t.row0 + x;
    const int nb = blocks_of(a, t, c, x), forced = min(nb, s.n_sink + s.n_local);
    const int k0 = min(s.n_sink, nb), k1 = max(nb - s.n_local, k0);        // the row's candidates
    const bool all = total >= nb;
    const int want = all ? k1 - k0 : min(max(total - forced, 0), k1 - k0);
    uint16_t* f16 = slab + wave * s.stride;
    const bool choose = want > 0 && want < k1 - k0;
    // lane's 8 blocks from j on: which of them are in [lo, hi), and their scores
    auto inside = [&](int j, int lo, int hi) {
      return (int)((1u << min(max(hi - j, 0), 8)) - 1) & ~(int)((1u << min(max(lo - j, 0), 8)) - 1);
    };
    auto eight = [&](int j, float (&f)[8]) {
      const uint4 w = *reinterpret_cast<const uint4*>(f16 + j);
      const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int e = 0; e < 4; e++) {
        f[2 * e] = bf16lo(ws[e]);
        f[2 * e + 1] = bf16hi(ws[e]);
      }
    };
    if (choose) {
      // the row's query in fp64
      double qsum[D / kWave];
#pragma unroll
      for (int y = 0; y < D / kWave; y++) qsum[y] = 0.0;
      for (int g = 0; g < a.g; g += 4) {
        uint16_t q[4][D / kWave];
#pragma unroll
        for (int z = 0; z < 4; z++)
#pragma unroll
          for (int y = 0; y < D / kWave; y++)
            q[z][y] = a.q[row * a.q_row + (int64_t)(h * a.g + min(g + z, a.g - 1)) * a.q_head + y * kWave + lane];
#pragma unroll
        for (int z = 0; z < 4; z++)
#pragma unroll
          for (int y = 0; y < D / kWave; y++) qsum[y] += g + z < a.g ? (double)bf16_to_f32(q[z][y]) : 0.0;
      }
      // the row's scores into LDS; their ends, and the largest norm of the means
      const uint16_t* src = s.scores + (((int64_t)xt * a.H + h) * a.tokens + x) * s.stride;
      float lo = INFINITY, hi = -INFINITY, norm = 0.f;
      bool odd = false;
      for (int y = lane; y < s.parts; y += kWave) norm = fmaxf(norm, s.norms[((int64_t)xt * a.H + h) * s.parts + y]);
      for (int j = 8 * lane; j < k1; j += 8 * kWave) {
        const uint4 w = *reinterpret_cast<const uint4*>(src + j);
        *reinterpret_cast<uint4*>(f16 + j) = w;
        const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
        const int on = inside(j, k0, k1);
#pragma unroll
        for (int e = 0; e < 8; e++) {
          const float f = (e & 1) ? bf16hi(ws[e >> 1]) : bf16lo(ws[e >> 1]);
          const bool mine_ = (on >> e) & 1;
          odd = odd || (mine_ && f != f);
          lo = fminf(lo, mine_ ? f : INFINITY);
          hi = fmaxf(hi, mine_ ? f : -INFINITY);
        }
      }
      hi = wave_max(hi);
      lo = -wave_max(-lo);
      norm = wave_max(norm);
      int open = 0, in = 0;
      float square = 0.f;
#pragma unroll
      for (int y = 0; y < D / kWave; y++) {
        qsum[y] /= a.g;
        square = fmaf((float)qsum[y], (float)qsum[y], square);
      }
      square = column_sum(row16_sum_f32(square));
      bool exact = __any(odd) || !(fmaxf(fabsf(lo), fabsf(hi)) < INFINITY) || !(square < INFINITY) || !(norm < INFINITY) || square < kTinySquare || norm < kTinySquare;
      wave_fence();
      if (!exact) {
        const float bound = 2.f * (kBound * sqrtf(square) * sqrtf(norm) + 0.00392f * fmaxf(fabsf(lo), fabsf(hi)));
        // narrow [lo, hi] down around the K-th largest
        int left = want;
        for (int level = 0; level < 4 && hi > lo; level++) {
          const float scale = kBins / (hi - lo), base = -lo * scale;
#pragma unroll
          for (int b = 0; b < kBins; b += kWave) mine.hist[b + lane] = 0;
          wave_fence();
          auto bin_of = [&](float f) { return min(max((int)fmaf(f, scale, base), 0), kBins - 1); };
          for (int j = 8 * lane; j < k1; j += 8 * kWave) {
            float f[8];
            eight(j, f);
            const int on = inside(j, k0, k1);
            if (level == 0 && __all(on == 255)) {        // lo and hi are the row's ends
#pragma unroll
              for (int e = 0; e < 8; e++) atomicAdd(&mine.hist[bin_of(f[e])], 1u);
              continue;
            }
#pragma unroll
            for (int e = 0; e < 8; e++)
              if (((on >> e) & 1) && f[e] >= lo && f[e] <= hi) atomicAdd(&mine.hist[bin_of(f[e])], 1u);
          }
          wave_fence();
          // lane y: bins 255 - 4 y .. 252 - 4 y, from the top
          int c[4], sum = 0;
#pragma unroll
          for (int e = 0; e < 4; e++) sum += c[e] = (int)mine.hist[kBins - 1 - 4 * lane - e];
          const int upto = wave_prefix(sum);
          const int src = __builtin_ctzll(__ballot(upto >= left) | (1ull << 63));
          int before = upto - sum, down = 0;
#pragma unroll
          for (int e = 0; e < 3; e++)
            if (down == e && before + c[e] < left) {
              before += c[e];
              down++;
            }
          const int here = __builtin_amdgcn_readlane(down == 0 ? c[0] : down == 1 ? c[1] : down == 2 ? c[2] : c[3], src);
          const int bin = __builtin_amdgcn_readlane(kBins - 1 - 4 * lane - down, src);
          before = __builtin_amdgcn_readlane(before, src);
          if (here <= kFewInBin) {
            // the bin's ends, moved apart by more than the rounding of bin_of
            const float width = (hi - lo) * (1.f / kBins), slack = (hi - lo) * (1.f / 65536.f) + fmaxf(fabsf(lo), fabsf(hi)) * (1.f / 1048576.f);
            hi = fmaf((float)(bin + 1), width, lo) + slack;
            lo = fmaf((float)bin, width, lo) - slack;
            break;
          }
          float top = -INFINITY, low = INFINITY;
          for (int j = 8 * lane; j < k1; j += 8 * kWave) {
            float f[8];
            eight(j, f);
            const int on = inside(j, k0, k1);
#pragma unroll
            for (int e = 0; e < 8; e++)
              if (((on >> e) & 1) && f[e] >= lo && f[e] <= hi && bin_of(f[e]) == bin) {
                top = fmaxf(top, f[e]);
                low = fminf(low, f[e]);
              }
          }
          hi = wave_max(top);
          lo = -wave_max(-low);
          left -= before;
        }
        // in, out, or open
        for (int j0 = 0; j0 < k1; j0 += 8 * kWave) {
          const int j = j0 + 8 * lane;
          int yes = 0, ask = 0;
          if (j < k1) {
            float f[8];
            eight(j, f);
            const int on = inside(j, k0, k1);
#pragma unroll
            for (int e = 0; e < 8; e++) {
              yes |= (f[e] - bound > hi) << e;
              ask |= (!(f[e] + bound < lo)) << e;
            }
            yes &= on;
            ask &= on & ~yes;
            // flags in the scores' place: 1 is in
            *reinterpret_cast<uint4*>(f16 + j) = make_uint4((yes & 1) | (yes & 2) << 15, (yes >> 2 & 1) | (yes >> 2 & 2) << 15,
                                                            (yes >> 4 & 1) | (yes >> 4 & 2) << 15, (yes >> 6 & 1) | (yes >> 6 & 2) << 15);
          }
          in += __popc(yes);
          if (__any(ask)) {
            const int c = __popc(ask);
            int at = wave_prefix(c);
            const int n = __builtin_amdgcn_readlane(at, kWave - 1);
            at += open - c;
            for (int m = ask; m; m &= m - 1, at++)
              if (at < kMostOpen) mine.id[at] = (uint16_t)(j + __builtin_ctz(m));
            open += n;
          }
        }
        in = __builtin_amdgcn_readlane(wave_prefix(in), kWave - 1);
        exact = open > kMostOpen;
      }
      wave_fence();
#pragma unroll
      for (int y = 0; y < D / kWave; y++) mine.qbar[y * kWave + lane] = qsum[y];
      wave_fence();
      if (exact) {
        select_by_digits<D>(a, s, t, h, k0, k1, want, mine.qbar, f16);
      } else {
        for (int u = 0; u < open; u += 8 * kTogether) {
          int row8[kTogether];
#pragma unroll
          for (int z = 0; z < kTogether; z++) {
            const int y = u + 8 * z + (lane >> 3);
            row8[z] = y < open ? (int)block_row(t.pages, (int)mine.id[y], s.r, a.num_phys) : -1;
          }
          uint32_t k[kTogether];
          exact_keys<D, kTogether>(a, s, h, row8, mine.qbar, k);
#pragma unroll
          for (int z = 0; z < kTogether; z++) {
            const int y = u + 8 * z + (lane >> 3);
            if (y < open && (lane & 7) == 0) mine.key[y] = k[z];
          }
        }
        wave_fence();
        for (int u = lane; u < open; u += kWave) {       // ids ascend: of equal scores the earlier entry
          const uint32_t k = mine.key[u];
          int rank = 0;
          for (int y = 0; y < open; y += 4) {            // entries behind the last one count for none
            const uint4 o = *reinterpret_cast<const uint4*>(&mine.key[y]);
            const uint32_t os[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
            for (int z = 0; z < 4; z++) rank += y + z < open && (os[z] > k || (os[z] == k && y + z < u));
          }
          if (rank < want - in) f16[mine.id[u]] = 1;
        }
      }
      wave_fence();
    }
    // the list, ascending
    int32_t* sel = s.sel_pages + (row * a.H + h) * a.max_sel;
    int at = 0;
    const bool every = want == k1 - k0;
    for (int j0 = 0; j0 < nb; j0 += 8 * kWave) {
      const int j = j0 + 8 * lane, real = inside(j, 0, nb);
      int take = every ? real : real & ~inside(j, s.n_sink, nb - s.n_local);
      if (choose && j < k1) {
        const uint4 w = *reinterpret_cast<const uint4*>(f16 + j);
        const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
        int flags = 0;
#pragma unroll
        for (int e = 0; e < 4; e++) flags |= (int)((ws[e] & 1) | (ws[e] >> 15 & 2)) << (2 * e);
        take |= flags & inside(j, k0, k1);
      }
      const int c = __popc(take);
      int place = wave_prefix(c);
      const int n = __builtin_amdgcn_readlane(place, kWave - 1);
      place += at - c;
      for (int m = take; m; m &= m - 1, place++)
        if (place < a.max_sel) sel[place] = j + __builtin_ctz(m);
      at += n;
    }
    for (int y = at + lane; y < a.max_sel; y += kWave) sel[y] = -1;
    if (h == 0 && lane == 0) s.sel_count[row] = at;
  }
}

// Tokens of a tile, and what the workspace holds of a launch.
struct SelectPlan {
  int tokens, stride, part, parts;
  int64_t tiles;                           // of all rows (an upper bound)
  int at_once;                             // of a launch
  size_t scores, bytes;
};
SelectPlan plan_of(const Geometry& g, int n) {
  SelectPlan p{};
  const int64_t batch = std::max(g.batch, 1);
  p.tokens = (int64_t)n <= 16 * batch ? 16 : 64;
  p.tiles = most_tiles(n, p.tokens, batch);
  p.stride = (g.max_pages + 63) & ~63;
  const size_t tile = (size_t)p.tokens * g.H * p.stride * sizeof(uint16_t);
  p.at_once = (int)std::max<int64_t>(1, std::min<int64_t>(p.tiles, (int64_t)(kScoreBytes / tile)));
  // parts of at least a unit a wave
  const int64_t work = std::max<int64_t>(1, std::min<int64_t>(p.at_once, std::max<int64_t>(batch, (n + p.tokens - 1) / p.tokens)) * g.H);
  const int least = kUnit * kWaves, most = (p.stride + least - 1) / least;
  const int parts = (int)std::max<int64_t>(1, std::min<int64_t>(most, kScoreWgs / work));
  p.part = ((p.stride + parts - 1) / parts + least - 1) / least * least;
  p.parts = (p.stride + p.part - 1) / p.part;
  p.scores = (tile * p.at_once + 255) / 256 * 256;
  p.bytes = p.scores + sizeof(float) * (size_t)p.at_once * g.H * p.parts;
  return p;
}

template <int D>
hipError_t launch(const ChunkArgs& a, SelectArgs& s, const SelectPlan& p, hipStream_t stream) {
  const size_t lds = sizeof(uint16_t) * (size_t)kWaves * s.stride;
  const int groups = (p.tokens + kWaves - 1) / kWaves;
  for (int64_t x = 0; x < p.tiles; x += p.at_once) {
    const unsigned tiles = (unsigned)std::min<int64_t>(p.at_once, p.tiles - x);
    s.tile0 = (int)x;
    const dim3 grid(tiles * a.H, (unsigned)p.parts);
    if (p.tokens == 64) hipLaunchKernelGGL((chunk_score_kernel<D, 4>), grid, dim3(kThreads), 0, stream, a, s);
    else hipLaunchKernelGGL((chunk_score_kernel<D, 1>), grid, dim3(kThreads), 0, stream, a, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((chunk_choose_kernel<D>), dim3(tiles * groups * a.H), dim3(kThreads), lds, stream, a, s);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

size_t chunk_select_workspace(const Geometry& g, int n) { return plan_of(g, n).bytes; }

// The same for any call of at most n rows and g.batch requests: the larger of both tiles' scores, and norms of as many parts as a
// row can have.
size_t chunk_select_workspace_up_to(const Geometry& g, int n) {
  const int64_t batch = std::max(g.batch, 1);
  const int stride = (g.max_pages + 63) & ~63;
  const int parts = (stride + kUnit * kWaves - 1) / (kUnit * kWaves);
  size_t most = 0;
  for (const int tokens : {16, 64}) {
    const int64_t rows = tokens == 16 ? std::min<int64_t>(n, 16 * batch) : n;
    const size_t tile = (size_t)tokens * g.H * stride * sizeof(uint16_t);
    const int64_t tiles = std::max<int64_t>(1, std::min<int64_t>(most_tiles(rows, tokens, batch), (int64_t)(kScoreBytes / tile)));
    most = std::max(most, (tile * tiles + 255) / 256 * 256 + sizeof(float) * (size_t)tiles * g.H * parts);
  }
  return most;
}

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
  const SelectPlan p = plan_of(g, rows.n);
  a.tokens = p.tokens;
  SelectArgs s{mean, budget, n_sink, n_local, g.r, sel_pages, sel_count, static_cast<uint16_t*>(ws),
               reinterpret_cast<float*>(static_cast<char*>(ws) + p.scores), p.stride, p.part, p.parts, 0};
  return g.Dqk == 128 ? launch<128>(a, s, p, stream) : launch<64>(a, s, p, stream);
}

}  // namespace vx
