// The blocks that each token of a chunk attends (vx_chunk_score_topk): block-mean scores of every block before
// its own, then the sink and local blocks and the best others.
#include <algorithm>

#include "chunk_common.h"

namespace vx {
using namespace chunk;
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;

struct SelectArgs {
  const float* mean;
  const int32_t* budget;
  int n_sink, n_local, r, D;
  int32_t* sel_pages;
  int32_t* sel_count;
};

// Sum over the workgroup of x; every thread receives it.
__device__ __forceinline__ int block_sum(int x, int* sh) {
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) x += __shfl_xor(x, s, kWave);
  __syncthreads();
  if (lane_id() == 0) sh[threadIdx.x >> 6] = x;
  __syncthreads();
  int t = 0;
#pragma unroll
  for (int w = 0; w < kWaves; w++) t += sh[w];
  return t;
}

// One row and KV head a workgroup.
__global__ __launch_bounds__(kThreads) void select_kernel(const ChunkArgs a, const SelectArgs s) {
  extern __shared__ uint32_t keys[];
  __shared__ double qbar[128];
  __shared__ int sh[kWaves];
  __shared__ int hist[256];
  const int tid = (int)threadIdx.x, h = (int)blockIdx.x % a.H;
  Tile t;
  if (!find_tile(a, (int)blockIdx.x / a.H, t)) return;
  const int64_t row = t.row0;
  const int nb = t.p0 < 0 ? 0 : min(min((t.p0 >> a.bs_shift) + 1, (t.len + a.bs - 1) >> a.bs_shift), a.max_blocks);
  if (tid < s.D) {
    double sum = 0.0;
    for (int r = 0; r < a.g; r++) sum += (double)bf16_to_f32(a.q[row * a.q_row + (int64_t)(h * a.g + r) * a.q_head + tid]);
    qbar[tid] = sum / a.g;
  }
  __syncthreads();
  const int forced = min(nb, s.n_sink + s.n_local), total = min(max(s.budget[t.i], 0), a.max_sel);
  const int c0 = min(s.n_sink, nb), c1 = max(nb - s.n_local, c0);         // candidates
  const bool all = total >= nb;
  const int want = all ? c1 - c0 : min(max(total - forced, 0), c1 - c0);
  uint32_t T = 0;                                                          // candidates with a larger key are in,
  int ties = 0;                                                            // and this many of its own
  if (all) {
    ties = c1 - c0;
    for (int j = c0 + tid; j < c1; j += kThreads) keys[j] = 0;
  } else if (want > 0) {
    for (int j = c0 + tid; j < c1; j += kThreads) {
      const float* m = s.mean + (block_row(t.pages, j, s.r, a.num_phys) * a.H + h) * s.D;
      double dot = 0.0;
      for (int c = 0; c < s.D; c++) dot = fma(qbar[c], (double)m[c], dot);
      keys[j] = float_key((float)dot);
    }
    ties = want;
    for (int shift = 24; shift >= 0; shift -= 8) {
      hist[tid] = 0;
      __syncthreads();
      const uint32_t above = shift == 24 ? 0u : ~0u << (shift + 8);
      for (int j = c0 + tid; j < c1; j += kThreads)
        if ((keys[j] & above) == T) atomicAdd(&hist[(keys[j] >> shift) & 255], 1);
      __syncthreads();
      int d = 255, left = ties;
      for (; d > 0 && hist[d] < left; d--) left -= hist[d];
      T |= (uint32_t)d << shift;
      ties = left;
      __syncthreads();
    }
  }
  __syncthreads();
  // the list, ascending: 256 blocks at a time
  int32_t* sel = s.sel_pages + (row * a.H + h) * a.max_sel;
  int at = 0, equal = 0;
  for (int j0 = 0; j0 < nb; j0 += kThreads) {
    const int j = j0 + tid;
    const bool cand = j >= c0 && j < c1 && (all || want > 0), must = j < nb && (j < s.n_sink || j >= nb - s.n_local);
    const bool tie = cand && !must && keys[j] == T;
    // ties before this thread's, by ballots
    int wt;
    const int tb = wave_excl_count(tie, &wt);
    __syncthreads();
    if (lane_id() == 0) sh[tid >> 6] = wt;
    __syncthreads();
    int before = equal + tb;
    for (int w = 0; w < kWaves; w++) {
      if (w < (tid >> 6)) before += sh[w];
      equal += sh[w];
    }
    const bool take = must || (cand && (keys[j] > T || (tie && before < ties)));
    const int b = wave_excl_count(take, &wt);
    __syncthreads();
    if (lane_id() == 0) sh[tid >> 6] = wt;
    __syncthreads();
    int place = at + b;
    for (int w = 0; w < kWaves; w++) {
      if (w < (tid >> 6)) place += sh[w];
      at += sh[w];
    }
    if (take && place < a.max_sel) sel[place] = j;
  }
  for (int x = at + tid; x < a.max_sel; x += kThreads) sel[x] = -1;
  if (h == 0 && tid == 0) s.sel_count[row] = at;
}

}  // namespace

size_t chunk_select_workspace(const Geometry& g, int n, int Hq) { return 16; }

hipError_t launch_chunk_select(const Geometry& g, const ChunkRows& rows, const float* mean, const uint16_t* mean_bf,
                               const int32_t* budget, int n_sink, int n_local, int max_sel, int32_t* sel_pages,
                               int32_t* sel_count, void* ws, hipStream_t stream) {
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
  a.tokens = 1;
  SelectArgs s{mean, budget, n_sink, n_local, g.r, g.Dqk, sel_pages, sel_count};
  const int64_t tiles = (int64_t)rows.n + g.batch;
  hipLaunchKernelGGL(select_kernel, dim3((unsigned)(tiles * g.H)), dim3(kThreads), sizeof(uint32_t) * (size_t)a.max_blocks,
                     stream, a, s);
  return hipGetLastError();
}

}  // namespace vx
