// Attention of a chunk's tokens over the paged cache: all of it (vx_chunk_attention), or the blocks listed for
// each token (vx_sparse_chunk_attention).
//
// chunk_rows_kernel takes the rows of a tile one by one, with each token's dot product in one lane.
#include <algorithm>
#include <cmath>

#include "chunk_common.h"

namespace vx {
using namespace chunk;
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kTileRows = 16;              // query rows (token, head of the group) of a tile

// The blocks listed for the tile's tokens: masks[id] holds a bit for each token that lists block id, ids the
// listed ones in ascending order.  Returns their count.  Every thread of the workgroup takes part.
__device__ __forceinline__ int listed_blocks(const ChunkArgs& a, const Tile& t, int h, uint32_t* words, uint16_t* ids) {
  __shared__ int wave_total[kWaves];
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

template <int D, int DV, int KT, bool SPARSE>
__global__ __launch_bounds__(kThreads) void chunk_rows_kernel(const ChunkArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
  const int h = (int)blockIdx.x % a.H;
  Tile t;
  if (!find_tile(a, (int)blockIdx.x / a.H, t)) return;
  Runs runs;
  if constexpr (SPARSE) {
    uint16_t* ids = reinterpret_cast<uint16_t*>(lds + (a.max_blocks + 1) / 2);
    runs.lo = 0;
    runs.hi = listed_blocks(a, t, h, lds, ids);
    runs.ids = ids;
    runs.masks = reinterpret_cast<const uint16_t*>(lds);
    runs.shift = a.bs_shift;
  } else {
    runs.lo = first_key(a, t.p0) >> 6;
    runs.hi = (end_key(a, t, t.p0 + t.n - 1) + 63) >> 6;
    runs.ids = nullptr;
    runs.masks = nullptr;
    runs.shift = 6;
  }
  for (int x = (int)threadIdx.x >> 6; x < t.n * a.g; x += kWaves) {
    RowState<DV> st;
    attend_row<D, DV, KT>(a, t, h, x % a.g, x / a.g, runs, st);
    store_row<DV>(a, t.row0 + x / a.g, h * a.g + x % a.g, 0, st);
  }
}

template <int D, int DV, int KT>
hipError_t launch_kt(const ChunkArgs& a, hipStream_t stream) {
  const int64_t tiles = (int64_t)a.num_rows / a.tokens + a.batch;
  const dim3 grid((unsigned)(tiles * a.H));
  if constexpr (D == DV) {
    if (a.sel_pages) {
      const size_t lds = sizeof(uint32_t) * ((a.max_blocks + 1) / 2) + sizeof(uint16_t) * a.max_blocks;
      hipLaunchKernelGGL((chunk_rows_kernel<D, DV, KT, true>), grid, dim3(kThreads), lds, stream, a);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((chunk_rows_kernel<D, DV, KT, false>), grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

template <int D, int DV>
hipError_t launch_d(const ChunkArgs& a, int kt, hipStream_t stream) {
  if (kt == kKvFp8E4M3) return launch_kt<D, DV, kKvFp8E4M3>(a, stream);
  if (kt == kKvFp8E5M2) return launch_kt<D, DV, kKvFp8E5M2>(a, stream);
  if constexpr (D == DV) {
    if (kt == kKvMxFp4) return launch_kt<D, DV, kKvMxFp4>(a, stream);
  }
  return launch_kt<D, DV, kKvBf16>(a, stream);
}

}  // namespace

size_t chunk_attention_workspace(const Geometry& g, int n, int Hq, bool sparse, int max_sel) { return 16; }

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
  a.tokens = kTileRows / a.g;
  a.splits = 1;
  if (g.Dqk == 128) return launch_d<128, 128>(a, g.kv_dtype, stream);
  if (g.Dqk == 64) return launch_d<64, 64>(a, g.kv_dtype, stream);
  return launch_d<576, 512>(a, g.kv_dtype, stream);
}

}  // namespace vx
