// Pages, block table and slot map of growing requests, built on the device (Sec. 4.1, C = (b, p, I)).
//
// extend  with L the row's tokens, n the new ones, need = ceil((L + n) / ps) - ceil(L / ps) and c the
//         free pages: a request is admitted when its row has room and need = 0 or the needs up to it
//         sum to at most c.  The sums never fall, so the admitted needs are those of the first
//         requests that need pages, and the pages taken before request i are min-like: the sum S of
//         the needs before it while S <= c, else the largest sum <= c.  One scan of (need, held,
//         new) therefore gives page_indptr, token_indptr and every page's place on the stack.
// release the pages past the kept tokens go back in the reverse order, so that a release takes an
//         extend back exactly.
// Each call is one workgroup that scans the requests and a launch that moves pages and slots, both
// bound by latency for a serving batch.
#include <climits>

#include "vx_device.h"
#include "vx_internal.h"

namespace vx {
namespace {

constexpr int kScanThreads = 1024;
constexpr int kFillThreads = 256;
constexpr int kFillPages = 1024;      // pages (or tokens) of a request per fill workgroup and round

// Workspace: {c0} then per request {old length, needs or returned pages before it}.
struct PlanWs {
  int32_t* head;      // [0] free pages before the call, [1] pages returned in all
  int32_t* old_len;
  int32_t* base;
};
__host__ __device__ inline PlanWs plan_ws(void* ws, int batch) {
  int32_t* p = static_cast<int32_t*>(ws);
  return PlanWs{p, p + 4, p + 4 + batch};
}

struct ExtendArgs {
  PagePool pool;
  int batch;
  const int32_t* rows;
  const int32_t* new_lens;
  int32_t* seq_lens;
  int32_t* page_indptr;
  int32_t* page_indices;
  int page_cap;
  int32_t* token_indptr;
  int64_t* slots;
  int slot_cap;
  int32_t* granted;
  int32_t* first_block;
  PlanWs ws;
};

struct ReleaseArgs {
  PagePool pool;
  int batch;
  const int32_t* rows;
  const int32_t* keep_lens;
  PlanWs ws;
};

__device__ __forceinline__ int64_t wave_incl_scan(int64_t x) {
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const int64_t y = __shfl_up(x, d, kWave);
    if (lane_id() >= d) x += y;
  }
  return x;
}

// Inclusive sums over the workgroup of N values per thread; total[] receives the sums.
template <int N>
__device__ __forceinline__ void group_scan(int64_t (&x)[N], int64_t (&total)[N], int64_t (*lds)[kScanThreads / kWave]) {
  const int w = (int)threadIdx.x >> 6;
#pragma unroll
  for (int v = 0; v < N; v++) {
    x[v] = wave_incl_scan(x[v]);
    if (lane_id() == kWave - 1) lds[v][w] = x[v];
  }
  __syncthreads();
#pragma unroll
  for (int v = 0; v < N; v++) {
    int64_t before = 0, all = 0;
    for (int k = 0; k < kScanThreads / kWave; k++) {
      if (k < w) before += lds[v][k];
      all += lds[v][k];
    }
    x[v] += before;
    total[v] = all;
  }
  __syncthreads();
}

__device__ __forceinline__ int64_t pages_of(int64_t tokens, int ps) { return (tokens + ps - 1) / ps; }

__global__ __launch_bounds__(kScanThreads) void extend_scan_kernel(const ExtendArgs a) {
  __shared__ int64_t lds[3][kScanThreads / kWave];
  __shared__ int64_t taken_lds;
  const PagePool& P = a.pool;
  const int64_t c = min(max(*P.free_count, 0), P.num_phys);
  const int unit = P.bs;
  int64_t carry[3] = {0, 0, 0};         // needs, held pages and new tokens of the requests before the tile
  int64_t taken = 0;                    // largest sum of needs <= c so far
  for (int i0 = 0; i0 < a.batch; i0 += kScanThreads) {
    const int i = i0 + (int)threadIdx.x;
    int row = -1, n = 0, L = 0;
    if (i < a.batch) {
      row = a.rows[i];
      n = max(a.new_lens[i], 0);
      if (row < 0 || row >= P.table_rows) row = -1;
      else L = max(P.lens[row], 0);
    }
    const int64_t held = min(pages_of(L, P.ps), (int64_t)P.table_stride);
    const int64_t want = pages_of((int64_t)L + n, P.ps);
    const bool fits = row >= 0 && want <= P.table_stride && (int64_t)L + n <= INT_MAX;
    const int64_t need = fits ? want - held : 0;
    int64_t x[3] = {need, held, n}, total[3];
    if (threadIdx.x == 0) taken_lds = taken;
    group_scan<3>(x, total, lds);
    const int64_t cum = carry[0] + x[0];
    const uint64_t below = __ballot(cum <= c);           // the wave's first lanes: the sums never fall
    if (below != 0 && lane_id() == 63 - __clzll(below))
      atomicMax(reinterpret_cast<unsigned long long*>(&taken_lds), (unsigned long long)cum);
    __syncthreads();
    taken = taken_lds;
    const int64_t before = cum - need;
    const bool ok = fits && (need == 0 || cum <= c);
    if (i < a.batch) {
      const int got = ok ? n : 0;
      const int64_t start = carry[1] + x[1] - held + (before <= c ? before : taken);
      a.page_indptr[i] = (int)min(start, (int64_t)a.page_cap);
      a.token_indptr[i] = (int)min(carry[2] + x[2] - n, (int64_t)INT_MAX);
      a.seq_lens[i] = L + got;
      a.granted[i] = got;
      if (a.first_block) a.first_block[i] = L / unit;
      a.ws.old_len[i] = L;
      a.ws.base[i] = ok ? (int)before : -1;                       // -1: refused
      if (row >= 0) P.lens[row] = L + got;
    }
#pragma unroll
    for (int v = 0; v < 3; v++) carry[v] += total[v];
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    a.page_indptr[a.batch] = (int)min(carry[1] + taken, (int64_t)a.page_cap);
    a.token_indptr[a.batch] = (int)min(carry[2], (int64_t)INT_MAX);
    a.ws.head[0] = (int)c;
    *P.free_count = (int)(c - taken);
  }
}

// Workgroups (piece, request): the request's pages into the page list and, the new ones, into its table
// row; its tokens' slots; and a share of the slots behind the last token.
__global__ __launch_bounds__(kFillThreads) void extend_fill_kernel(const ExtendArgs a) {
  const PagePool& P = a.pool;
  const int i = (int)blockIdx.y, piece = (int)blockIdx.x, pieces = (int)gridDim.x;
  const int row = a.rows[i];
  const int L = a.ws.old_len[i], base = a.ws.base[i], c0 = a.ws.head[0], now = a.seq_lens[i];
  const int start = a.page_indptr[i], end = a.page_indptr[i + 1];
  const int t0 = a.token_indptr[i], t1 = min(a.token_indptr[i + 1], a.slot_cap);
  const int tail = min(a.token_indptr[a.batch], a.slot_cap);
  const bool known = row >= 0 && row < P.table_rows;
  int32_t* list = P.table + (int64_t)(known ? row : 0) * P.table_stride;
  const int held = known ? (int)min(pages_of(L, P.ps), (int64_t)P.table_stride) : 0;
  const int pages = known ? (int)min(pages_of(now, P.ps), (int64_t)P.table_stride) : 0;
  auto page_at = [&](int x) { return x < held ? list[x] : P.free_pages[c0 - 1 - (base + x - held)]; };
  // one piece covers kFillPages pages of the row, and the pieces cover the whole row
  for (int x = piece * kFillPages + (int)threadIdx.x; x < min(pages, (piece + 1) * kFillPages); x += kFillThreads) {
    const int p = page_at(x);
    if ((int64_t)start + x < end) a.page_indices[start + x] = p;
    if (x >= held) list[x] = p;
  }
  for (int64_t t = (int64_t)t0 + piece * kFillThreads + threadIdx.x; t < t1; t += (int64_t)pieces * kFillThreads) {
    const int64_t pos = L + (t - t0);
    a.slots[t] = base >= 0 ? (int64_t)page_at((int)(pos / P.ps)) * P.ps + pos % P.ps : -1;
  }
  const int64_t wg = (int64_t)i * pieces + piece, wgs = (int64_t)a.batch * pieces;
  for (int64_t t = tail + wg * kFillThreads + threadIdx.x; t < a.slot_cap; t += wgs * kFillThreads) a.slots[t] = -1;
}

__global__ __launch_bounds__(kScanThreads) void release_scan_kernel(const ReleaseArgs a) {
  __shared__ int64_t lds[1][kScanThreads / kWave];
  const PagePool& P = a.pool;
  const int64_t c = min(max(*P.free_count, 0), P.num_phys);
  int64_t carry = 0;
  for (int i0 = 0; i0 < a.batch; i0 += kScanThreads) {
    const int i = i0 + (int)threadIdx.x;
    int row = -1, L = 0, keep = 0;
    if (i < a.batch) {
      row = a.rows[i];
      if (row < 0 || row >= P.table_rows) row = -1;
      else L = max(P.lens[row], 0);
      keep = a.keep_lens ? min(max(a.keep_lens[i], 0), L) : 0;
    }
    const int64_t back = max(min(pages_of(L, P.ps), (int64_t)P.table_stride) - pages_of(keep, P.ps), (int64_t)0);
    int64_t x[1] = {back}, total[1];
    group_scan<1>(x, total, lds);
    if (i < a.batch) {
      a.ws.old_len[i] = L;
      a.ws.base[i] = (int)min(carry + x[0] - back, (int64_t)INT_MAX);
      if (row >= 0) P.lens[row] = keep;
    }
    carry += total[0];
  }
  if (threadIdx.x == 0) {
    const int64_t all = min(carry, (int64_t)P.num_phys);
    a.ws.head[0] = (int)c;
    a.ws.head[1] = (int)all;
    *P.free_count = (int)min(c + all, (int64_t)P.num_phys);
  }
}

__global__ __launch_bounds__(kFillThreads) void release_fill_kernel(const ReleaseArgs a) {
  const PagePool& P = a.pool;
  const int i = (int)blockIdx.y;
  const int row = a.rows[i];
  if (row < 0 || row >= P.table_rows) return;
  const int L = a.ws.old_len[i], base = a.ws.base[i], c0 = a.ws.head[0], all = a.ws.head[1];
  const int keep = a.keep_lens ? min(max(a.keep_lens[i], 0), L) : 0;
  const int first = (int)pages_of(keep, P.ps), last = (int)min(pages_of(L, P.ps), (int64_t)P.table_stride);
  const int32_t* list = P.table + (int64_t)row * P.table_stride;
  for (int x = first + (int)(blockIdx.x * kFillThreads + threadIdx.x); x < last; x += (int)gridDim.x * kFillThreads) {
    const int64_t at = (int64_t)c0 + all - 1 - ((int64_t)base + x - first);
    if (at >= 0 && at < P.num_phys) P.free_pages[at] = list[x];
  }
}

// Workgroups per request: one per `per` pages of its row.
unsigned fill_pieces(int stride, int per) { return (unsigned)((stride + per - 1) / per); }

}  // namespace

size_t plan_workspace_bytes(int batch) { return sizeof(int32_t) * (4 + 2 * (size_t)batch); }

hipError_t launch_page_extend(const PagePool& pool, int batch, const int32_t* rows, const int32_t* new_lens,
                              int32_t* seq_lens, int32_t* page_indptr, int32_t* page_indices, int page_cap,
                              int32_t* token_indptr, int64_t* slots, int slot_cap, int32_t* granted,
                              int32_t* first_block, void* ws, hipStream_t stream) {
  if (batch == 0) return hipSuccess;
  const ExtendArgs a{pool, batch, rows, new_lens, seq_lens, page_indptr, page_indices, page_cap,
                     token_indptr, slots, slot_cap, granted, first_block, plan_ws(ws, batch)};
  hipLaunchKernelGGL(extend_scan_kernel, dim3(1), dim3(kScanThreads), 0, stream, a);
  const dim3 grid(fill_pieces(pool.table_stride, kFillPages), (unsigned)batch);
  hipLaunchKernelGGL(extend_fill_kernel, grid, dim3(kFillThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_page_release(const PagePool& pool, int batch, const int32_t* rows, const int32_t* keep_lens, void* ws,
                               hipStream_t stream) {
  if (batch == 0) return hipSuccess;
  const ReleaseArgs a{pool, batch, rows, keep_lens, plan_ws(ws, batch)};
  hipLaunchKernelGGL(release_scan_kernel, dim3(1), dim3(kScanThreads), 0, stream, a);
  const dim3 grid(fill_pieces(pool.table_stride, 4 * kFillPages), (unsigned)batch);
  hipLaunchKernelGGL(release_fill_kernel, grid, dim3(kFillThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace vx
