// Pages, block table and slot map of growing requests, built on the device (Sec. 4.1, C = (b, p, I)).
//
// extend  with L the row's tokens, n the new ones, need = ceil((L + n) / ps) - ceil(L / ps) and c the
//         free pages: a request is granted its tokens when its row has room and need = 0 or the needs
//         up to it sum to at most c.  The sums never fall, so the granted needs are those of the first
//         requests that need pages, and the pages taken before request i are the sum S of the needs
//         before it while S <= c, else the largest sum <= c.  Sums of (need, held, new) over the
//         requests before i therefore place its list, its tokens and its pages on the stack.
// release the pages past the kept tokens go back in the reverse order, so that a release takes an
//         extend back exactly.
// Each call is one launch, bound by the latency of its dependent reads: request, length, place on the
// stack, page.  Every workgroup sums all the requests itself (12 bytes each, from L2), places a range
// of at most kPlanRange of them and moves their pages.  The lengths and the free count, which every
// workgroup reads, change only after the last one has read them: a counter in the workspace tells,
// and that last workgroup writes them.  Extend and release, 64 requests of 8192 to 32768 tokens: 6.8 and
// 5.2 us (with the sums in a launch of one workgroup before the move 9.0 and 4.2 us, and two more
// launches of 2.4 us each for the host); 4096 requests, 2 million page entries and 1.2 million slots:
// 27 and 15 us (74 and 21 us; with four times the workgroups 70 and 21, since each sums all requests).
// Whole requests admitted and ended: 64 of 1.2 million tokens 19 us for both calls (12 without slots), 4096 of 37
// million tokens, 2.3 million pages, 151 us (41 without slots): a slot's page is loaded and waited for turn by turn.
#include <algorithm>
#include <climits>

#include "vx_device.h"
#include "vx_internal.h"

namespace vx {
namespace {

constexpr int kPlanThreads = 512;
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kPlanRanges = 256;      // ranges of requests (one per CU)
constexpr int kPlanRange = 256;       // most requests of a range: a batch has at most 65535
constexpr int kPlanWgs = 256;        // most workgroups
constexpr int kLaneAsks = kPlanRange / kWave;
constexpr int kLanePages = 4;         // pages (or tokens) a lane moves per turn
constexpr int kTurn = kWave * kLanePages;

struct ExtendArgs {
  PagePool pool;
  int batch, range;                   // requests, and those of a range
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
  uint32_t* ctr;
};

struct ReleaseArgs {
  PagePool pool;
  int batch, range;
  const int32_t* rows;
  const int32_t* keep_lens;
  uint32_t* ctr;
};

// Pages of 2^shift tokens (a division costs as much as all the rest of a request).
__device__ __forceinline__ int64_t pages_of(int64_t tokens, int shift) {
  return (tokens + ((int64_t)1 << shift) - 1) >> shift;
}

// What request j asks for.  row -1: outside the table.
struct Ask {
  int row, L, n, held;
  int64_t need;
  bool fits;
};
// Its row, -1 outside the table or past the batch; loads unconditional, so that several requests' can
// be in flight.
__device__ __forceinline__ int row_of(const int32_t* rows, int batch, const PagePool& P, int j) {
  const int row = rows[min(j, batch - 1)];
  return j < batch && row >= 0 && row < P.table_rows ? row : -1;
}
__device__ __forceinline__ Ask ask_with(const PagePool& P, int row, int len, int n) {
  Ask q{row, row >= 0 ? max(len, 0) : 0, max(n, 0), 0, 0, false};
  q.held = (int)min(pages_of(q.L, P.ps_shift), (int64_t)P.table_stride);
  const int64_t want = pages_of((int64_t)q.L + q.n, P.ps_shift);
  q.fits = q.row >= 0 && want <= P.table_stride;
  q.need = q.fits ? want - q.held : 0;
  return q;
}
__device__ __forceinline__ Ask ask_of(const ExtendArgs& a, int j) {
  const int row = row_of(a.rows, a.batch, a.pool, j);
  const int n = a.new_lens[min(j, a.batch - 1)];
  return ask_with(a.pool, row, a.pool.lens[max(row, 0)], j < a.batch ? n : 0);
}

constexpr int kAsks = 4;              // requests a thread reads per round trip

// f(j, ask) for this thread's share of all requests.
template <class F>
__device__ __forceinline__ void each_ask(const ExtendArgs& a, F f) {
  for (int j0 = (int)threadIdx.x; j0 < a.batch; j0 += kAsks * kPlanThreads) {
    int row[kAsks], n[kAsks], len[kAsks];
#pragma unroll
    for (int b = 0; b < kAsks; b++) {
      const int j = j0 + b * kPlanThreads;
      row[b] = row_of(a.rows, a.batch, a.pool, j);
      n[b] = a.new_lens[min(j, a.batch - 1)];
      if (j >= a.batch) n[b] = 0;
    }
#pragma unroll
    for (int b = 0; b < kAsks; b++) len[b] = a.pool.lens[max(row[b], 0)];
#pragma unroll
    for (int b = 0; b < kAsks; b++) f(j0 + b * kPlanThreads, ask_with(a.pool, row[b], len[b], n[b]));
  }
}

// Pages that request j gives back: [first, last) of its row.
struct Back {
  int row, keep, first, last;
};
__device__ __forceinline__ Back back_with(const PagePool& P, int row, int len, int keep) {
  const int L = row >= 0 ? max(len, 0) : 0;
  Back q{row, min(max(keep, 0), L), 0, 0};
  q.last = (int)min(pages_of(L, P.ps_shift), (int64_t)P.table_stride);
  q.first = min((int)pages_of(q.keep, P.ps_shift), q.last);
  return q;
}
template <class F>
__device__ __forceinline__ void each_back(const ReleaseArgs& a, F f) {
  for (int j0 = (int)threadIdx.x; j0 < a.batch; j0 += kAsks * kPlanThreads) {
    int row[kAsks], keep[kAsks], len[kAsks];
#pragma unroll
    for (int b = 0; b < kAsks; b++) {
      const int j = j0 + b * kPlanThreads;
      row[b] = row_of(a.rows, a.batch, a.pool, j);
      keep[b] = a.keep_lens ? a.keep_lens[min(j, a.batch - 1)] : 0;
    }
#pragma unroll
    for (int b = 0; b < kAsks; b++) len[b] = a.pool.lens[max(row[b], 0)];
#pragma unroll
    for (int b = 0; b < kAsks; b++) f(j0 + b * kPlanThreads, back_with(a.pool, row[b], len[b], keep[b]));
  }
}

// Inclusive sums over the wave's lanes (DPP row shifts, then the rows' ends to the rows above).
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t dpp_add(int64_t x) {
  const int lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)((uint64_t)x >> 32), CTRL, ROWS, 0xf, false);
  return x + (int64_t)(((uint64_t)(uint32_t)hi << 32) | (uint32_t)lo);
}
__device__ __forceinline__ int64_t wave_scan(int64_t x) {
  x = dpp_add<0x111, 0xf>(x);         // row_shr 1, 2, 4, 8
  x = dpp_add<0x112, 0xf>(x);
  x = dpp_add<0x114, 0xf>(x);
  x = dpp_add<0x118, 0xf>(x);
  x = dpp_add<0x142, 0xa>(x);         // row_bcast 15 into rows 1 and 3
  return dpp_add<0x143, 0xc>(x);      // row_bcast 31 into rows 2 and 3
}

// The waves' sums of N values, in LDS; a barrier, then group_total.
template <int N>
using WaveSums = int64_t[N][kPlanWaves];
template <int N>
__device__ __forceinline__ void put_wave_sums(const int64_t (&x)[N], WaveSums<N>& lds) {
#pragma unroll
  for (int v = 0; v < N; v++) {
    const int64_t y = wave_scan(x[v]);
    if (lane_id() == kWave - 1) lds[v][threadIdx.x >> 6] = y;
  }
}
template <int N>
__device__ __forceinline__ void group_total(int64_t (&x)[N], const WaveSums<N>& lds) {
#pragma unroll
  for (int v = 0; v < N; v++) {
    x[v] = 0;
#pragma unroll
    for (int k = 0; k < kPlanWaves; k++) x[v] += lds[v][k];
  }
}

// The needs in order, when they sum to more than the c free pages: the largest sum <= c, and the sum
// before request r0.  COMMIT writes the granted lengths on the way.  Every thread of the workgroup.
struct ShortLds {
  WaveSums<1> sums;
  int64_t taken, before;
};
template <bool COMMIT>
__device__ __forceinline__ void short_pool(const ExtendArgs& a, int64_t c, int r0, ShortLds& lds, int64_t& taken,
                                           int64_t& before_r0) {
  int64_t carry = 0;
  if (threadIdx.x == 0) lds.taken = 0;
  for (int j0 = 0; j0 < a.batch; j0 += kPlanThreads) {
    const int j = j0 + (int)threadIdx.x, w = (int)threadIdx.x >> 6;
    const Ask q = ask_of(a, j);
    const int64_t mine = wave_scan(q.need);
    __syncthreads();
    if (lane_id() == kWave - 1) lds.sums[0][w] = mine;
    __syncthreads();
    int64_t cum = carry + mine;
    for (int k = 0; k < kPlanWaves; k++) {
      if (k < w) cum += lds.sums[0][k];
      carry += lds.sums[0][k];
    }
    const uint64_t below = __ballot(cum <= c);             // the wave's first lanes: the sums never fall
    if (below != 0 && lane_id() == 63 - __clzll(below))
      atomicMax(reinterpret_cast<unsigned long long*>(&lds.taken), (unsigned long long)cum);
    if (COMMIT && q.fits && (q.need == 0 || cum <= c)) a.pool.lens[q.row] = q.L + q.n;
    if (j == r0) lds.before = cum - q.need;
  }
  __syncthreads();
  taken = lds.taken;
  before_r0 = lds.before;
  __syncthreads();
}

// A request of the workgroup's range, placed.
struct Placed {
  int row, L, n, now, base;           // base: pages taken before it, -1 when refused
  int64_t start, token;               // its page list's and its tokens' first entries
};

// A thread's loads have arrived: ahead of the barrier behind which arrive() says so.
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }

// Whether this workgroup is the last of the launch to get here; the counter wraps back to zero.  One
// thread, behind a barrier that every thread has reached with its loads (wait_loads).
__device__ __forceinline__ uint32_t arrive(uint32_t* ctr) {
  const uint32_t wgs = gridDim.x * gridDim.y;
  return __builtin_amdgcn_atomic_inc32(ctr, wgs - 1, __ATOMIC_RELAXED, "agent") == wgs - 1;
}

// Grid (pieces, ranges): the pieces of a range share out its pages and tokens.
__global__ __launch_bounds__(kPlanThreads) void extend_kernel(const ExtendArgs a) {
  __shared__ WaveSums<5> sums;
  __shared__ ShortLds short_lds;
  __shared__ Ask asks[kPlanRange];
  __shared__ Placed placed[kPlanRange];
  __shared__ uint32_t last;
  const PagePool& P = a.pool;
  const int tid = (int)threadIdx.x;
  const int r0 = (int)blockIdx.y * a.range, nr = min(a.range, a.batch - r0);
  const int piece = (int)blockIdx.x, pieces = (int)gridDim.x;
  const int64_t c = min(max(*P.free_count, 0), P.num_phys);

  int64_t s[5] = {0, 0, 0, 0, 0};     // needs, new tokens; before the range: needs, held, new
  each_ask(a, [&](int j, const Ask& q) {
    s[0] += q.need;
    s[1] += q.n;
    if (j < r0) {
      s[2] += q.need;
      s[3] += q.held;
      s[4] += q.n;
    } else if (j < r0 + nr) {
      asks[j - r0] = q;
    }
  });
  put_wave_sums<5>(s, sums);
  wait_loads();
  __syncthreads();
  group_total<5>(s, sums);
  const bool shortage = s[0] > c;     // uniform
  int64_t taken = s[0], before_r0 = s[2];
  if (shortage) short_pool<false>(a, c, r0, short_lds, taken, before_r0);
  // no more reads of the lengths or the free count from here
  if (tid == 0) last = arrive(a.ctr);

  // the first wave places the range, kLaneAsks consecutive requests a lane
  if (tid < kWave) {
    Ask q[kLaneAsks];
    int64_t need = 0, held = 0, n = 0;
#pragma unroll
    for (int b = 0; b < kLaneAsks; b++) {
      const int k = tid * kLaneAsks + b;
      if (k < nr) q[b] = asks[k];
      else q[b] = Ask{-1, 0, 0, 0, 0, false};
      need += q[b].need;
      held += q[b].held;
      n += q[b].n;
    }
    int64_t cum = before_r0 + wave_scan(need) - need;
    int64_t lists = s[3] + wave_scan(held) - held, token = s[4] + wave_scan(n) - n;
    auto granted_before = [&](int64_t sum) { return sum <= c ? sum : taken; };
#pragma unroll
    for (int b = 0; b < kLaneAsks; b++) {
      const int k = tid * kLaneAsks + b, i = r0 + k;
      if (k >= nr) break;
      const int64_t before = cum;
      cum += q[b].need;
      const bool ok = q[b].fits && (q[b].need == 0 || cum <= c);
      const int got = ok ? q[b].n : 0;
      const Placed p{q[b].row, q[b].L, q[b].n, q[b].L + got, ok ? (int)before : -1, lists + granted_before(before), token};
      placed[k] = p;
      lists += q[b].held;
      token += q[b].n;
      if (piece != 0) continue;
      a.page_indptr[i] = (int)min(p.start, (int64_t)a.page_cap);
      a.token_indptr[i] = (int)min(p.token, (int64_t)INT_MAX);
      a.seq_lens[i] = p.now;
      a.granted[i] = got;
      if (a.first_block) a.first_block[i] = q[b].L >> P.bs_shift;
      if (i == a.batch - 1) {
        a.page_indptr[a.batch] = (int)min(lists + granted_before(cum), (int64_t)a.page_cap);
        a.token_indptr[a.batch] = (int)min(token, (int64_t)INT_MAX);
      }
    }
  }
  __syncthreads();

  // Turn t of request k belongs to wave (t + k) mod the range's waves: long requests spread over all
  // of them, and so do many short ones.
  const int waves = pieces * kPlanWaves, me = piece * kPlanWaves + __builtin_amdgcn_readfirstlane(tid >> 6);
  for (int k = 0, t0 = me; k < nr; k++, t0 = t0 == 0 ? waves - 1 : t0 - 1) {
    const Placed p = placed[k];
    if (p.row < 0) continue;
    int32_t* list = P.table + (int64_t)p.row * P.table_stride;
    const int held = (int)min(pages_of(p.L, P.ps_shift), (int64_t)P.table_stride);
    const int pages = (int)min(pages_of(p.now, P.ps_shift), (int64_t)P.table_stride);
    const int32_t* top = P.free_pages + (c - 1 - p.base + held);   // page x >= held is top[-x]
    for (int64_t x0 = (int64_t)t0 * kTurn; x0 < pages; x0 += (int64_t)waves * kTurn) {
      int page[kLanePages];
#pragma unroll
      for (int b = 0; b < kLanePages; b++) {
        const int x = min((int)x0 + kWave * b + lane_id(), pages - 1);   // no branch: one round trip for all
        page[b] = *(x < held ? list + x : top - x);
      }
#pragma unroll
      for (int b = 0; b < kLanePages; b++) {
        const int x = (int)x0 + kWave * b + lane_id();
        if (x >= pages) continue;
        if (p.start + x < a.page_cap) a.page_indices[p.start + x] = page[b];
        if (x >= held) list[x] = page[b];
      }
    }
  }
  for (int k = 0, t0 = me; k < nr; k++, t0 = t0 == 0 ? waves - 1 : t0 - 1) {
    const Placed p = placed[k];
    const int64_t end = min(p.token + p.n, (int64_t)a.slot_cap);
    const int32_t* list = P.table + (int64_t)max(p.row, 0) * P.table_stride;
    const int held = (int)min(pages_of(p.L, P.ps_shift), (int64_t)P.table_stride);
    const int32_t* top = P.free_pages + (c - 1 - p.base + held);
    for (int64_t t = p.token + (int64_t)t0 * kWave + lane_id(); t < end; t += (int64_t)waves * kWave) {
      int64_t slot = -1;
      if (p.base >= 0) {
        const int pos = p.L + (int)(t - p.token), x = pos >> P.ps_shift;
        const int64_t page = *(x < held ? list + x : top - x);
        slot = page * (1 << P.ps_shift) + (pos - (x << P.ps_shift));
      }
      a.slots[t] = slot;
    }
  }
  const int64_t wg = (int64_t)blockIdx.y * pieces + piece, wgs = (int64_t)gridDim.y * pieces;
  for (int64_t t = s[1] + wg * kPlanThreads + tid; t < a.slot_cap; t += wgs * kPlanThreads) a.slots[t] = -1;

  __syncthreads();
  if (!last) return;
  if (shortage) {
    int64_t ignored;
    short_pool<true>(a, c, 0, short_lds, taken, ignored);
  } else {
    each_ask(a, [&](int, const Ask& w) {
      if (w.fits) P.lens[w.row] = w.L + w.n;
    });
  }
  if (tid == 0) *P.free_count = (int)(c - taken);
}

__global__ __launch_bounds__(kPlanThreads) void release_kernel(const ReleaseArgs a) {
  __shared__ WaveSums<2> sums;
  __shared__ Back back[kPlanRange];
  __shared__ int64_t base[kPlanRange];
  __shared__ uint32_t last;
  const PagePool& P = a.pool;
  const int tid = (int)threadIdx.x;
  const int r0 = (int)blockIdx.y * a.range, nr = min(a.range, a.batch - r0);
  const int piece = (int)blockIdx.x, pieces = (int)gridDim.x;
  const int64_t c = min(max(*P.free_count, 0), P.num_phys);
  int64_t s[2] = {0, 0};              // pages given back, in all and before the range
  each_back(a, [&](int j, const Back& q) {
    s[0] += q.last - q.first;
    if (j < r0) s[1] += q.last - q.first;
    else if (j < r0 + nr) back[j - r0] = q;
  });
  put_wave_sums<2>(s, sums);
  wait_loads();
  __syncthreads();
  group_total<2>(s, sums);
  if (tid == 0) last = arrive(a.ctr);
  if (tid < kWave) {
    int64_t sum = 0;
#pragma unroll
    for (int b = 0; b < kLaneAsks; b++) {
      const int k = tid * kLaneAsks + b;
      sum += k < nr ? back[k].last - back[k].first : 0;
    }
    int64_t at = s[1] + wave_scan(sum) - sum;
#pragma unroll
    for (int b = 0; b < kLaneAsks; b++) {
      const int k = tid * kLaneAsks + b;
      if (k >= nr) break;
      base[k] = at;
      at += back[k].last - back[k].first;
    }
  }
  __syncthreads();
  // a stack that is full (pages given back twice) drops the pages that do not fit
  const int64_t all = min(s[0], (int64_t)P.num_phys);
  const int waves = pieces * kPlanWaves, me = piece * kPlanWaves + __builtin_amdgcn_readfirstlane(tid >> 6);
  for (int k = 0, t0 = me; k < nr; k++, t0 = t0 == 0 ? waves - 1 : t0 - 1) {
    const Back b = back[k];
    const int32_t* list = P.table + (int64_t)max(b.row, 0) * P.table_stride;
    for (int64_t y = b.first + (int64_t)t0 * kWave + lane_id(); y < b.last;
         y += (int64_t)waves * kWave) {
      const int64_t at = c + all - 1 - (base[k] + y - b.first);
      if (at >= 0 && at < P.num_phys) P.free_pages[at] = list[y];
    }
  }
  __syncthreads();
  if (!last) return;
  each_back(a, [&](int, const Back& w) {
    if (w.row >= 0) P.lens[w.row] = w.keep;
  });
  if (tid == 0) *P.free_count = (int)min(c + all, (int64_t)P.num_phys);
}

// Requests of a range, and the grid: a piece per `per` entries that a range's waves move.
int range_of(int batch) { return (batch + kPlanRanges - 1) / kPlanRanges; }
dim3 plan_grid(int batch, int range, int64_t entries) {
  const int ranges = (batch + range - 1) / range;
  const int64_t per = kPlanWaves * kTurn;
  const int64_t pieces = std::min<int64_t>(std::max<int64_t>((entries + per - 1) / per, 1), std::max(kPlanWgs / ranges, 1));
  return dim3((unsigned)pieces, (unsigned)ranges);
}

}  // namespace

size_t plan_workspace_bytes(int) { return 256; }

hipError_t launch_page_extend(const PagePool& pool, int batch, const int32_t* rows, const int32_t* new_lens,
                              int32_t* seq_lens, int32_t* page_indptr, int32_t* page_indices, int page_cap,
                              int32_t* token_indptr, int64_t* slots, int slot_cap, int32_t* granted,
                              int32_t* first_block, void* ws, hipStream_t stream) {
  if (batch == 0) return hipSuccess;
  const int range = range_of(batch), ranges = (batch + range - 1) / range;
  const ExtendArgs a{pool, batch, range, rows, new_lens, seq_lens, page_indptr, page_indices, page_cap,
                     token_indptr, slots, slot_cap, granted, first_block, static_cast<uint32_t*>(ws)};
  const int64_t entries = std::max<int64_t>((int64_t)pool.table_stride * range, slot_cap / ranges);
  hipLaunchKernelGGL(extend_kernel, plan_grid(batch, range, entries), dim3(kPlanThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_page_release(const PagePool& pool, int batch, const int32_t* rows, const int32_t* keep_lens, void* ws,
                               hipStream_t stream) {
  if (batch == 0) return hipSuccess;
  const int range = range_of(batch);
  const ReleaseArgs a{pool, batch, range, rows, keep_lens, static_cast<uint32_t*>(ws)};
  // a step's release moves few pages; whole rows take more turns
  const dim3 grid = plan_grid(batch, range, (int64_t)pool.table_stride * range / 4);
  hipLaunchKernelGGL(release_kernel, grid, dim3(kPlanThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace vx
