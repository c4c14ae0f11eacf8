// What the split kernels share: their arguments, the request order by selection count, the merge of a
// split pair's partials and the agent-coherent accesses that carry them.
#pragma once
#include <climits>

#include "vx_device.h"
#include "vx_internal.h"

namespace vx {
namespace dec {

constexpr int kMergeBatch = 8;            // split partials a merge thread loads per round trip

struct DecodeArgs {
  const uint16_t* q;
  const void* k;              // bf16, or fp8 codes
  const void* v;
  const int32_t* indptr;
  const int32_t* indices;
  const int32_t* seq_lens;
  const int32_t* sel_pages;
  const int32_t* sel_count;
  uint16_t* out;
  float* part_o;
  float* part_lse;
  int max_sel, H, g, Hq, ps, num_phys;
  int bs, r;                  // selection unit: blocks of bs tokens, r per page (r = 1: pages)
  int S;                      // workgroups per pair (GQA: most splits of a pair)
  int T;                      // GQA: selection slots per split
  uint32_t* ctr;              // [pairs] split counters, zero between calls (GQA)
  float scale_log2;           // sm_scale * log2(e), times the K scale of an fp8 cache
  float v_scale;              // V scale of an fp8 cache (1 for bf16)
  int order_block;            // GQA, one workgroup per pair: > 0 orders the requests by selection
                              // count (balanced_request) with blocks of this many; 0 keeps them
};

// Every argument into SGPRs at once: one scalar round trip at the kernel's start, where the
// compiler would otherwise load the arguments in batches at their first uses, each behind a
// wait for the one before.
__device__ __forceinline__ void load_args(const DecodeArgs& a) {
  asm volatile("" ::"s"(a.q), "s"(a.k), "s"(a.v), "s"(a.indptr), "s"(a.indices), "s"(a.seq_lens), "s"(a.sel_pages),
               "s"(a.sel_count), "s"(a.out), "s"(a.part_o), "s"(a.part_lse), "s"(a.ctr));
  asm volatile("" ::"s"(a.max_sel), "s"(a.H), "s"(a.g), "s"(a.Hq), "s"(a.ps), "s"(a.num_phys), "s"(a.bs), "s"(a.r),
               "s"(a.S), "s"(a.T), "s"(a.scale_log2), "s"(a.v_scale), "s"(a.order_block));
}

// ------------------------------------------------------------------------------------
// request order by selection count (one workgroup per pair)
// ------------------------------------------------------------------------------------
// The dispatcher places a grid's workgroups one per CU in turn, so with H pairs per request the
// requests whose workgroups share a CU sit C = CUs / H positions apart in the grid.  With skewed
// selection counts (lognormal contexts) a CU that draws several long requests ends last.  The
// workgroup at request position ui serves instead the request of rank snake(ui) when the requests
// are ranked by count (descending; equal counts keep their own order, so equal counts change
// nothing): snake reverses every other block of C positions, so each CU pairs long requests with
// short ones.
constexpr int kBalanceMaxBatch = 1024;

__device__ __forceinline__ int snake_pos(int i, int C, int B) {
  const int m = i / C, j = i - m * C, n = min(C, B - m * C);
  return m * C + ((m & 1) ? n - 1 - j : j);
}

// B <= kBalanceMaxBatch requests.  Ranks by the key (count << 16) | (0xffff - snake_pos(i)): keys
// are distinct, so the ranks are a permutation, and with equal counts rank(i) = snake_pos(i) and
// every workgroup keeps its request.  Uniform over the workgroup (two barriers).
__device__ __forceinline__ int balanced_request(const DecodeArgs& a, int ui, int B) {
  __shared__ uint32_t key[kBalanceMaxBatch];
  __shared__ int target;
  const int C = a.order_block, nt = (int)blockDim.x;
  for (int i = (int)threadIdx.x; i < B; i += nt) {
    const uint32_t c = (uint32_t)min(max(a.sel_count[i], 0), 0xffff);
    key[i] = (c << 16) | (uint32_t)(0xffff - snake_pos(i, C, B));
  }
  __syncthreads();
  const int want = snake_pos(ui, C, B);
  for (int i = (int)threadIdx.x; i < B; i += nt) {
    const uint32_t k = key[i];
    int r = 0;
    for (int x = 0; x < B; x++) r += key[x] > k;
    if (r == want) target = i;
  }
  __syncthreads();
  return target;
}

// ------------------------------------------------------------------------------------
// merge of a split pair (LSE-weighted combination of its S partials)
// ------------------------------------------------------------------------------------
// Output channels 4x .. 4x+3 of pair `pair` from its first S partials (rows pair*Smax + s):
// online LSE combine over batches of kMergeBatch splits, every load of a batch issued before
// any is used (slots past S re-read the last split and weigh zero).  A split that saw no token
// has lse = -inf and an unwritten partial, which is never read into the sum.  lse_at(u) and
// o_at(u) load the log2-sum-exp and the 4 channels of partial row u (offset (u*g + c)*Dv + d).
template <class LseAt, class OAt>
__device__ __forceinline__ void merge_one(int S, int Smax, int H, int g, int Hq, int Dv, uint16_t* out, int pair,
                                          int x, LseAt lse_at, OAt o_at) {
  const int i = pair / H, h = pair - i * H;
  const int c = (4 * x) / Dv, d = 4 * x - c * Dv;
  const int64_t first = (int64_t)pair * Smax;
  float mx = -INFINITY, wsum = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s0 = 0; s0 < S; s0 += kMergeBatch) {
    float l[kMergeBatch];
    float4 p[kMergeBatch];
#pragma unroll
    for (int b = 0; b < kMergeBatch; b++) {
      const int64_t u = first + min(s0 + b, S - 1);
      l[b] = lse_at(u * g + c);
      p[b] = o_at((u * g + c) * Dv + d);
    }
    float bm = -INFINITY;
#pragma unroll
    for (int b = 0; b < kMergeBatch; b++) {
      if (s0 + b >= S) l[b] = -INFINITY;
      bm = fmaxf(bm, l[b]);
    }
    const float m_new = fmaxf(mx, bm);
    if (m_new == -INFINITY) continue;                       // no tokens so far
    const float scale = exp2f(mx - m_new);                  // 0 while mx is -inf
    wsum *= scale;
    o.x *= scale;
    o.y *= scale;
    o.z *= scale;
    o.w *= scale;
#pragma unroll
    for (int b = 0; b < kMergeBatch; b++) {
      if (l[b] == -INFINITY) continue;
      const float wgt = exp2f(l[b] - m_new);
      wsum += wgt;
      o.x += wgt * p[b].x;
      o.y += wgt * p[b].y;
      o.z += wgt * p[b].z;
      o.w += wgt * p[b].w;
    }
    mx = m_new;
  }
  if (wsum > 0.f) {
    const float inv = 1.f / wsum;
    o.x *= inv;
    o.y *= inv;
    o.z *= inv;
    o.w *= inv;
  }
  uint16_t* dst = out + ((int64_t)i * Hq + (int64_t)h * g) * Dv;
  *reinterpret_cast<uint2*>(dst + c * Dv + d) = make_uint2(f32_to_bf16_rne(o.x) | (f32_to_bf16_rne(o.y) << 16),
                                                           f32_to_bf16_rne(o.z) | (f32_to_bf16_rne(o.w) << 16));
}

// ---- agent-coherent partials -------------------------------------------------------------
// Buffer loads and stores with the sc1 cache policy are coherent across the XCDs' L2 caches
// (the form the compiler gives agent-scope atomic loads and stores): a store writes through
// to memory, a load does not return a line another XCD may have changed.  Raw buffer accesses
// are also bounds-checked against the resource's byte count.
constexpr int kAgentCoherent = 16;                 // cache policy bits: sc1
typedef unsigned int u32x4v_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ __amdgpu_buffer_rsrc_t coherent_rsrc(const void* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00020000);
}
__device__ __forceinline__ void coherent_store4(__amdgpu_buffer_rsrc_t r, uint32_t byte_off, float4 v) {
  const u32x4v_t w = {__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w)};
  __builtin_amdgcn_raw_buffer_store_b128(w, r, (int)byte_off, 0, kAgentCoherent);
}
__device__ __forceinline__ void coherent_store1(__amdgpu_buffer_rsrc_t r, uint32_t byte_off, float v) {
  __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), r, (int)byte_off, 0, kAgentCoherent);
}
__device__ __forceinline__ float4 coherent_load4(__amdgpu_buffer_rsrc_t r, uint32_t byte_off) {
  const u32x4v_t w = __builtin_amdgcn_raw_buffer_load_b128(r, (int)byte_off, 0, kAgentCoherent);
  return make_float4(__uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z), __uint_as_float(w.w));
}
__device__ __forceinline__ float coherent_load1(__amdgpu_buffer_rsrc_t r, uint32_t byte_off) {
  return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, (int)byte_off, 0, kAgentCoherent));
}
// Wait until this wave's vector-memory operations (the partial stores) have completed.
__device__ __forceinline__ void wait_vm_all() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// ------------------------------------------------------------------------------------
// the GQA work plan
// ------------------------------------------------------------------------------------
// A pair with selection count cnt has ceil(cnt / T) splits of at most T slots (one split when
// cnt = 0, which writes zeros).  T is fixed on the host, so a split's slot range is known before
// the count is.
__device__ __forceinline__ int splits_of(int cnt, int T) { return cnt > 0 ? (cnt + T - 1) / T : 1; }

}  // namespace dec

// The mxfp4 split kernel (decode_mx.hip), workgroups of four waves.
void launch_decode_mx(const dec::DecodeArgs& a, int D, unsigned grid, hipStream_t stream);

}  // namespace vx
