// Rows into and out of the paged cache by slot (slot = page * page_size + token in the page).
//
// vx_kv_write rounds bf16 rows to the cache's type; vx_kv_read gives the cache's values as bf16.
// A task is 8 consecutive channels of one row and head, K and V side by side.  Four consecutive rows
// of a head share a wave (16 chunks each), so that rows of consecutive slots, whose V codes of an
// mxfp4 cache interleave by four, fill whole lines together.  Bound by HBM: a row of D channels is
// 2 D bytes of bf16 and 2 D (bf16), D (fp8) or 17 D / 32 (mxfp4) bytes of cache, for K and V each.
// 100003 rows of 4 heads of 128 channels written and 50001 read, in random order: E4M3 86 us (5.3 TB/s),
// bf16 112 us (5.5), mxfp4 96 us (4.1: a lone V row touches four times its bytes).  Two or four tasks a
// thread are no faster there, and 64 rows take 3.2 and 4.1 us instead of 2.7.
// The MLA latent (576 channels, K alone), 100003 rows in random order: bf16 written 44.8 us (5.2 TB/s) and read
// 41.8 (5.5), E4M3 38.7 (4.5) and 34.4 (5.0); 64 rows 2.1 to 2.3 us.
#include "mxfp4.h"
#include "vx_device.h"
#include "vx_internal.h"

namespace vx {
namespace {

constexpr int kRowThreads = 256;

struct RowArgs {
  uint8_t* k;
  uint8_t* v;
  const uint16_t* k_in;
  const uint16_t* v_in;
  uint16_t* k_out;
  uint16_t* v_out;
  int64_t k_row, k_head, v_row, v_head;    // strides of the bf16 rows, in elements
  const int64_t* slots;
  int n, H, h_shift, ps, ps_shift, num_phys;
  float k_scale, v_scale;
};

// A thread's task.
struct Task {
  int n, h, c8;
  bool in;                                 // false past the last row
};
template <int D>
__device__ __forceinline__ Task row_task(const RowArgs& a) {
  constexpr uint32_t CH = D / 8;
  const uint32_t x = blockIdx.x * kRowThreads + threadIdx.x;
  const uint32_t y = x / CH, z = y >> 2;
  const uint32_t nq = z >> a.h_shift;
  Task t;
  t.c8 = (int)(x - y * CH);
  t.h = (int)(z - (nq << a.h_shift));
  t.n = (int)(nq * 4 + (y & 3));
  t.in = t.n < a.n;
  return t;
}

// Page and token of a slot; false for a slot outside the cache.
__device__ __forceinline__ bool slot_place(const RowArgs& a, int64_t slot, int64_t& page, int& t) {
  page = slot >> a.ps_shift;
  t = (int)(slot & (a.ps - 1));
  return slot >= 0 && page < a.num_phys;
}

// 8 values of a row as fp8 codes: value / scale, to the nearest even code, finite values and
// infinities at most the format's largest.
template <int KT>
__device__ __forceinline__ uint2 encode_fp8(const uint4& w, float scale) {
  constexpr float kTop = KT == kKvFp8E4M3 ? 448.f : 57344.f;
  const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
  float x[8];
#pragma unroll
  for (int e = 0; e < 4; e++) {
    x[2 * e] = bf16lo(ws[e]) / scale;
    x[2 * e + 1] = bf16hi(ws[e]) / scale;
  }
#pragma unroll
  for (int e = 0; e < 8; e++) x[e] = x[e] != x[e] ? x[e] : fminf(fmaxf(x[e], -kTop), kTop);
  int lo = 0, hi = 0;
  if constexpr (KT == kKvFp8E4M3) {
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[4], x[5], hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[6], x[7], hi, true);
  } else {
    lo = __builtin_amdgcn_cvt_pk_bf8_f32(x[0], x[1], lo, false);
    lo = __builtin_amdgcn_cvt_pk_bf8_f32(x[2], x[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_bf8_f32(x[4], x[5], hi, false);
    hi = __builtin_amdgcn_cvt_pk_bf8_f32(x[6], x[7], hi, true);
  }
  return make_uint2((uint32_t)lo, (uint32_t)hi);
}

template <int KT>
__device__ __forceinline__ uint4 decode_fp8(const uint2& w, float scale) {
  const int ws[2] = {(int)w.x, (int)w.y};
  uint32_t o[4];
#pragma unroll
  for (int h = 0; h < 2; h++) {
    float2_t lo, hi;
    if constexpr (KT == kKvFp8E4M3) {
      lo = __builtin_amdgcn_cvt_pk_f32_fp8(ws[h], false);
      hi = __builtin_amdgcn_cvt_pk_f32_fp8(ws[h], true);
    } else {
      lo = __builtin_amdgcn_cvt_pk_f32_bf8(ws[h], false);
      hi = __builtin_amdgcn_cvt_pk_f32_bf8(ws[h], true);
    }
    o[2 * h] = f32_to_bf16_rne(lo[0] * scale) | (f32_to_bf16_rne(lo[1] * scale) << 16);
    o[2 * h + 1] = f32_to_bf16_rne(hi[0] * scale) | (f32_to_bf16_rne(hi[1] * scale) << 16);
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// Largest of the four adjacent lanes that hold a group.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xf, 0xf, false));
  return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, false));
}

template <int D, int KT>
__device__ __forceinline__ void write_chunk(const RowArgs& a, bool v, int64_t page, int t, int h, int c8, bool ok,
                                            const uint4& w) {
  uint8_t* base = v ? a.v : a.k;
  if constexpr (KT == kKvMxFp4) {
    const uint32_t e = mx::group_scale(quad_max(mx::amax_bits(w)));   // every lane of the quad takes part
    if (!ok) return;
    uint8_t* slice = base + (page * a.H + h) * mx::slice_bytes(a.ps, D);
    const uint32_t codes = mx::encode8(w, e);
    if (v) mx::put_v_codes(slice, t, c8, D, codes);
    else *reinterpret_cast<uint32_t*>(slice + mx::k_code(t, c8, D)) = codes;
    if ((c8 & 3) == 0)
      slice[mx::codes_bytes(a.ps, D) + (v ? mx::v_scale(t, c8 >> 2, D) : mx::k_scale(t, c8 >> 2, D))] = (uint8_t)e;
  } else if (ok) {
    const int64_t at = ((page * a.H + h) * a.ps + t) * D + 8 * c8;
    if constexpr (KT == kKvBf16) *reinterpret_cast<uint4*>(base + 2 * at) = w;
    else *reinterpret_cast<uint2*>(base + at) = encode_fp8<KT>(w, v ? a.v_scale : a.k_scale);
  }
}

template <int D, int KT>
__global__ __launch_bounds__(kRowThreads) void write_kernel(const RowArgs a) {
  const Task q = row_task<D>(a);
  const int n = min(q.n, a.n - 1);
  const int64_t slot = a.slots[n];         // travels with the rows
  const uint4 wk = load_stream_u4(a.k_in + n * a.k_row + q.h * a.k_head + 8 * q.c8);
  const uint4 wv = a.v ? load_stream_u4(a.v_in + n * a.v_row + q.h * a.v_head + 8 * q.c8) : uint4{};
  int64_t page;
  int t;
  const bool ok = slot_place(a, slot, page, t) && q.in;
  write_chunk<D, KT>(a, false, page, t, q.h, q.c8, ok, wk);
  if (a.v) write_chunk<D, KT>(a, true, page, t, q.h, q.c8, ok, wv);
}

// A row given back, past the caches: 40001 rows of 8 heads from an mxfp4 cache 57.1 -> 43.6 us, and the
// 8192 rows written ahead of them, whose lines it no longer displaces, 16.4 -> 13.1.
__device__ __forceinline__ void put_row(uint16_t* dst, const uint4& w) {
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, w), reinterpret_cast<u32x4_t*>(dst));
}

// 8 channels of a cache row as loaded (bf16: 16 bytes; fp8: 8; mxfp4: 4 bytes of codes, and the scale),
// and as bf16 values.
template <int D, int KT>
__device__ __forceinline__ uint4 load_chunk(const RowArgs& a, bool v, int64_t page, int t, int h, int c8) {
  const uint8_t* base = v ? a.v : a.k;
  if constexpr (KT == kKvMxFp4) {
    const uint8_t* slice = base + (page * a.H + h) * mx::slice_bytes(a.ps, D);
    const uint32_t w = v ? mx::get_v_codes(slice, t, c8, D)
                         : *reinterpret_cast<const uint32_t*>(slice + mx::k_code(t, c8, D));
    const uint32_t e =
        slice[mx::codes_bytes(a.ps, D) + (v ? mx::v_scale(t, c8 >> 2, D) : mx::k_scale(t, c8 >> 2, D))];
    return make_uint4(w, e, 0, 0);
  } else {
    const int64_t at = ((page * a.H + h) * a.ps + t) * D + 8 * c8;
    if constexpr (KT == kKvBf16) return *reinterpret_cast<const uint4*>(base + 2 * at);
    const uint2 w = *reinterpret_cast<const uint2*>(base + at);
    return make_uint4(w.x, w.y, 0, 0);
  }
}
template <int KT>
__device__ __forceinline__ uint4 chunk_values(const uint4& w, float scale) {
  if constexpr (KT == kKvMxFp4) {
    const float s = mx::scale_operand(w.y);
    return make_uint4(mx::pair_bf16<0>(w.x, s), mx::pair_bf16<1>(w.x, s), mx::pair_bf16<2>(w.x, s),
                      mx::pair_bf16<3>(w.x, s));
  } else if constexpr (KT == kKvBf16) {
    return w;
  } else {
    return decode_fp8<KT>(make_uint2(w.x, w.y), scale);
  }
}

template <int D, int KT>
__global__ __launch_bounds__(kRowThreads) void read_kernel(const RowArgs a) {
  const Task q = row_task<D>(a);
  if (!q.in) return;
  int64_t page;
  int t;
  uint4 k{}, v{};
  if (slot_place(a, a.slots[q.n], page, t)) {
    k = load_chunk<D, KT>(a, false, page, t, q.h, q.c8);
    if (a.v) v = load_chunk<D, KT>(a, true, page, t, q.h, q.c8);
    k = chunk_values<KT>(k, a.k_scale);
    v = chunk_values<KT>(v, a.v_scale);
  }
  put_row(a.k_out + q.n * a.k_row + q.h * a.k_head + 8 * q.c8, k);
  if (a.v) put_row(a.v_out + q.n * a.v_row + q.h * a.v_head + 8 * q.c8, v);
}

template <int D, int KT>
hipError_t launch(const RowArgs& all, bool write, hipStream_t stream) {
  // a launch has fewer than 2^32 threads
  const int most = (1 << 30) / (all.H * (D / 8)) & ~3;
  RowArgs a = all;
  for (int done = 0; done < all.n; done += a.n) {
    a.n = all.n - done < most ? all.n - done : most;
    a.slots = all.slots + done;
    if (write) {
      a.k_in = all.k_in + done * all.k_row;
      if (a.v) a.v_in = all.v_in + done * all.v_row;
    } else {
      a.k_out = all.k_out + done * all.k_row;
      if (a.v) a.v_out = all.v_out + done * all.v_row;
    }
    const int64_t tasks = ((int64_t)a.n + 3) / 4 * 4 * a.H * (D / 8);
    const dim3 grid((unsigned)((tasks + kRowThreads - 1) / kRowThreads));
    if (write) hipLaunchKernelGGL((write_kernel<D, KT>), grid, dim3(kRowThreads), 0, stream, a);
    else hipLaunchKernelGGL((read_kernel<D, KT>), grid, dim3(kRowThreads), 0, stream, a);
  }
  return hipGetLastError();
}

template <int D>
hipError_t launch_kt(const RowArgs& a, int kt, bool write, hipStream_t stream) {
  if (kt == kKvFp8E4M3) return launch<D, kKvFp8E4M3>(a, write, stream);
  if (kt == kKvFp8E5M2) return launch<D, kKvFp8E5M2>(a, write, stream);
  if constexpr (D != 576) {
    if (kt == kKvMxFp4) return launch<D, kKvMxFp4>(a, write, stream);
  }
  return launch<D, kKvBf16>(a, write, stream);
}

hipError_t launch_rows(const Geometry& g, RowArgs& a, bool write, hipStream_t stream) {
  if (a.n == 0) return hipSuccess;
  a.k = static_cast<uint8_t*>(const_cast<void*>(g.k));
  a.v = static_cast<uint8_t*>(const_cast<void*>(g.v));
  a.H = g.H;
  a.h_shift = __builtin_ctz((unsigned)g.H);
  a.ps = g.ps;
  a.ps_shift = __builtin_ctz((unsigned)g.ps);
  a.num_phys = g.num_phys_pages;
  a.k_scale = g.k_scale;
  a.v_scale = g.v_scale;
  if (g.Dqk == 128) return launch_kt<128>(a, g.kv_dtype, write, stream);
  if (g.Dqk == 64) return launch_kt<64>(a, g.kv_dtype, write, stream);
  return launch_kt<576>(a, g.kv_dtype, write, stream);
}

}  // namespace

hipError_t launch_kv_write(const Geometry& g, const RowView& k, const RowView& v, const int64_t* slots, int n,
                           hipStream_t stream) {
  RowArgs a{};
  a.k_in = static_cast<const uint16_t*>(k.rows);
  a.v_in = static_cast<const uint16_t*>(v.rows);
  a.k_row = k.row_stride;
  a.k_head = k.head_stride;
  a.v_row = v.row_stride;
  a.v_head = v.head_stride;
  a.slots = slots;
  a.n = n;
  return launch_rows(g, a, true, stream);
}

hipError_t launch_kv_read(const Geometry& g, const RowView& k, const RowView& v, const int64_t* slots, int n,
                          hipStream_t stream) {
  RowArgs a{};
  a.k_out = static_cast<uint16_t*>(const_cast<void*>(k.rows));
  a.v_out = static_cast<uint16_t*>(const_cast<void*>(v.rows));
  a.k_row = k.row_stride;
  a.k_head = k.head_stride;
  a.v_row = v.row_stride;
  a.v_head = v.head_stride;
  a.slots = slots;
  a.n = n;
  return launch_rows(g, a, false, stream);
}

}  // namespace vx
