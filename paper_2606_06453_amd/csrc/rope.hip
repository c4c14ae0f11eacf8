// Rows of a fused projection into the paged cache, their keys and queries rotated by their positions
// (vx_rope_kv_write).
//
// y = scale (a cos t - b sin t, b cos t + a sin t) for the pairs (a, b) of a row, t = position * frequency.
// Far positions leave an fp32 angle nothing to turn by (at 2^20 its step is 2^-4), so angle, sine, cosine
// and products are fp64; a row's angles are computed once for all its heads and held in LDS.  A
// workgroup takes a few rows, or a part of one row's heads where there are few.
//
// Tasks, 8 channels each: the K chunks (a thread reads its chunk and the one that holds its partners, so that the four
// lanes of a 4-bit group hold neighbouring chunks whatever the pairing), the V chunks, then the queries: both chunks of
// a pair of halves by one thread, which makes q_out == q safe, and the chunks that pass.  A thread sends for the
// chunks of a few tasks before it works on the first, for the kernel is bound by memory: 100003 rows of 36 heads of 128
// channels into E4M3 319 us (5.5 TB/s, a large copy's rate; one task at a time 384), 8192 rows of 48 heads into
// mxfp4 38 us.
#include "cache_rows.h"
#include "mxfp4.h"
#include "vx_device.h"
#include "vx_internal.h"

namespace vx {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeRows = 2;               // most rows of a workgroup

struct RopeArgs {
  uint8_t* k;
  uint8_t* v;
  const uint16_t* q_in;
  uint16_t* q_out;
  const uint16_t* k_in;
  const uint16_t* v_in;
  int64_t q_row, q_head, o_row, o_head, k_row, k_head, v_row, v_head;
  const float* inv_freq;
  const int32_t* axis;
  const int64_t* pos;
  int64_t pos_stride;
  const int64_t* slots;
  int n, H, Hq, ps, ps_shift, num_phys, num_axes;
  int first, half;                         // first rotated channel, pairs
  int interleaved;
  int rows;                                // rows of a workgroup
  int k_tasks, v_tasks;                    // of a row
  int turned, passed;                      // query tasks of a head
  uint32_t turned_inv, passed_inv;         // 2^32 / them, rounded up
  float scale, k_scale, v_scale;
};

// Sine and cosine of x >= 0 in fp64: x less the nearest multiple of pi / 2 (held in two parts, each product
// inside an fma), then the Taylor series on [-pi / 4, pi / 4], whose first terms left out are below 2^-56.
__device__ __forceinline__ double2 cos_sin(double x) {
  constexpr double kHalfPiHi = 1.57079632679489655800, kHalfPiLo = 6.12323399573676603587e-17;
  const double k = rint(x * 0.63661977236758134308);
  const double r = fma(-k, kHalfPiLo, fma(-k, kHalfPiHi, x)), z = r * r;
  double s = 1.0 / 355687428096000.0;                                     // 1 / 17!
  s = fma(s, z, -1.0 / 1307674368000.0);
  s = fma(s, z, 1.0 / 6227020800.0);
  s = fma(s, z, -1.0 / 39916800.0);
  s = fma(s, z, 1.0 / 362880.0);
  s = fma(s, z, -1.0 / 5040.0);
  s = fma(s, z, 1.0 / 120.0);
  s = fma(s, z, -1.0 / 6.0);
  s = fma(s * z, r, r);
  double c = -1.0 / 6402373705728000.0;                                   // 1 / 18!
  c = fma(c, z, 1.0 / 20922789888000.0);
  c = fma(c, z, -1.0 / 87178291200.0);
  c = fma(c, z, 1.0 / 479001600.0);
  c = fma(c, z, -1.0 / 3628800.0);
  c = fma(c, z, 1.0 / 40320.0);
  c = fma(c, z, -1.0 / 720.0);
  c = fma(c, z, 1.0 / 24.0);
  c = fma(c, z, -0.5);
  c = fma(c, z, 1.0);
  const int quarter = (int)((int64_t)k & 3);
  const double cc = (quarter & 1) ? s : c, ss = (quarter & 1) ? c : s;
  return make_double2(quarter == 1 || quarter == 2 ? -cc : cc, quarter >= 2 ? -ss : ss);
}

__device__ __forceinline__ void widen8(const uint4& w, float (&x)[8]) {
  const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int e = 0; e < 4; e++) {
    x[2 * e] = bf16lo(ws[e]);
    x[2 * e + 1] = bf16hi(ws[e]);
  }
}
__device__ __forceinline__ uint4 narrow8(const float (&x)[8]) {
  uint32_t o[4];
#pragma unroll
  for (int e = 0; e < 4; e++) o[e] = f32_to_bf16_rne(x[2 * e]) | (f32_to_bf16_rne(x[2 * e + 1]) << 16);
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// The two results of a pair.
__device__ __forceinline__ float turn_a(float a, float b, const double2& cs) {
  return (float)((double)a * cs.x - (double)b * cs.y);
}
__device__ __forceinline__ float turn_b(float a, float b, const double2& cs) {
  return (float)((double)b * cs.x + (double)a * cs.y);
}

// A chunk's codes of a 4-bit cache (byte e of its group's scale beside the group's first chunk).
template <int D>
__device__ __forceinline__ void put_mx(const RopeArgs& a, uint8_t* base, bool v, int64_t page, int t, int h, int c8,
                                       uint32_t codes, uint32_t e) {
  uint8_t* slice = base + (page * a.H + h) * mx::slice_bytes(a.ps, D);
  if (v) mx::put_v_codes(slice, t, c8, D, codes);
  else *reinterpret_cast<uint32_t*>(slice + mx::k_code(t, c8, D)) = codes;
  if ((c8 & 3) == 0)
    slice[mx::codes_bytes(a.ps, D) + (v ? mx::v_scale(t, c8 >> 2, D) : mx::k_scale(t, c8 >> 2, D))] = (uint8_t)e;
}

// 8 rotated channels of K into the cache.
template <int D, int KT>
__device__ __forceinline__ void store_k(const RopeArgs& a, int64_t page, int t, int h, int c8, bool ok, float (&x)[8]) {
  if constexpr (KT == kKvMxFp4) {
    // the rule of mx::group_scale and mx::encode8 on fp32 values
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; e++) m = max(m, __float_as_uint(x[e]) & 0x7fffffffu);
    m = quad_max(m);                       // every lane of the quad takes part
    const int e0 = min(max((int)((m + 0x200000u) >> 23) - 2, mx::kMinScale), mx::kMaxScale);
    const uint32_t e = m >= 0x7f800000u ? (uint32_t)mx::kNanScale : (uint32_t)e0;
    const float s = __uint_as_float(e << 23);
    uint32_t codes = 0;
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], s, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], s, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], s, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], s, 3);
    if (ok) put_mx<D>(a, a.k, false, page, t, h, c8, e == (uint32_t)mx::kNanScale ? 0u : codes, e);
  } else if (ok) {
    const int64_t at = ((page * a.H + h) * a.ps + t) * D + 8 * c8;
    if constexpr (KT == kKvBf16) {
      *reinterpret_cast<uint4*>(a.k + 2 * at) = narrow8(x);
    } else {
#pragma unroll
      for (int e = 0; e < 8; e++) x[e] = x[e] / a.k_scale;
      *reinterpret_cast<uint2*>(a.k + at) = fp8_codes<KT>(x);
    }
  }
}

// 8 channels of V into the cache, as vx_kv_write stores them.
template <int D, int KT>
__device__ __forceinline__ void store_v(const RopeArgs& a, int64_t page, int t, int h, int c8, bool ok, const uint4& w) {
  if constexpr (KT == kKvMxFp4) {
    const uint32_t e = mx::group_scale(quad_max(mx::amax_bits(w)));
    if (ok) put_mx<D>(a, a.v, true, page, t, h, c8, mx::encode8(w, e), e);
  } else if (ok) {
    const int64_t at = ((page * a.H + h) * a.ps + t) * D + 8 * c8;
    if constexpr (KT == kKvBf16) *reinterpret_cast<uint4*>(a.v + 2 * at) = w;
    else *reinterpret_cast<uint2*>(a.v + at) = encode_fp8<KT>(w, a.v_scale);
  }
}

// Chunk c8 of a row rotated: its own 8 channels x, from them and their partners y (halves).
__device__ __forceinline__ void turn_chunk(const RopeArgs& a, int c8, const double2* cs, float (&x)[8], const float (&y)[8]) {
  const int c = 8 * c8 - a.first;                      // channel inside the rotated part
  if (c < 0 || c >= 2 * a.half) return;
  if (a.interleaved) {
#pragma unroll
    for (int e = 0; e < 4; e++) {
      const double2 w = cs[(c >> 1) + e];
      const float p = x[2 * e], r = x[2 * e + 1];
      x[2 * e] = turn_a(p, r, w);
      x[2 * e + 1] = turn_b(p, r, w);
    }
  } else {
    const bool low = c < a.half;
    const double2* w = cs + (low ? c : c - a.half);
#pragma unroll
    for (int e = 0; e < 8; e++) x[e] = low ? turn_a(x[e], y[e], w[e]) : turn_b(y[e], x[e], w[e]);
  }
}

// Chunk that holds the partners of chunk c8 (itself, where there are none or they lie in it).
__device__ __forceinline__ int partner_chunk(const RopeArgs& a, int c8) {
  const int c = 8 * c8 - a.first;
  if (a.interleaved || c < 0 || c >= 2 * a.half) return c8;
  return c < a.half ? c8 + a.half / 8 : c8 - a.half / 8;
}

// `count` tasks of the workgroups of a row group, N at a time: load(x) sends for task x's chunks, use(x, chunks) does it.
template <int N, class Load, class Use>
__device__ __forceinline__ void tasks_of(int count, Load load, Use use) {
  const int step = (int)(gridDim.y * kRopeThreads);
  for (int x = (int)(blockIdx.y * kRopeThreads + threadIdx.x); x < count; x += N * step) {
    decltype(load(0)) got[N];
#pragma unroll
    for (int n = 0; n < N; n++)
      if (x + n * step < count) got[n] = load(x + n * step);
#pragma unroll
    for (int n = 0; n < N; n++)
      if (x + n * step < count) use(x + n * step, got[n]);
  }
}

struct TwoChunks {
  uint4 own, other;
};
__device__ __forceinline__ uint4 chunk_at(const uint16_t* p) { return *reinterpret_cast<const uint4*>(p); }

template <int D, int KT>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(const RopeArgs a) {
  extern __shared__ __attribute__((aligned(16))) double2 angles[];         // [rows][half]
  constexpr int CH = D / 8;
  const int n0 = (int)blockIdx.x * a.rows, rows = min(a.rows, a.n - n0);
  for (int x = (int)threadIdx.x; x < rows * a.half; x += kRopeThreads) {
    const int r = x / a.half, c = x - r * a.half;
    const int ax = a.axis ? min(max(a.axis[c], 0), a.num_axes - 1) : 0;
    const int64_t p = a.pos[ax * a.pos_stride + n0 + r];
    double2 w = cos_sin((double)p * (double)a.inv_freq[c]);
    w.x *= a.scale;
    w.y *= a.scale;
    angles[x] = w;
  }
  __syncthreads();
  // row of task x, at most kRopeRows of them
  auto row_of = [&](int x, int per_row, int& z) {
    int r = 0;
#pragma unroll
    for (int y = 1; y < kRopeRows; y++) r += x >= y * per_row;
    z = x - r * per_row;
    return r;
  };
  auto place = [&](int64_t n, int64_t& page, int& t) {
    const int64_t slot = a.slots[n];
    page = slot >> a.ps_shift;
    t = (int)(slot & (a.ps - 1));
    return slot >= 0 && page < a.num_phys;
  };
  tasks_of<2>(rows * a.k_tasks,
      [&](int x) {
        int z;
        const int64_t n = n0 + row_of(x, a.k_tasks, z);
        const int h = z / CH, c8 = z - h * CH;
        const uint16_t* row = a.k_in + n * a.k_row + h * a.k_head;
        return TwoChunks{chunk_at(row + 8 * c8), chunk_at(row + 8 * partner_chunk(a, c8))};
      },
      [&](int x, const TwoChunks& got) {
        int z, t;
        const int r = row_of(x, a.k_tasks, z), h = z / CH, c8 = z - h * CH;
        int64_t page;
        const bool ok = place(n0 + r, page, t);
        float own[8], other[8];
        widen8(got.own, own);
        widen8(got.other, other);
        turn_chunk(a, c8, angles + r * a.half, own, other);
        store_k<D, KT>(a, page, t, h, c8, ok, own);
      });
  tasks_of<4>(rows * a.v_tasks,
      [&](int x) {
        int z;
        const int64_t n = n0 + row_of(x, a.v_tasks, z);
        const int h = z / CH, c8 = z - h * CH;
        return load_stream_u4(a.v_in + n * a.v_row + h * a.v_head + 8 * c8);
      },
      [&](int x, const uint4& got) {
        int z, t;
        const int r = row_of(x, a.v_tasks, z), h = z / CH, c8 = z - h * CH;
        int64_t page;
        const bool ok = place(n0 + r, page, t);
        store_v<D, KT>(a, page, t, h, c8, ok, got);
      });
  if (!a.q_in) return;
  // source and destination of a head's rows, and the channel of task z of it
  auto query = [&](int x, int per_head, uint32_t inv, int& r, int& z, const uint16_t*& src, uint16_t*& dst) {
    r = row_of(x, a.Hq * per_head, z);
    const int h = per_head == 1 ? z : (int)__umulhi((uint32_t)z, inv);
    z -= h * per_head;
    src = a.q_in + (n0 + r) * a.q_row + h * a.q_head;
    dst = a.q_out + (n0 + r) * a.o_row + h * a.o_head;
  };
  tasks_of<2>(rows * a.Hq * a.turned,
      [&](int x) {
        int r, z;
        const uint16_t* src;
        uint16_t* dst;
        query(x, a.turned, a.turned_inv, r, z, src, dst);
        src += a.first + 8 * z;
        return TwoChunks{chunk_at(src), a.interleaved ? uint4{} : chunk_at(src + a.half)};
      },
      [&](int x, const TwoChunks& got) {
        int r, z;
        const uint16_t* src;
        uint16_t* dst;
        query(x, a.turned, a.turned_inv, r, z, src, dst);
        dst += a.first + 8 * z;
        const double2* cs = angles + r * a.half;
        float p[8], q[8];
        widen8(got.own, p);
        if (a.interleaved) {
#pragma unroll
          for (int e = 0; e < 4; e++) {
            const double2 w = cs[4 * z + e];
            const float u = p[2 * e], v = p[2 * e + 1];
            p[2 * e] = turn_a(u, v, w);
            p[2 * e + 1] = turn_b(u, v, w);
          }
        } else {
          widen8(got.other, q);
#pragma unroll
          for (int e = 0; e < 8; e++) {
            const double2 w = cs[8 * z + e];
            const float u = p[e], v = q[e];
            p[e] = turn_a(u, v, w);
            q[e] = turn_b(u, v, w);
          }
          *reinterpret_cast<uint4*>(dst + a.half) = narrow8(q);
        }
        *reinterpret_cast<uint4*>(dst) = narrow8(p);
      });
  if (a.passed == 0 || (a.q_in == a.q_out)) return;      // in place they are there
  auto passing = [&](int z) { return 8 * z < a.first ? 8 * z : 8 * z + 2 * a.half; };
  tasks_of<4>(rows * a.Hq * a.passed,
      [&](int x) {
        int r, z;
        const uint16_t* src;
        uint16_t* dst;
        query(x, a.passed, a.passed_inv, r, z, src, dst);
        return load_stream_u4(src + passing(z));
      },
      [&](int x, const uint4& got) {
        int r, z;
        const uint16_t* src;
        uint16_t* dst;
        query(x, a.passed, a.passed_inv, r, z, src, dst);
        *reinterpret_cast<uint4*>(dst + passing(z)) = got;
      });
}

template <int D, int KT>
hipError_t launch(const RopeArgs& all, hipStream_t stream) {
  constexpr int kMost = 1 << 24;           // rows of a launch, which has fewer than 2^32 threads
  RopeArgs a = all;
  for (int done = 0; done < all.n; done += a.n) {
    a.n = min(all.n - done, kMost);
    a.q_in = all.q_in + done * all.q_row;
    a.q_out = all.q_out + done * all.o_row;
    a.k_in = all.k_in + done * all.k_row;
    a.v_in = all.v_in + done * all.v_row;
    a.pos = all.pos + done;
    a.slots = all.slots + done;
    const int groups = (a.n + a.rows - 1) / a.rows;
    const int whole = (a.rows * (a.k_tasks + a.v_tasks + a.Hq * (a.turned + a.passed)) + kRopeThreads - 1) / kRopeThreads;
    int parts = 1;
    while (groups * parts < 1024 && parts < whole) parts *= 2;
    hipLaunchKernelGGL((rope_kernel<D, KT>), dim3((unsigned)groups, (unsigned)parts), dim3(kRopeThreads),
                       sizeof(double2) * (size_t)a.rows * a.half, stream, a);
  }
  return hipGetLastError();
}

template <int D>
hipError_t launch_kt(const RopeArgs& a, int kt, hipStream_t stream) {
  if (kt == kKvFp8E4M3) return launch<D, kKvFp8E4M3>(a, stream);
  if (kt == kKvFp8E5M2) return launch<D, kKvFp8E5M2>(a, stream);
  if constexpr (D != 576) {
    if (kt == kKvMxFp4) return launch<D, kKvMxFp4>(a, stream);
  }
  return launch<D, kKvBf16>(a, stream);
}

}  // namespace

hipError_t launch_rope_kv_write(const Geometry& g, const Rotation& rope, const RowView& q, const RowView& q_out, int Hq,
                                const RowView& k, const RowView& v, const int64_t* positions, int64_t positions_stride,
                                const int64_t* slots, int n, hipStream_t stream) {
  if (n == 0) return hipSuccess;
  RopeArgs a{};
  a.k = static_cast<uint8_t*>(const_cast<void*>(g.k));
  a.v = static_cast<uint8_t*>(const_cast<void*>(g.v));
  a.q_in = static_cast<const uint16_t*>(q.rows);
  a.q_out = static_cast<uint16_t*>(const_cast<void*>(q_out.rows));
  a.k_in = static_cast<const uint16_t*>(k.rows);
  a.v_in = static_cast<const uint16_t*>(v.rows);
  a.q_row = q.row_stride;
  a.q_head = q.head_stride;
  a.o_row = q_out.row_stride;
  a.o_head = q_out.head_stride;
  a.k_row = k.row_stride;
  a.k_head = k.head_stride;
  a.v_row = v.row_stride;
  a.v_head = v.head_stride;
  a.inv_freq = rope.inv_freq;
  a.axis = rope.axis;
  a.num_axes = rope.num_axes;
  a.first = rope.first;
  a.half = rope.dim / 2;
  a.interleaved = rope.interleaved;
  a.scale = rope.scale;
  a.pos = positions;
  a.pos_stride = positions_stride;
  a.slots = slots;
  a.n = n;
  a.H = g.H;
  a.Hq = Hq;
  a.ps = g.ps;
  a.ps_shift = __builtin_ctz((unsigned)g.ps);
  a.num_phys = g.num_phys_pages;
  a.k_scale = g.k_scale;
  a.v_scale = g.v_scale;
  a.rows = n >= 1024 * kRopeRows ? kRopeRows : 1;
  a.k_tasks = g.H * (g.Dqk / 8);
  a.v_tasks = g.v ? g.H * (g.Dv / 8) : 0;
  a.turned = rope.interleaved ? a.half / 4 : a.half / 8;
  a.passed = (g.Dqk - rope.dim) / 8;
  a.turned_inv = (uint32_t)(((1ull << 32) + a.turned - 1) / a.turned);
  a.passed_inv = a.passed ? (uint32_t)(((1ull << 32) + a.passed - 1) / a.passed) : 0;
  if (g.Dqk == 128) return launch_kt<128>(a, g.kv_dtype, stream);
  if (g.Dqk == 64) return launch_kt<64>(a, g.kv_dtype, stream);
  return launch_kt<576>(a, g.kv_dtype, stream);
}

}  // namespace vx
