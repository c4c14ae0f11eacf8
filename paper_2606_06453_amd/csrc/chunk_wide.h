// The wide tile kernel: four waves of 16 RT query rows each share every 64 or 32 tokens of K and V in LDS.
//
// LDS holds bf16 channels in D / 64 planes of 128 bytes a token, chunks of 16 bytes.  bf16 rows go there straight from
// memory (each lane of a load picks its source, so the swizzle costs nothing), other types pass through registers,
// where they are widened.  Operands of S^T = K Q^T are 16-byte reads of a token; those of O^T = V^T P^T are transposing
// reads of four tokens by 16 channels.  Chunk c of token t of a plane lies at place c ^ (t & 7), where neither kind of
// read collides: 36 and 41 cycles of a CU for 8 KiB (without the swizzle 131 and 136).  A read's plane is a constant of
// its address, so that few registers hold addresses.
// Two buffers: the next tokens travel while the present ones are multiplied.
#pragma once
#include "chunk_tile.h"

namespace vx {
namespace chunk {

typedef __attribute__((address_space(3))) uint8_t lds_u8;
__device__ __forceinline__ uint32_t lds_address(const uint8_t* p) { return (uint32_t)(uintptr_t)(lds_u8*)p; }
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short v4i16_t;

// Direct-to-LDS loads: lane l's 16 bytes at base + off go to LDS address lds + 16 l; the second form also loads base2 +
// off to lds + GAP.  In assembly, for the compiler would wait for loads that it sees before every read of LDS;
// `land_run` waits instead.  M0 holds the LDS address; the compiler reserves it, so its value is saved and restored.
__device__ __forceinline__ void send16(const uint8_t* base, uint32_t off, uint32_t lds) {
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %2, %3\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "s"(lds), "v"(off), "s"(base)
      : "memory");
}
template <int GAP>
__device__ __forceinline__ void send16(const uint8_t* base, const uint8_t* base2, uint32_t off, uint32_t lds) {
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %2, %3\n\t"
      "s_add_u32 m0, m0, %5\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %2, %4\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "s"(lds), "v"(off), "s"(base), "s"(base2), "n"(GAP)
      : "memory", "scc");
}

// A barrier that completes this wave's LDS accesses first.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <int D, int DV, int KT, int TOKENS>
struct Wide {
  static constexpr bool kAlias = D != DV;
  static constexpr int TK = TOKENS;                      // tokens of a buffer
  static constexpr int UNITS = TK / 16;                  // runs of 16 tokens
  static constexpr int PLANE = TK * 128;                 // bytes of 64 channels
  static constexpr int WPU = 4 / UNITS;                  // waves that load a run
  static constexpr int NI = D / 32 / WPU;                // pieces of a wave: 8 tokens of a plane
  static constexpr int TILE = TK * D * 2;                // bytes of K
  static constexpr int BUF = kAlias ? TILE : 2 * TILE;
};

// Piece k of a wave's part of a run: its first token, and its plane.
template <int D, int DV, int KT, int TOKENS>
__device__ __forceinline__ void piece(int wave, int k, int& token, int& plane) {
  using G = Wide<D, DV, KT, TOKENS>;
  const int x = G::NI * (wave % G::WPU) + k;
  token = 8 * (x & 1);
  plane = x >> 1;
}

// A wave's part of a run on its way through registers: fp8, 16 codes a lane and piece; mxfp4, a lane's D / 4 codes of
// one K row and the codes of D / 16 channels of four V rows, and their scales.
template <int D, int DV, int KT, int TOKENS>
struct Travel {
  static constexpr bool kMx = KT == kKvMxFp4;
  static constexpr int N = kMx ? 1 : (D / 64 + Wide<D, DV, KT, TOKENS>::WPU - 1) / Wide<D, DV, KT, TOKENS>::WPU;
  static constexpr int W = kMx ? D / 32 : 4;
  // mxfp4: of two waves that load a run one takes K, the other V
  static __device__ __forceinline__ bool takes_k(int wave) { return Wide<D, DV, KT, TOKENS>::WPU == 1 || (wave & 1) == 0; }
  static __device__ __forceinline__ bool takes_v(int wave) { return Wide<D, DV, KT, TOKENS>::WPU == 1 || (wave & 1) == 1; }
  uint32_t k[N][W], v[Wide<D, DV, KT, TOKENS>::kAlias ? 1 : N][W], k_scale, v_scale;
};

// fp8: the plane of a wave's piece x of a run (none: D / 64), of which lane l takes the l % 4th 16 channels of token l / 4.
template <int D, int DV, int KT, int TOKENS>
__device__ __forceinline__ int codes_plane(int wave, int x) {
  using G = Wide<D, DV, KT, TOKENS>;
  return min(G::WPU * x + wave % G::WPU, D / 64);
}

// Starts a run's way into the buffer (bf16), or into registers.  t: its first token's place in the page; left: its
// tokens before the last one that any row attends (other types: what lies behind arrives as zeros).
template <int D, int DV, int KT, int TOKENS>
__device__ __forceinline__ void send_run(const ChunkArgs& a, const uint8_t* ks, const uint8_t* vs, int t, int left, int wave,
                                         int lane, uint8_t* buf, Travel<D, DV, KT, TOKENS>& r) {
  using G = Wide<D, DV, KT, TOKENS>;
  using T = Travel<D, DV, KT, TOKENS>;
  if constexpr (KT == kKvBf16) {
    const uint32_t dst = lds_address(buf) + (wave / G::WPU) * 16 * 128;
    const uint32_t at = 2 * ((lane >> 3) * D + 8 * ((lane & 7) ^ (lane >> 3)));
#pragma unroll
    for (int k = 0; k < G::NI; k++) {
      int token, plane;
      piece<D, DV, KT, TOKENS>(wave, k, token, plane);
      const uint32_t to = dst + plane * G::PLANE + token * 128;
      const int from = 2 * ((t + token) * D + 64 * plane);
      if constexpr (G::kAlias) send16(ks + from, at, to);
      else send16<G::TILE>(ks + from, vs + from, at, to);
    }
  } else if constexpr (T::kMx) {
    const int col = lane & 15, grp = lane >> 4;
    if (T::takes_k(wave)) {
      load_words<T::W>(rows_of<D, KT>(ks, t, 16), lane * (D / 8), r.k[0]);
      r.k_scale = __builtin_amdgcn_raw_buffer_load_b8(scales_of<D>(a, ks, t), (lane >> 2) * (D / 32) + (lane & 3) * D / 128, 0, 0);
    }
    if (T::takes_v(wave)) {
      load_words<T::W>(rows_of<D, KT>(vs, t, 16), lane * (D / 8), r.v[0]);
      r.v_scale = __builtin_amdgcn_raw_buffer_load_b32(scales_of<D>(a, vs, t), (grp * (D / 32) + col * (D / 16) / 32) * 4, 0, 0);
      const int n = left - 4 * grp;                      // byte x: token 4 grp + x; a scale of 0 is 2^-127
      r.v_scale &= n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1;
    }
  } else {
    const int n = min(left, 16);
#pragma unroll
    for (int x = 0; x < T::N; x++) {
      const int plane = codes_plane<D, DV, KT, TOKENS>(wave, x);
      if (plane == D / 64) continue;
      const int off = (lane >> 2) * D + 16 * (lane & 3) + 64 * plane;
      load_words<4>(rows_of<D, KT>(ks, t, n), off, r.k[x]);
      if constexpr (!G::kAlias) load_words<4>(rows_of<D, KT>(vs, t, n), off, r.v[x]);
    }
  }
}

// Chunk c of token `token` of a run whose first plane is at `run`.
template <int PLANE>
__device__ __forceinline__ uint4* chunk_place(uint8_t* run, int token, int c) {
  return reinterpret_cast<uint4*>(run + (c >> 3) * PLANE + token * 128 + 16 * ((c ^ token) & 7));
}
template <int KT>
__device__ __forceinline__ uint4 widen_codes(uint32_t lo, uint32_t hi) {
  return make_uint4(fp8_pair<KT, false>(lo), fp8_pair<KT, true>(lo), fp8_pair<KT, false>(hi), fp8_pair<KT, true>(hi));
}
__device__ __forceinline__ uint4 widen_mx(uint32_t w, float s) {
  return make_uint4(mx::pair_bf16<0>(w, s), mx::pair_bf16<1>(w, s), mx::pair_bf16<2>(w, s), mx::pair_bf16<3>(w, s));
}

// Ends it: widened rows into the buffer; of bf16 rows, those of V behind the last token that any row attends (which may
// hold anything) are set to zero.
template <int D, int DV, int KT, int TOKENS>
__device__ __forceinline__ void land_run(int wave, int lane, int left, uint8_t* buf, const Travel<D, DV, KT, TOKENS>& r) {
  using G = Wide<D, DV, KT, TOKENS>;
  using T = Travel<D, DV, KT, TOKENS>;
  uint8_t* run = buf + (wave / G::WPU) * 16 * 128;
  if constexpr (KT == kKvBf16) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (left < 16) {
      for (int k = 0; k < G::NI; k++) {
        int token, plane;
        piece<D, DV, KT, TOKENS>(wave, k, token, plane);
        uint8_t* dst = run + plane * G::PLANE + token * 128 + 16 * lane + (G::kAlias ? 0 : G::TILE);
        if (token + (lane >> 3) >= left) *reinterpret_cast<uint4*>(dst) = make_uint4(0, 0, 0, 0);
      }
    }
  } else if constexpr (T::kMx) {
    if (T::takes_k(wave)) {                              // lane holds D / 4 channels of token lane / 4
      const float s = mx::scale_operand(r.k_scale);
#pragma unroll
      for (int x = 0; x < D / 32; x++) *chunk_place<G::PLANE>(run, lane >> 2, (lane & 3) * (D / 32) + x) = widen_mx(r.k[0][x], s);
    }
    if (T::takes_v(wave)) {                              // channels col D / 16 .. of tokens 4 grp + x
      const int col = lane & 15, grp = lane >> 4;
#pragma unroll
      for (int x = 0; x < 4; x++) {
        const float f = mx::scale_operand((r.v_scale >> (8 * x)) & 255);
        if constexpr (D == 128) {
          *chunk_place<G::PLANE>(run + G::TILE, 4 * grp + x, col) = widen_mx(r.v[0][x], f);
        } else {
          const uint32_t w = r.v[0][x >> 1];
          uint2* p = reinterpret_cast<uint2*>(chunk_place<G::PLANE>(run + G::TILE, 4 * grp + x, col >> 1)) + (col & 1);
          *p = (x & 1) ? make_uint2(mx::pair_bf16<2>(w, f), mx::pair_bf16<3>(w, f)) : make_uint2(mx::pair_bf16<0>(w, f), mx::pair_bf16<1>(w, f));
        }
      }
    }
  } else {
#pragma unroll
    for (int x = 0; x < T::N; x++) {
      const int plane = codes_plane<D, DV, KT, TOKENS>(wave, x), token = lane >> 2;
      if (plane == D / 64) continue;
      // every other pair of tokens begins with its second chunk: first chunks alone leave half of the banks idle
      const int odd = (token >> 1) & 1;
      auto put = [&](uint8_t* to, const uint32_t (&w)[T::W]) {
#pragma unroll
        for (int e = 0; e < 2; e++)
          *chunk_place<G::PLANE>(to + plane * G::PLANE, token, 2 * (lane & 3) + (e ^ odd)) =
              widen_codes<KT>(odd ? w[2 - 2 * e] : w[2 * e], odd ? w[3 - 2 * e] : w[2 * e + 1]);
      };
      put(run, r.k[x]);
      if constexpr (!G::kAlias) put(run + G::TILE, r.v[x]);
    }
  }
}

// Operand A of S^T: 16 tokens from t0, k-step kk (channels 32 kk + 8 grp ..).
template <int PLANE>
__device__ __forceinline__ bf16x8_t k_from_lds(const uint8_t* tile, int t0, int kk, int col, int grp) {
  const int c = (4 * (kk & 1) + grp) ^ (col & 7);
  return *reinterpret_cast<const bf16x8_t*>(tile + (t0 + col) * 128 + 16 * c + (kk >> 1) * PLANE);
}

// Operand A of O^T: channels 16 j + col of tokens t0 + 4 grp + 0..3 and t0 + 16 + 4 grp + 0..3.  Lane 4 r + x of
// 16 reads channels 4 x .. 4 x + 3 of row r; the transposing read gives it channel `lane` of the four rows.
template <int PLANE>
__device__ __forceinline__ bf16x8_t v_from_lds(const uint8_t* tile, int t0, int j, int col, int grp) {
  const int row = 4 * grp + (col >> 2), x = col & 3, c = (2 * (j & 3) + (x >> 1)) ^ (row & 7);
  lds_u8* p = (lds_u8*)(tile + (t0 + row) * 128 + 16 * c + 8 * (x & 1) + (j >> 2) * PLANE);
  const v4i16_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16_t*)p);
  const v4i16_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16_t*)(p + 16 * 128));
  typedef short s16x8_t __attribute__((ext_vector_type(8)));
  const s16x8_t w = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return __builtin_bit_cast(bf16x8_t, w);
}

}  // namespace chunk
}  // namespace vx
