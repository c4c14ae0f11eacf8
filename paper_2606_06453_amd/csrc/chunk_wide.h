// The wide tile kernel: four waves of 16 RT query rows each share every 64 (latent: 32) tokens of K and V
// in LDS.
//
// LDS holds bf16 rows of 16-byte chunks.  bf16 rows go there straight from memory (each lane of a load picks
// its source, so the swizzle costs nothing), other types pass through registers, where they are widened.
// Operands of S^T = K Q^T are 16-byte reads of a row; those of O^T = V^T P^T are transposing reads of four
// tokens by 16 channels.  Chunk c of token t lies at place c ^ f(t) of its row (f: `swizzle`), which spreads the 16
// rows that a K read touches, and the 8 rows of half a V read, over all banks.
// Two buffers: the next tokens travel while the present ones are multiplied.
#pragma once
#include "chunk_tile.h"

namespace vx {
namespace chunk {

typedef __attribute__((address_space(3))) uint8_t lds_u8;
__device__ __forceinline__ uint32_t lds_address(const uint8_t* p) { return (uint32_t)(uintptr_t)(lds_u8*)p; }
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short v4i16_t;

// One direct-to-LDS load: lane l's 16 bytes at base + off go to LDS address lds + 16 l.  In assembly, for the
// compiler would wait for loads that it sees before every read of LDS; `land_run` waits instead.  M0 holds the
// LDS address; the compiler reserves it, so its value is saved and restored here.
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

// A barrier that completes this wave's LDS accesses first.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Place of a row's chunks: XOR within groups of 16 (D = 128) or 8 chunks.
template <int D>
__device__ __forceinline__ int swizzle(int token) {
  if constexpr (D == 128) return ((token & 7) << 1) | ((token >> 3) & 1);
  else return (((token >> 1) & 3) << 1) | ((token >> 3) & 1);
}

template <int D, int DV, int KT>
struct Wide {
  static constexpr bool kAlias = D != DV;
  static constexpr int TK = kAlias ? 32 : 64;            // tokens of a buffer
  static constexpr int UNITS = TK / 16;                  // runs of 16 tokens
  static constexpr int CH = D / 8;                       // chunks of a row
  static constexpr int WPU = 4 / UNITS;                  // waves that load a run
  static constexpr int NI = 16 * CH / 64 / WPU;          // 64-chunk pieces of a wave
  static constexpr int TILE = TK * D * 2;                // bytes of K
  static constexpr int BUF = kAlias ? TILE : 2 * TILE;
};

// Element chunk of lane `lane` in piece k of the wave's part of a run: token and logical chunk.
template <int D, int DV, int KT>
__device__ __forceinline__ void piece(int wave, int k, int lane, int& token, int& c) {
  using G = Wide<D, DV, KT>;
  const int slot = 64 * ((wave % G::WPU) * G::NI + k) + lane;
  token = slot / G::CH;
  c = (slot % G::CH) ^ swizzle<D>(token);
}

// A wave's pieces of a run on their way through registers (types below 16 bits).
template <int D, int DV, int KT>
struct Travel {
  static constexpr int N = Wide<D, DV, KT>::NI;
  uint2 k[N], v[Wide<D, DV, KT>::kAlias ? 1 : N];        // mxfp4: codes and scale
};

// Starts a run's way into the buffer (bf16), or into registers.  t: its first token's place in the page.
template <int D, int DV, int KT>
__device__ __forceinline__ void send_run(const ChunkArgs& a, const uint8_t* ks, const uint8_t* vs, int t, int wave,
                                         int lane, uint8_t* buf, Travel<D, DV, KT>& r) {
  using G = Wide<D, DV, KT>;
  const int unit = wave / G::WPU;
#pragma unroll
  for (int k = 0; k < G::NI; k++) {
    int token, c;
    piece<D, DV, KT>(wave, k, lane, token, c);
    if constexpr (KT == kKvBf16) {
      const uint32_t dst = lds_address(buf) + unit * 16 * D * 2 + 1024 * ((wave % G::WPU) * G::NI + k);
      const uint32_t at = 2 * (token * D + 8 * c);
      send16(ks + 2 * t * D, at, dst);
      if constexpr (!G::kAlias) send16(vs + 2 * t * D, at, dst + G::TILE);
    } else if constexpr (KT == kKvMxFp4) {
      const int base = mx::codes_bytes(a.ps, D);
      r.k[k] = make_uint2(*reinterpret_cast<const uint32_t*>(ks + mx::k_code(t + token, c, D)),
                          ks[base + mx::k_scale(t + token, c >> 2, D)]);
      r.v[k] = make_uint2(mx::get_v_codes(vs, t + token, c, D), vs[base + mx::v_scale(t + token, c >> 2, D)]);
    } else {
      const int at = (t + token) * D + 8 * c;
      r.k[k] = *reinterpret_cast<const uint2*>(ks + at);
      if constexpr (!G::kAlias) r.v[k] = *reinterpret_cast<const uint2*>(vs + at);
    }
  }
}

template <int KT>
__device__ __forceinline__ uint4 widen_chunk(const uint2& w) {
  if constexpr (KT == kKvMxFp4) {
    const float s = mx::scale_operand(w.y);
    return make_uint4(mx::pair_bf16<0>(w.x, s), mx::pair_bf16<1>(w.x, s), mx::pair_bf16<2>(w.x, s), mx::pair_bf16<3>(w.x, s));
  } else {
    return make_uint4(fp8_pair<KT, false>(w.x), fp8_pair<KT, true>(w.x), fp8_pair<KT, false>(w.y), fp8_pair<KT, true>(w.y));
  }
}

// Ends it: widened rows into the buffer, and V rows of tokens that lie behind every row's last (from `left` tokens
// into the run on) set to zero, for they may hold anything.
template <int D, int DV, int KT>
__device__ __forceinline__ void land_run(int wave, int lane, int left, uint8_t* buf, const Travel<D, DV, KT>& r) {
  using G = Wide<D, DV, KT>;
  const int unit = wave / G::WPU;
  if constexpr (KT != kKvBf16) {
#pragma unroll
    for (int k = 0; k < G::NI; k++) {
      uint8_t* dst = buf + unit * 16 * D * 2 + 1024 * ((wave % G::WPU) * G::NI + k) + 16 * lane;
      *reinterpret_cast<uint4*>(dst) = widen_chunk<KT>(r.k[k]);
      if constexpr (!G::kAlias) *reinterpret_cast<uint4*>(dst + G::TILE) = widen_chunk<KT>(r.v[k]);
    }
  } else {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }
  if (left < 16) {
    for (int k = 0; k < G::NI; k++) {
      int token, c;
      piece<D, DV, KT>(wave, k, lane, token, c);
      uint8_t* dst = buf + unit * 16 * D * 2 + 1024 * ((wave % G::WPU) * G::NI + k) + 16 * lane + (G::kAlias ? 0 : G::TILE);
      if (token >= left) *reinterpret_cast<uint4*>(dst) = make_uint4(0, 0, 0, 0);
    }
  }
}

// Operand A of S^T: 16 tokens from t0, k-step kk (channels 32 kk + 8 grp ..).
template <int D>
__device__ __forceinline__ bf16x8_t k_from_lds(const uint8_t* tile, int t0, int kk, int col, int grp) {
  const int token = t0 + col, c = (4 * kk + grp) ^ swizzle<D>(col);
  return *reinterpret_cast<const bf16x8_t*>(tile + token * D * 2 + 16 * c);
}

// Operand A of O^T: channels 16 j + col of tokens t0 + 4 grp + 0..3 and t0 + 16 + 4 grp + 0..3.  Lane 4 r + x of
// 16 reads channels 4 x .. 4 x + 3 of row r; the transposing read gives it channel `lane` of the four rows.
template <int D>
__device__ __forceinline__ bf16x8_t v_from_lds(const uint8_t* tile, int t0, int j, int col, int grp) {
  const int row = 4 * grp + (col >> 2), x = col & 3;
  const int c = (2 * j + (x >> 1)) ^ swizzle<D>(row);
  lds_u8* p = (lds_u8*)(tile + (t0 + row) * D * 2 + 16 * c + 8 * (x & 1));
  const v4i16_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16_t*)p);
  const v4i16_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16_t*)(p + 16 * D * 2));
  typedef short s16x8_t __attribute__((ext_vector_type(8)));
  const s16x8_t w = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return __builtin_bit_cast(bf16x8_t, w);
}

}  // namespace chunk
}  // namespace vx
