// Building blocks of the cross-attention kernels: fragments of fp32 and bf16 tiles for the 32 x 32 matrix-core products, tiles
// of strided tensors, valid keys.
//
// As everywhere in this library the product's D tile has the query (dK, dV: the key) on its column, which is a lane pair, and a
// D tile is the B operand of the next contraction as it stands.  bf16: v_mfma_f32_32x32x16_bf16 (bsa_mfma.h).  fp32:
// v_mfma_f32_32x32x2_f32, lane (col, grp) holds element grp of the contraction's pair; a 16-byte fragment (four channels a
// lane) feeds four of them.
#pragma once

#include "bsa_mfma.h"

namespace bsa {

// ---- element types ----
template <typename T> struct Elt;
template <> struct Elt<uint16_t> {
  using Frag = bf16x8;   // 16 bytes of a row: channels 8 chunk ..
  struct Frag8 { bf16x8 v; };  // eight rows (contraction slots) of a channel, or of a D tile's column
  static constexpr int CE = 8;  // elements of a 16-byte chunk
  static __device__ inline Frag zero() { return as_frag(u32x4{0, 0, 0, 0}); }
  static __device__ inline void mma(f32x16& d, const Frag& a, const Frag& b) { d = mfma32(a, b, d); }
  static __device__ inline void mma8(f32x16& d, const Frag8& a, const Frag8& b) { d = mfma32(a.v, b.v, d); }
  static __device__ inline Frag8 column(const f32x16& d, int h) { return {d_to_b(d, h)}; }  // registers 8 h ..: rounded to bf16
  static __device__ inline float dot(const Frag& a, const Frag& b) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = __builtin_fmaf((float)a[i], (float)b[i], s);
    return s;
  }
};
template <> struct Elt<float> {
  using Frag = f32x4;
  struct Frag8 { float v[8]; };
  static constexpr int CE = 4;
  static __device__ inline Frag zero() { return f32x4{0.f, 0.f, 0.f, 0.f}; }
  static __device__ inline void mma(f32x16& d, const Frag& a, const Frag& b) {
#pragma unroll
    for (int i = 0; i < 4; ++i) d = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], d, 0, 0, 0);
  }
  static __device__ inline void mma8(f32x16& d, const Frag8& a, const Frag8& b) {
#pragma unroll
    for (int i = 0; i < 8; ++i) d = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[i], b.v[i], d, 0, 0, 0);
  }
  static __device__ inline Frag8 column(const f32x16& d, int h) {
    Frag8 f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f.v[i] = d[8 * h + i];
    return f;
  }
  static __device__ inline float dot(const Frag& a, const Frag& b) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) s = __builtin_fmaf(a[i], b[i], s);
    return s;
  }
};

// ---- LDS tiles: rows of DP channels, chunk c of row r at chunk position c ^ swizzle(r) ----
// bf16: see bsa_mfma.h.  fp32: row fragments want the 16 rows of a pass at 16 chunk positions; the reads along a channel take rows
// r and r + 4 at once, which bit 3 keeps in different halves of the 64 banks.
template <typename T, int DP>
__device__ inline int tile_swz(int r) {
  if (sizeof(T) == 4) return ((r & 4) << 1) | ((r & 8) >> 1) | (r & 3);
  return swz<(DP == 64 ? 64 : 128)>(r);
}

template <typename T, int DP>
struct TileView {
  using E = Elt<T>;
  static constexpr int RB = DP * (int)sizeof(T);
  static constexpr int CPR = RB / 16;
  int lane;
  __device__ inline explicit TileView(int lane_) : lane(lane_) {}
  // chunk 2 s + grp of row `row` + col
  __device__ inline typename E::Frag row(const uint8_t* tile, int row0, int s) const {
    const int r = row0 + (lane & 31), c = 2 * s + (lane >> 5);
    return *reinterpret_cast<const typename E::Frag*>(tile + r * RB + ((c ^ tile_swz<T, DP>(r)) << 4));
  }
  // rows row0 + 16 h + 8 (t / 4) + 4 grp + t % 4, t = 0..7, of channel 32 dt + col; row0 a multiple of 16
  __device__ inline typename E::Frag8 along(const uint8_t* tile, int row0, int dt) const {
    const int grp = lane >> 5;
    if constexpr (sizeof(T) == 2) {
      const int L16 = lane & 15, q16 = lane >> 4, rsub = L16 >> 2, jj = L16 & 3, cl = 2 * (q16 & 1) + (jj >> 1);
      const int r = row0 + 4 * grp + rsub, c = 4 * dt + cl;
      const uint8_t* p0 = tile + r * RB + ((c ^ tile_swz<T, DP>(r)) << 4) + 8 * (jj & 1);
      const uint8_t* p1 = tile + (r + 8) * RB + ((c ^ tile_swz<T, DP>(r + 8)) << 4) + 8 * (jj & 1);
      return {lds_frag_tr(p0, p1)};
    } else {
      typename E::Frag8 f;
      const int ch = 32 * dt + (lane & 31);
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const int r = row0 + 8 * (t >> 2) + 4 * grp + (t & 3);
        f.v[t] = *reinterpret_cast<const float*>(tile + r * RB + (((ch >> 2) ^ tile_swz<T, DP>(r)) << 4) + 4 * (ch & 3));
      }
      return f;
    }
  }
};

// What rows and channels that do not exist read instead.
__device__ __constant__ const uint4 kZeroChunk = {0, 0, 0, 0};

// Requests a tile of ROWS rows from a tensor whose row r starts at base + r * stride (elements); rows whose bit in `there` is
// not set, and channels from d on, arrive as zeros.  All NT threads of the workgroup take part; counted by vmcnt.
template <typename T, int DP, int ROWS, int NT>
__device__ inline void request_tile(uint8_t* tile, const T* base, int64_t stride, uint64_t there, int d, int tid) {
  using V = TileView<T, DP>;
  constexpr int CHUNKS = ROWS * V::CPR;
  static_assert(CHUNKS % NT == 0, "whole requests");
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
#pragma unroll
  for (int n = 0; n < CHUNKS / NT; ++n) {
    const int i = n * NT + tid, r = i / V::CPR, c = (i % V::CPR) ^ tile_swz<T, DP>(r);
    const void* src = ((there >> r) & 1) && c * V::E::CE < d ? (const void*)(base + r * stride + c * V::E::CE) : (const void*)&kZeroChunk;
    dma16(src, tile + (n * NT + wave * 64) * 16);
  }
}

// Which of the KT keys from `first` on are valid, as bits.
struct Keys {
  int n;                 // valid length
  const uint8_t* mask;   // the batch entry's, or NULL
  __device__ inline Keys(const CrossArgs& a, int b) : n(a.kv_len ? max(0, min(a.kv_len[b], a.S)) : a.S), mask(a.kv_mask ? a.kv_mask + (int64_t)b * a.S : nullptr) {}
  __device__ inline uint64_t bits(int first, int count, int lane) const {
    const int s = first + lane;
    bool ok = lane < count && s < n;
    if (mask && ok) ok = mask[s] != 0;
    return __ballot(ok);
  }
};

// The 16 registers of a D tile hold rows 8 (r / 4) + 4 grp + r % 4.
__device__ inline constexpr int d_row(int r) { return 8 * (r / 4) + (r % 4); }

// Four adjacent channels.
__device__ inline void store4(uint16_t* p, f32x4 v) { *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])}; }
__device__ inline void store4(float* p, f32x4 v) { *reinterpret_cast<f32x4*>(p) = v; }

// The column of a [DT x 32 channels][32 columns] accumulator as a row of d channels at p.
template <typename T, int DT>
__device__ inline void store_column(T* p, const f32x16 (&acc)[DT], float scale, int d, int grp) {
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const int ch = 32 * dt + 8 * r4 + 4 * grp;
      if (ch < d) store4(p + ch, f32x4{acc[dt][4 * r4], acc[dt][4 * r4 + 1], acc[dt][4 * r4 + 2], acc[dt][4 * r4 + 3]} * scale);
    }
}

template <typename T, int DT>
__device__ inline void store_zeros(T* p, int d, int grp) {
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const int ch = 32 * dt + 8 * r4 + 4 * grp;
      if (ch < d) store4(p + ch, f32x4{0.f, 0.f, 0.f, 0.f});
    }
}

}  // namespace bsa
