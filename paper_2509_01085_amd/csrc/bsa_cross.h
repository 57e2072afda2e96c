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

// The arguments of a call where the kernel finds them: a piece of work loads what it needs from there.  By value, all of them would sit
// in scalar registers for the whole kernel, or in lanes of vector registers when those run out.
using Args = const __attribute__((address_space(4))) CrossArgs;
__device__ inline Args* kernel_args() {
#ifdef __HIP_DEVICE_COMPILE__
  return (Args*)__builtin_amdgcn_kernarg_segment_ptr();  // CrossArgs is every kernel's first argument
#else
  return nullptr;
#endif
}
__device__ inline Args* afresh(Args* a) {
  asm volatile("" : "+s"(a));
  return a;
}

// A lane number that the compiler takes for a new one: what a piece of work computes from it is not kept for the next.
__device__ inline int afresh(int lane) {
  asm volatile("" : "+v"(lane));
  return lane;
}

// A value that is the same in all lanes, in a scalar register.
__device__ inline int same(int v) { return __builtin_amdgcn_readfirstlane(v); }

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
  static constexpr int CE = 4;
  static __device__ inline Frag zero() { return f32x4{0.f, 0.f, 0.f, 0.f}; }
  static __device__ inline void mma(f32x16& d, const Frag& a, const Frag& b) {
#pragma unroll
    for (int i = 0; i < 4; ++i) d = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], d, 0, 0, 0);
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
  // bf16: rows row0 + 8 (t / 4) + 4 grp + t % 4, t = 0..7, of channel 32 dt + col; row0 a multiple of 16
  __device__ inline auto along(const uint8_t* tile, int row0, int dt) const {
    const int grp = lane >> 5, L16 = lane & 15, q16 = lane >> 4, rsub = L16 >> 2, jj = L16 & 3, cl = 2 * (q16 & 1) + (jj >> 1);
    const int r = row0 + 4 * grp + rsub, c = 4 * dt + cl;
    const uint8_t* p0 = tile + r * RB + ((c ^ tile_swz<T, DP>(r)) << 4) + 8 * (jj & 1);
    const uint8_t* p1 = tile + (r + 8) * RB + ((c ^ tile_swz<T, DP>(r + 8)) << 4) + 8 * (jj & 1);
    return typename E::Frag8{lds_frag_tr(p0, p1)};
  }
  // D[dt] += channels 32 dt .. 32 dt + 31 of rows row0 .. row0 + 31 (a multiple of 32) times x, whose element r stands for row d_row(r).
  // fp32: a value is one product's operand, and a product takes no longer than a value from LDS.  They run eight ahead of the products,
  // neighbours of which add to different accumulators.  (Row r has its chunks at c ^ (8 grp | r % 8): the address of row
  // 16 h + 8 a + 4 grp + e is that of 8 a + 4 grp + e and a constant, and a channel tile an exclusive or of bit 7 and a constant.)
  // With the reads where the compiler puts them, one ahead of each product, dK and dV of 2,520 queries took 172 us instead of 127.
  __device__ inline void gather(f32x16 (&acc)[DP / 32], const uint8_t* tile, int row0, const f32x16& x) const {
    constexpr int DT = DP / 32;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const auto b = E::column(x, h);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) E::mma8(acc[dt], along(tile, row0 + 16 * h, dt), b);
      }
    } else {
      constexpr int AHEAD = 8, N = 16 * DT;
      const int grp = lane >> 5, col = lane & 31;
      int at[8];
#pragma unroll
      for (int t = 0; t < 8; ++t)
        at[t] = row0 * RB + (8 * (t >> 2) + 4 * grp + (t & 3)) * RB + ((((col >> 2) ^ (t & 7)) | (grp << 3)) << 4) + 4 * (col & 3);
      auto value = [&](int n) {
        const int r = n / DT, dt = n % DT;
        return *reinterpret_cast<const float*>(tile + (at[r & 7] ^ ((dt & 1) << 7)) + (r >> 3) * 16 * RB + (dt >> 1) * 256);
      };
      float f[AHEAD];
#pragma unroll
      for (int n = 0; n < AHEAD; ++n) f[n] = value(n);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < N; ++n) {
        acc[n % DT] = __builtin_amdgcn_mfma_f32_32x32x2f32(f[n % AHEAD], x[n / DT], acc[n % DT], 0, 0, 0);
        if (n + AHEAD < N) f[n % AHEAD] = value(n + AHEAD);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
};

// The fragments of a bf16 tile by LDS byte offset, so that the tile's place folds into the instruction: AT is the tile's offset from
// `base`.
template <int D>
struct Fragments {
  static constexpr int RB = D * 2, DT = D / 32, DS = D / 16;
  int koffs[DS], voffs[2][DT];
  __device__ inline Fragments(uint32_t base, int lane) {
    const int grp = lane >> 5, col = lane & 31;
#pragma unroll
    for (int s = 0; s < DS; ++s) koffs[s] = base + col * RB + (((2 * s + grp) ^ swz<D>(col)) << 4);
    const int L16 = lane & 15, q16 = lane >> 4, rsub = L16 >> 2, jj = L16 & 3;
    const int cl = 2 * (q16 & 1) + (jj >> 1), rhi = D == 128 ? rsub : (rsub >> 1);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        voffs[h][dt] = base + (8 * h + 4 * grp + rsub) * RB + ((((dt ^ rhi) << 2) | (cl ^ (2 * h + grp))) << 4) + 8 * (jj & 1);
  }
  __device__ inline void move(int by) {
#pragma unroll
    for (int s = 0; s < DS; ++s) koffs[s] += by;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) voffs[h][dt] += by;
  }
  template <int AT> __device__ inline bf16x8 row(int row0, int s) const { return frag_at(koffs[s] + AT + row0 * RB); }
  template <int AT> __device__ inline bf16x8 along(int row0, int dt) const { return frag_tr_at(voffs[0][dt] + AT + row0 * RB, voffs[1][dt] + AT + row0 * RB); }
};

// What rows and channels that do not exist read instead.
__device__ __constant__ const uint4 kZeroChunk = {0, 0, 0, 0};

// Requests tiles of ROWS rows from a tensor whose row r starts at base + r * stride (elements).  All NT threads of the workgroup
// take part; counted by vmcnt.  Chunks from channel d on are never requested: clear() zeroes them once.
template <typename T, int DP, int ROWS, int NT>
struct Requests {
  using V = TileView<T, DP>;
  static constexpr int N = ROWS * V::CPR / NT;  // requests of a thread
  static_assert(ROWS * V::CPR % NT == 0, "whole requests");
  // The rows of the next instruction are a scalar step on, and where they are 16 or a multiple, the swizzle is the same.
  static constexpr bool STEPS = NT / V::CPR % 16 == 0;
  uint32_t off;  // byte offset from the tile's first row; not used unless all fit (near)
  int64_t step;
  int tid, d;
  __device__ inline int row(int n) const { return (n * NT + tid) / V::CPR; }
  __device__ inline int channel(int n) const { return (((n * NT + tid) % V::CPR) ^ tile_swz<T, DP>(row(n))) * V::E::CE; }
  __device__ inline Requests(int64_t stride, int d_, int tid_) : step(NT / V::CPR * stride * (int64_t)sizeof(T)), tid(tid_), d(d_) {
    off = (uint32_t)((row(0) * stride + channel(0)) * (int64_t)sizeof(T));
  }
  __device__ __forceinline__ void clear(uint8_t* tile) const {
#pragma unroll
    for (int n = 0; n < N; ++n)
      if (channel(n) >= d) *reinterpret_cast<u32x4*>(tile + (n * NT + tid) * 16) = u32x4{0, 0, 0, 0};
  }
  // All rows of the tile are there and offsets fit: no arithmetic for a lane.
  __device__ __forceinline__ void whole(uint8_t* tile, const T* base) const {
    const uint64_t sbase = uniform64(base);
    const uint32_t lds = uniform_lds(tile + (tid >> 6) * 1024);
#pragma unroll
    for (int n = 0; n < N; ++n)
      if (channel(n) < d) {
        const uint64_t from = uniform64((const void*)(sbase + n * step));  // (behind a condition of the lane's, and still the same for all)
        dma16_raw(from, STEPS ? off : off + (channel(n) - channel(0)) * (int)sizeof(T), same(lds + n * NT * 16));
      }
  }
  // The first `left` rows are there (offsets fit).  The others' weights are zero: the last row stands in for them, or (ZEROS) zeros, so that
  // an infinity of its own makes no NaN.  (Zeros written here: 492 of 512 states, 33,280 queries, 12 heads 141 us, requested from a chunk of zeros
  // 142, the last row 139.)
  template <bool ZEROS>
  __device__ __forceinline__ void cut(uint8_t* tile, const T* base, int64_t stride, int left) const {
    const uint64_t sbase = uniform64(base);
    const uint32_t lds = uniform_lds(tile + (tid >> 6) * 1024), step = (uint32_t)(stride * (int64_t)sizeof(T));
#pragma unroll
    for (int n = 0; n < N; ++n)
      if (channel(n) < d) {
        if (!ZEROS || row(n) < left)
          dma16_raw(uniform64((const void*)sbase), min(row(n), left - 1) * step + channel(n) * (uint32_t)sizeof(T), same(lds + n * NT * 16));
        else *reinterpret_cast<u32x4*>(tile + (n * NT + tid) * 16) = u32x4{0, 0, 0, 0};
      }
  }
  // Rows whose bit in `there` is not set arrive as zeros.
  __device__ __forceinline__ void some(uint8_t* tile, const T* base, int64_t stride, uint64_t there) const {
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
#pragma unroll 1
    for (int n = 0; n < N; ++n) {
      const int r = row(n), ch = channel(n);
      const void* src = ((there >> r) & 1) && ch < d ? (const void*)(base + r * stride + ch) : (const void*)&kZeroChunk;
      dma16(src, tile + (n * NT + wave * 64) * 16);
    }
  }
  template <bool ZEROS = false>
  __device__ __forceinline__ void load(uint8_t* tile, const T* base, int64_t stride, uint64_t there, bool near) const {
    if (near && there == (ROWS == 64 ? ~0ull : (1ull << ROWS) - 1)) whole(tile, base);
    else if (near && there && !(there & (there + 1))) cut<ZEROS>(tile, base, stride, __popcll(there));
    else some(tile, base, stride, there);
  }
};

// Which of the KT keys from `first` on are valid, as bits.
struct Keys {
  int n;                 // valid length (b is the same for all lanes: a scalar load)
  const uint8_t* mask;   // the batch entry's, or NULL
  __device__ inline Keys(Args& a, int b) : n(a.kv_len ? max(0, min(((const __attribute__((address_space(4))) int32_t*)a.kv_len)[b], a.S)) : a.S), mask(a.kv_mask ? a.kv_mask + (int64_t)b * a.S : nullptr) {}
  __device__ inline uint64_t bits(int first, int count, int lane) const {
    if (!mask) {  // (uniform: a length alone)
      const int left = n - first;
      return left >= count ? (count == 64 ? ~0ull : (1ull << count) - 1) : left <= 0 ? 0 : (1ull << left) - 1;
    }
    // (The load is waited for here.  Asked for a tile ahead, or 64 tiles ahead, it cost every walk more than masks gained by it.)
    const int s = first + lane;
    const bool in = lane < count && s < n;
    const uint8_t m = mask[in ? s : 0];
    return __ballot(in && m != 0);
  }
};

// The 16 registers of a D tile hold rows 8 (r / 4) + 4 grp + r % 4.
__device__ inline constexpr int d_row(int r) { return 8 * (r / 4) + (r % 4); }

// Four adjacent channels.
__device__ inline void store4(uint16_t* p, f32x4 v) { *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])}; }
__device__ inline void store4(float* p, f32x4 v) { *reinterpret_cast<f32x4*>(p) = v; }

// The column of a [DT x 32 channels][32 columns] accumulator as a row of d channels at p.  A lane has four channels of every
// eight and its partner (lane ^ 32) the other four; for bf16 the two exchange them, so that each stores 16 bytes.
template <typename T, int DT>
__device__ inline void store_column(T* p, const f32x16 (&acc)[DT], float scale, int d, int grp, bool live) {
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {  // channels 16 k .. + 15 of the tile: this lane 8 grp .. + 7
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_bf16(acc[dt][8 * k + 2 * i] * scale, acc[dt][8 * k + 2 * i + 1] * scale);
        const auto x = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), y = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
        const int ch = 32 * dt + 16 * k + 8 * grp;
        if (live && ch < d) *reinterpret_cast<u32x4*>(p + ch) = u32x4{x[0], y[0], x[1], y[1]};
      }
    } else {
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const int ch = 32 * dt + 8 * r4 + 4 * grp;
        if (live && ch < d) store4(p + ch, f32x4{acc[dt][4 * r4], acc[dt][4 * r4 + 1], acc[dt][4 * r4 + 2], acc[dt][4 * r4 + 3]} * scale);
      }
    }
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

constexpr int kWaves = 4, kThreads = 64 * kWaves;

// ---- how a launch's work is dealt out ----
// A unit (128 query rows of one key head; dK and dV: a tile of keys) takes a number of steps (key tiles; query tiles).
//   EACH    workgroup n takes unit n;
//   SHARES  all steps of a launch, unit after unit, are cut into equal shares: a workgroup's first and last piece may then
//           be parts of a unit, whose fp32 results it leaves for a second launch that adds them up in order.  Keeps the chip
//           full where units are few, long or (valid lengths) unlike.
// (Runs of whole units, dealt out ahead of time, were slower than the hardware's handing out of single ones: 33,280 rows, 12 heads,
// 512 keys, forward 151 and 159 us.)
enum { EACH = 0, SHARES = 1 };
struct Deal {
  int grid;     // workgroups
  int way;
  int by_keys;  // units are tiles of `tile` keys and take `steps` steps; else `rows` units an entry of a step per `tile` valid keys
  int tile, steps;
  int rows;     // units of a batch entry: (by_keys) of S keys
};  // (all steps of a launch together: less than 2^31, the host has made sure)

struct Ledger {
  const Deal& dl;
  const int* len;
  int B, S, Hkv, lane;
  __device__ inline Ledger(Args& a, const Deal& dl_, int lane_) : dl(dl_), len(a.kv_len), B(a.B), S(a.S), Hkv(a.Hkv), lane(lane_) {}
  __device__ inline int valid(int b) const { return len ? max(0, min(len[b], S)) : S; }  // b may differ from lane to lane
  __device__ inline int tiles(int b) const { return (int)((uint32_t)(valid(b) + dl.tile - 1) / (uint32_t)dl.tile); }
  __device__ inline int steps(int b) const { return dl.by_keys ? dl.steps : tiles(b); }
  __device__ inline int units(int b) const { return dl.by_keys ? Hkv * tiles(b) : dl.rows; }  // that take steps
  __device__ inline int weight(int b) const { return units(b) * steps(b); }
  __device__ inline int scan(int v) const {  // inclusive, over the lanes
    const int lane = afresh(this->lane);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int w = __shfl_up(v, o);
      if (lane >= o) v += w;
    }
    return v;
  }
  // Steps of all entries; `below`: of those below b.
  __device__ inline int total(int b, int& below) const {
    if (!len) {
      const int w = weight(0);
      below = b * w;
      return B * w;
    }
    int sum = 0;
    for (int b0 = 0; b0 < B; b0 += 64) {
      const int v = b0 + lane < B ? weight(b0 + lane) : 0, to = scan(v);
      if (b >= b0 && b < b0 + 64) below = sum + same(__shfl(to - v, b - b0));
      sum += same(__shfl(to, 63));
    }
    return sum;
  }
  // The entry that step `pos` is of, and the step that it begins with.
  __device__ inline int entry(int pos, int& base) const {
    if (!len) {
      const int w = weight(0), b = (int)((uint32_t)pos / (uint32_t)w);
      base = b * w;
      return b;
    }
    base = 0;
    for (int b0 = 0;; b0 += 64) {
      const int v = b0 + lane < B ? weight(b0 + lane) : 0, to = scan(v);
      const uint64_t past = __ballot(base + to > pos);
      if (past || b0 + 64 >= B) {
        const int l = same(__builtin_ctzll(past | (1ull << 63)));
        base += same(__shfl(to - v, l));
        return b0 + l;
      }
      base += same(__shfl(to, 63));
    }
  }
};

// One piece of a workgroup's work: steps t0 .. t1 - 1 of a unit.
struct Piece {
  int b, t0, t1;
  int unit;   // of the entry
  int slot;   // of its partial results; -1: the unit is whole
};

// A workgroup's pieces, one after the other.  ONE: EACH, so there is one.
template <bool ONE>
struct Dealer {
  const Ledger led;
  int pos, end, units, unit, b, t, steps;
  bool fresh;  // no piece taken yet
  __device__ inline Dealer(Args& a, const Deal& dl, int lane) : led(a, dl, lane), t(0), fresh(true) {
    if constexpr (ONE) {
      b = (int)(blockIdx.x / (uint32_t)dl.rows);
      unit = (int)blockIdx.x - b * dl.rows;
      steps = same(led.steps(b));
      return;
    }
    int none = 0;
    const int total = led.total(-1, none), per = (int)((uint32_t)(total + dl.grid - 1) / (uint32_t)dl.grid);
    pos = min((int)blockIdx.x * per, total);  // (grid * per < total + grid)
    end = min(pos + per, total);
    if (pos >= end) return;
    const int base = enter();
    unit = (int)((uint32_t)(pos - base) / (uint32_t)steps);
    t = pos - base - unit * steps;
  }
  __device__ inline int enter() {
    int base;
    b = led.entry(pos, base);
    steps = same(led.steps(b));
    units = same(led.units(b));
    unit = 0;
    return base;
  }
  __device__ inline bool next(Piece& pc) {
    if constexpr (ONE) {
      pc = Piece{b, 0, steps, unit, -1};
      return true;
    }
    if (pos >= end) return false;
    if (unit >= units) enter();
    pc.b = b;
    pc.unit = unit;
    pc.t0 = t;
    pc.t1 = min(steps, t + (end - pos));
    pc.slot = t == 0 && pc.t1 == steps ? -1 : 2 * (int)blockIdx.x + !fresh;
    pos += pc.t1 - t;
    t = 0;  // (a share ends in a unit's middle or goes on with the next unit)
    ++unit;
    fresh = false;
    return true;
  }
};

// The partial results of a unit of entry b: how many there are (0: the unit is whole, -1: nobody worked on it) and their slots.
struct Parts {
  int n, per, first, w0;
  __device__ inline Parts(Args& a, const Deal& dl, int lane, int b, int unit) : n(-1), per(0), first(0), w0(0) {
    const Ledger led(a, dl, lane);
    const int steps = same(led.steps(b));
    if (dl.way != SHARES || steps == 0 || unit >= same(led.units(b))) return;
    int below = 0;
    const int total = led.total(b, below);
    per = (int)((uint32_t)(total + dl.grid - 1) / (uint32_t)dl.grid);
    first = below + unit * steps;
    w0 = (int)((uint32_t)first / (uint32_t)per);
    n = (int)((uint32_t)(first + steps - 1) / (uint32_t)per) - w0;
    if (n) ++n;
  }
  __device__ inline int slot(int k) const { return 2 * (w0 + k) + ((w0 + k) * per < first); }
};

// Partial results: [slot][wavefront][value][lane] floats.
template <int VALUES>
__device__ inline float* part_of(float* base, int slot, int wave, int lane) {
  return base + (((int64_t)slot * kWaves + wave) * VALUES) * 64 + lane;
}

// The query tiles of dK and dV: 32 tokens of a head from first_token(i) on; where the last one would reach past Lq it begins
// earlier and the tokens that it shares with its neighbour weigh nothing in it.
__host__ __device__ inline int query_tiles(int Lq) { return (Lq + 31) / 32; }
__host__ __device__ inline int first_token(int Lq, int i) { return Lq < 32 ? 0 : (32 * i < Lq - 32 ? 32 * i : Lq - 32); }

// dK and dV of bf16 tensors with d <= 128 and Lq >= 32 (bsa_cross_dkv.hip); stat: the row statistics that the dQ launch left.
size_t cross_dkv_fast_parts(const CrossArgs& a);
int grant_cross_dkv_fast(const CrossArgs& a);  // before any launch of the call
int launch_cross_dkv_fast(const CrossArgs& a, const float* stat, float* part, hipStream_t st);

}  // namespace bsa
