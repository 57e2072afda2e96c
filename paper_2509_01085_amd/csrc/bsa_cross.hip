// Cross attention: every query row attends to the valid states of an encoder.  Forward, dQ, and dK and dV, for fp32 and
// bf16, any head dimension up to 256.
//
// The G query heads that share keys are one matrix of M = G Lq rows, so shared heads cost nothing in the forward and dQ and
// their gradients come out summed.  A workgroup has four wavefronts of 32 rows (forward, dQ) or 32 keys (dK, dV); the other
// side's tiles stream through LDS in a ring of two, one barrier a tile.  Where there are few workgroups, the walk is split into
// segments whose fp32 partial results a second launch joins, in a fixed order.
#include <algorithm>

#include "bsa_cross.h"

namespace bsa {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kUnitRows = 32 * kWaves;

template <typename T> constexpr int key_tile() { return sizeof(T) == 2 ? 64 : 32; }

// A launch's work: `units` of kUnitRows rows (keys) each, walked in `nseg` segments of `per` tiles.
struct Plan {
  int tiles, nseg, per;
  int64_t units;
};

// Segments only where the units leave half of the chip's 512 workgroup slots empty, and of four tiles at least.
static Plan make_plan(int64_t units, int64_t tiles) {
  Plan p;
  p.units = units;
  p.tiles = (int)tiles;
  int64_t n = units * 2 > 512 ? 1 : std::min<int64_t>(512 / units, (tiles + 3) / 4);
  if (n < 1) n = 1;
  p.per = (int)((tiles + n - 1) / n);
  p.nseg = (int)((tiles + p.per - 1) / p.per);
  return p;
}
static int row_units(const CrossArgs& a) { return (a.M + kUnitRows - 1) / kUnitRows; }
static Plan rows_plan(const CrossArgs& a) {
  const int kt = a.dtype == BSA_F32 ? 32 : 64;
  return make_plan((int64_t)a.B * a.Hkv * row_units(a), (a.S + kt - 1) / kt);
}
static int query_tiles(const CrossArgs& a) { return (a.Lq + 31) / 32; }  // of a head
static Plan keys_plan(const CrossArgs& a) {
  return make_plan((int64_t)a.B * a.Hkv * ((a.S + kUnitRows - 1) / kUnitRows), (int64_t)a.G * query_tiles(a));
}
static int padded_d(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

// Partial results: [segment][unit][wavefront][value][lane] floats.
template <int VALUES>
__device__ inline float* part_of(float* base, int64_t units, int seg, int64_t unit, int wave, int lane) {
  return base + (((seg * units + unit) * kWaves + wave) * VALUES) * 64 + lane;
}

struct RowUnit {
  int64_t unit;
  int b, hk, m, g, l;  // batch entry, key head, row, its head in the group and token
  bool live;
  __device__ inline RowUnit(const CrossArgs& a, int64_t unit_, int wave, int lane, int units_of_head) : unit(unit_) {
    const int bh = (int)(unit / units_of_head);
    b = bh / a.Hkv;
    hk = bh - b * a.Hkv;
    m = (int)(unit - (int64_t)bh * units_of_head) * kUnitRows + 32 * wave + (lane & 31);
    live = m < a.M;
    g = live ? m / a.Lq : 0;
    l = live ? m - g * a.Lq : 0;
  }
  __device__ inline int head(const CrossArgs& a) const { return hk * a.G + g; }
  __device__ inline int64_t offset(const CrossArgs& a, const bsa_strides_t& s) const { return b * s.b + (int64_t)head(a) * s.h + (int64_t)l * s.l; }
  __device__ inline int64_t flat(const CrossArgs& a) const { return ((int64_t)b * a.H + head(a)) * a.Lq + l; }
};

// Chunk c of a row, zeros where there is none.
template <typename T>
__device__ inline typename Elt<T>::Frag row_chunk(const T* p, int c, bool live, int d) {
  const int ch = c * Elt<T>::CE;
  return live && ch < d ? *reinterpret_cast<const typename Elt<T>::Frag*>(p + ch) : Elt<T>::zero();
}

// The lane's own row (B operand), chunk 2 s + grp: in registers, or, where 256 channels would fill them, read again from the
// first-level cache at every use.
template <typename T, int DP, bool HELD>
struct RowFrags {
  using E = Elt<T>;
  static constexpr int DS = DP * sizeof(T) / 32;
  const T* p;
  bool live;
  int d, grp;
  typename E::Frag f[HELD ? DS : 1];
  __device__ inline RowFrags(const T* p_, bool live_, int d_, int grp_) : p(p_), live(live_), d(d_), grp(grp_) {
    if constexpr (HELD) {
#pragma unroll
      for (int s = 0; s < DS; ++s) f[s] = row_chunk(p, 2 * s + grp, live, d);
#pragma unroll
      for (int s = 0; s < DS; ++s) settle(f[s]);  // waited for here, not behind the first tile's requests
    }
  }
  // D += rows row0 .. row0 + 31 of the tile times this
  __device__ inline void times(f32x16& acc, const TileView<T, DP>& view, const uint8_t* tile, int row0) const {
    if constexpr (HELD) {
#pragma unroll
      for (int s = 0; s < DS; ++s) E::mma(acc, view.row(tile, row0, s), f[s]);
    } else {
      const int n = (d / E::CE + 1) / 2;
      for (int s = 0; s < n; s += 2)  // (the chunks past d are zeros on both sides)
#pragma unroll
        for (int i = 0; i < 2; ++i) E::mma(acc, view.row(tile, row0, s + i), row_chunk(p, 2 * (s + i) + grp, live, d));
    }
  }
  __device__ inline float dot(const T* other) const {
    float sum = 0.f;
    if constexpr (HELD) {
#pragma unroll
      for (int s = 0; s < DS; ++s) sum += E::dot(f[s], row_chunk(other, 2 * s + grp, live, d));
    } else {
      const int n = (d / E::CE + 1) / 2;
      for (int s = 0; s < n; ++s) sum += E::dot(row_chunk(p, 2 * s + grp, live, d), row_chunk(other, 2 * s + grp, live, d));
    }
    return sum;
  }
};
template <typename T, int DP> constexpr bool held() { return DP * sizeof(T) <= 512; }  // one row beside an accumulator of DP channels

// ---- forward ----
// O = 0 and LSE = -inf without a valid key; a row whose valid logits are all -inf has no softmax and is NaN.
template <typename T, int DT>
__device__ inline void finish_row(const CrossArgs& a, const RowUnit& u, const f32x16 (&acc)[DT], float m, float l, bool any, int grp) {
  if (!u.live) return;
  store_column<T, DT>(static_cast<T*>(a.O_out) + u.offset(a, a.o), acc, any ? 1.f / l : 0.f, a.d, grp);
  if (grp == 0) a.LSE_out[u.flat(a)] = any ? __builtin_fmaf(m, a.sm_scale, __builtin_amdgcn_logf(l) * kLn2) : -INFINITY;
}

template <typename T, int DP>
__global__ __launch_bounds__(kThreads, 1) void cross_fwd_kernel(CrossArgs a, Plan plan, int units_of_head, float* part) {
  using E = Elt<T>;
  constexpr int KT = key_tile<T>(), NK = KT / 32, DT = DP / 32, TILE = KT * DP * sizeof(T);
  extern __shared__ __align__(16) uint8_t smem[];  // [2][K tile | V tile]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), grp = lane >> 5;
  const int seg = (int)(blockIdx.x / plan.units);
  const RowUnit u(a, blockIdx.x % plan.units, wave, lane, units_of_head);
  const Keys keys(a, u.b);
  const TileView<T, DP> view(lane);
  const T* K = static_cast<const T*>(a.K) + u.b * a.k.b + u.hk * a.k.h;
  const T* V = static_cast<const T*>(a.V) + u.b * a.v.b + u.hk * a.v.h;

  const RowFrags<T, DP, held<T, DP>()> q(static_cast<const T*>(a.Q) + u.offset(a, a.q), u.live, a.d, grp);
  f32x16 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
  float m = -INFINITY, l = 0.f;
  const float c = a.sm_scale * kLog2e;
  bool any = false;
  const int t0 = seg * plan.per, t1 = min(t0 + plan.per, (keys.n + KT - 1) / KT);
  uint64_t bits = 0;
  auto request = [&](int t) -> uint64_t {
    const uint64_t there = keys.bits(t * KT, KT, lane);
    uint8_t* at = smem + (t & 1) * 2 * TILE;
    request_tile<T, DP, KT, kThreads>(at, K + (int64_t)t * KT * a.k.l, a.k.l, there, a.d, tid);
    request_tile<T, DP, KT, kThreads>(at + TILE, V + (int64_t)t * KT * a.v.l, a.v.l, there, a.d, tid);
    return there;
  };
  if (t0 < t1) bits = request(t0);
  for (int t = t0; t < t1; ++t) {
    wait_vm<0>();
    raw_barrier();
    const uint64_t now = bits;
    if (t + 1 < t1) bits = request(t + 1);
    if (now == 0) continue;
    any = true;
    const uint8_t* kt = smem + (t & 1) * 2 * TILE;
    const uint8_t* vt = kt + TILE;
    f32x16 s[NK];
#pragma unroll
    for (int k = 0; k < NK; ++k)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[k][r] = 0.f;
#pragma unroll
    for (int k = 0; k < NK; ++k) q.times(s[k], view, kt, 32 * k);
    if (now != (KT == 64 ? ~0ull : 0xffffffffull)) {
      const uint64_t own = now >> (4 * grp);
#pragma unroll
      for (int k = 0; k < NK; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (!((own >> (32 * k + d_row(r))) & 1)) s[k][r] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int k = 0; k < NK; ++k)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[k][r]);
    top = pair_max(top);
    if (__any(top > m)) {
      const float next = fmaxf(m, top);
      const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - next) * c);
      m = next;
      l *= f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] *= f;
    }
    const float base = m == -INFINITY ? 0.f : m * c;  // (all logits so far are -inf: they weigh nothing)
#pragma unroll
    for (int k = 0; k < NK; ++k)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[k][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[k][r], c, -base));
        l += s[k][r];
      }
#pragma unroll
    for (int k = 0; k < NK; ++k)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const auto p = E::column(s[k], h);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) E::mma8(o[dt], view.along(vt, 32 * k + 16 * h, dt), p);
      }
  }
  l = pair_sum(l);
  if (plan.nseg == 1) {
    finish_row<T, DT>(a, u, o, m, l, any, grp);
    return;
  }
  float* out = part_of<DT * 16 + 2>(part, plan.units, seg, u.unit, wave, lane);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) out[(dt * 16 + r) * 64] = o[dt][r];
  out[DT * 16 * 64] = m;
  out[(DT * 16 + 1) * 64] = any ? l : -1.f;  // (a sum is never negative)
}

template <typename T, int DP>
__global__ __launch_bounds__(kThreads) void cross_fwd_combine_kernel(CrossArgs a, Plan plan, int units_of_head, float* part) {
  constexpr int DT = DP / 32, VALUES = DT * 16 + 2;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const RowUnit u(a, blockIdx.x, wave, lane, units_of_head);
  const float c = a.sm_scale * kLog2e;
  float m = -INFINITY;
  bool any = false;
  for (int s = 0; s < plan.nseg; ++s) {
    const float* in = part_of<VALUES>(part, plan.units, s, u.unit, wave, lane);
    if (in[(DT * 16 + 1) * 64] == -1.f) continue;
    any = true;
    m = fmaxf(m, in[DT * 16 * 64]);
  }
  f32x16 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
  float l = 0.f;
  for (int s = 0; s < plan.nseg; ++s) {
    const float* in = part_of<VALUES>(part, plan.units, s, u.unit, wave, lane);
    const float ls = in[(DT * 16 + 1) * 64], ms = in[DT * 16 * 64];
    if (ls == -1.f) continue;
    const float f = ms == -INFINITY && ls == 0.f ? 0.f : __builtin_amdgcn_exp2f((ms - m) * c);
    l = __builtin_fmaf(ls, f, l);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[dt][r] = __builtin_fmaf(in[(dt * 16 + r) * 64], f, o[dt][r]);
  }
  finish_row<T, DT>(a, u, o, m, l, any, lane >> 5);
}

// ---- dQ ----
// dQ^T += K^T dS^T over the key tiles, S^T and dP^T recomputed.  Ahead of the walk each wavefront forms delta of its rows and leaves
// (LSE, -delta) for the other kernel: per head and 32 tokens [32] LSE log2(e), [32] -delta; tokens past the last
// have LSE = +inf, i.e. weights of zero.
template <typename T, int DP>
__global__ __launch_bounds__(kThreads, 1) void cross_dq_kernel(CrossArgs a, Plan plan, int units_of_head, float* stat, float* part) {
  using E = Elt<T>;
  constexpr int KT = key_tile<T>(), NK = KT / 32, DT = DP / 32, TILE = KT * DP * sizeof(T);
  extern __shared__ __align__(16) uint8_t smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), grp = lane >> 5;
  const int seg = (int)(blockIdx.x / plan.units);
  const RowUnit u(a, blockIdx.x % plan.units, wave, lane, units_of_head);
  const Keys keys(a, u.b);
  const TileView<T, DP> view(lane);
  const T* K = static_cast<const T*>(a.K) + u.b * a.k.b + u.hk * a.k.h;
  const T* V = static_cast<const T*>(a.V) + u.b * a.v.b + u.hk * a.v.h;

  const RowFrags<T, DP, held<T, DP>()> q(static_cast<const T*>(a.Q) + u.offset(a, a.q), u.live, a.d, grp);
  const RowFrags<T, DP, DP <= 128> gr(static_cast<const T*>(a.dO) + u.offset(a, a.go), u.live, a.d, grp);
  float delta = gr.dot(static_cast<const T*>(a.O) + u.offset(a, a.o));
  delta = pair_sum(delta);
  const float lse2 = u.live ? a.LSE_in[u.flat(a)] * kLog2e : INFINITY;
  if (seg == 0 && grp == 0 && u.live) {
    const int tiles = (a.Lq + 31) / 32;
    float* at = stat + (((int64_t)u.b * a.H + u.head(a)) * tiles + (u.l >> 5)) * 64;
    at[u.l & 31] = lse2;
    at[32 + (u.l & 31)] = -delta;
    if (u.l == a.Lq - 1)
      for (int i = (u.l & 31) + 1; i < 32; ++i) {
        at[i] = INFINITY;
        at[32 + i] = 0.f;
      }
  }

  f32x16 dq[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) dq[dt][r] = 0.f;
  const float c = a.sm_scale * kLog2e;
  const int t0 = seg * plan.per, t1 = min(t0 + plan.per, (keys.n + KT - 1) / KT);
  uint64_t bits = 0;
  auto request = [&](int t) -> uint64_t {
    const uint64_t there = keys.bits(t * KT, KT, lane);
    uint8_t* at = smem + (t & 1) * 2 * TILE;
    request_tile<T, DP, KT, kThreads>(at, K + (int64_t)t * KT * a.k.l, a.k.l, there, a.d, tid);
    request_tile<T, DP, KT, kThreads>(at + TILE, V + (int64_t)t * KT * a.v.l, a.v.l, there, a.d, tid);
    return there;
  };
  if (t0 < t1) bits = request(t0);
  for (int t = t0; t < t1; ++t) {
    wait_vm<0>();
    raw_barrier();
    const uint64_t now = bits;
    if (t + 1 < t1) bits = request(t + 1);
    if (now == 0) continue;
    const uint8_t* kt = smem + (t & 1) * 2 * TILE;
    const uint8_t* vt = kt + TILE;
    const uint64_t own = now >> (4 * grp);
    const bool whole = now == (KT == 64 ? ~0ull : 0xffffffffull);
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      f32x16 s, dp;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
      q.times(s, view, kt, 32 * k);
      gr.times(dp, view, vt, 32 * k);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -lse2));
      if (!whole)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (!((own >> (32 * k + d_row(r))) & 1)) s[r] = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] *= dp[r] - delta;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const auto ds = E::column(s, h);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) E::mma8(dq[dt], view.along(kt, 32 * k + 16 * h, dt), ds);
      }
    }
  }
  if (plan.nseg == 1) {
    if (u.live) store_column<T, DT>(static_cast<T*>(a.dQ) + u.offset(a, a.gq), dq, a.sm_scale, a.d, grp);
    return;
  }
  float* out = part_of<DT * 16>(part, plan.units, seg, u.unit, wave, lane);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) out[(dt * 16 + r) * 64] = dq[dt][r];
}

template <int DT>
__device__ inline void sum_parts(f32x16 (&acc)[DT], float* part, const Plan& plan, int64_t unit, int wave, int lane) {
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[dt][r] = 0.f;
  for (int s = 0; s < plan.nseg; ++s) {
    const float* in = part_of<DT * 16>(part, plan.units, s, unit, wave, lane);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[dt][r] += in[(dt * 16 + r) * 64];
  }
}

template <typename T, int DP>
__global__ __launch_bounds__(kThreads) void cross_dq_combine_kernel(CrossArgs a, Plan plan, int units_of_head, float* part) {
  constexpr int DT = DP / 32;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const RowUnit u(a, blockIdx.x, wave, lane, units_of_head);
  f32x16 dq[DT];
  sum_parts<DT>(dq, part, plan, u.unit, wave, lane);
  if (u.live) store_column<T, DT>(static_cast<T*>(a.dQ) + u.offset(a, a.gq), dq, a.sm_scale, a.d, lane >> 5);
}

// ---- dK, dV ----
// A wavefront owns 32 keys; dV^T += dO^T P and dK^T += Q^T dS over the query tiles (32 tokens of one head) of the heads that share them.
struct KeyUnit {
  int64_t unit;
  int b, hk, first, key;
  bool there;   // the lane's key exists
  __device__ inline KeyUnit(const CrossArgs& a, int64_t unit_, int wave, int lane, int units_of_head) : unit(unit_) {
    const int bh = (int)(unit / units_of_head);
    b = bh / a.Hkv;
    hk = bh - b * a.Hkv;
    first = (int)(unit - (int64_t)bh * units_of_head) * kUnitRows;
    key = first + 32 * wave + (lane & 31);
    there = key < a.S;
  }
};

// WHAT: both at once, or (256 channels, whose two accumulators would not leave the registers for the rows) dK and dV by workgroups of
// their own, which form S twice.
enum { BOTH = 0, ONLY_K = 1, ONLY_V = 2 };

template <typename T, int DP, int WHAT>
__device__ inline void dkv_walk(CrossArgs a, Plan plan, int units_of_head, const float* stat, float* part) {
  using E = Elt<T>;
  constexpr int DT = DP / 32, TILE = 32 * DP * sizeof(T), STAGE = 2 * TILE + 256;
  constexpr bool WITH_K = WHAT != ONLY_V, WITH_V = WHAT != ONLY_K;
  extern __shared__ __align__(16) uint8_t smem[];  // [2][Q tile | dO tile | LSE, -delta]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), grp = lane >> 5;
  const int seg = (int)(blockIdx.x / plan.units);
  const KeyUnit u(a, blockIdx.x % plan.units, wave, lane, units_of_head);
  const Keys keys(a, u.b);
  const TileView<T, DP> view(lane);
  const uint64_t mine = keys.bits(u.first + 32 * wave, 32, lane);                   // valid keys of the wavefront
  const bool valid = (mine >> (lane & 31)) & 1;
  const bool work = __syncthreads_or(mine != 0);                                   // of the workgroup
  const T* K = static_cast<const T*>(a.K) + u.b * a.k.b + u.hk * a.k.h + u.key * a.k.l;
  const T* V = static_cast<const T*>(a.V) + u.b * a.v.b + u.hk * a.v.h + u.key * a.v.l;
  const RowFrags<T, DP, held<T, DP>()> kf(K, valid, a.d, grp), vf(WITH_K ? V : K, valid, a.d, grp);
  f32x16 dk[WITH_K ? DT : 1], dv[WITH_V ? DT : 1];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      if (WITH_K) dk[dt][r] = 0.f;
      if (WITH_V) dv[dt][r] = 0.f;
    }
  const float c = a.sm_scale * kLog2e;
  const int tiles = (a.Lq + 31) / 32;  // of a head
  const int t0 = seg * plan.per, t1 = work ? min(t0 + plan.per, plan.tiles) : t0;
  auto request = [&](int t) {
    const int g = t / tiles, i = t - g * tiles, head = u.hk * a.G + g, left = a.Lq - 32 * i;
    const uint64_t there = left >= 32 ? 0xffffffffull : (1ull << left) - 1;
    uint8_t* at = smem + (t & 1) * STAGE;
    const T* Q = static_cast<const T*>(a.Q) + u.b * a.q.b + (int64_t)head * a.q.h + (int64_t)32 * i * a.q.l;
    const T* G = static_cast<const T*>(a.dO) + u.b * a.go.b + (int64_t)head * a.go.h + (int64_t)32 * i * a.go.l;
    request_tile<T, DP, 32, kThreads>(at, Q, a.q.l, there, a.d, tid);
    request_tile<T, DP, 32, kThreads>(at + TILE, G, a.go.l, there, a.d, tid);
    if (tid < 16) dma16(stat + (((int64_t)u.b * a.H + head) * tiles + i) * 64 + 4 * tid, at + 2 * TILE);
  };
  if (t0 < t1) request(t0);
  for (int t = t0; t < t1; ++t) {
    wait_vm<0>();
    raw_barrier();
    if (t + 1 < t1) request(t + 1);
    if (mine == 0) continue;
    const uint8_t* qt = smem + (t & 1) * STAGE;
    const uint8_t* gt = qt + TILE;
    const f32x4* st = reinterpret_cast<const f32x4*>(qt + 2 * TILE) + grp;
    f32x16 s, dp;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
    kf.times(s, view, qt, 0);
    if constexpr (WITH_K) vf.times(dp, view, gt, 0);
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const f32x4 lse = st[2 * r4], nd = st[8 + 2 * r4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 4 * r4 + e;
        s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -lse[e]));
        dp[r] = s[r] * (dp[r] + nd[e]);
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if constexpr (WITH_V) {
        const auto p = E::column(s, h);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) E::mma8(dv[dt], view.along(gt, 16 * h, dt), p);
      }
      if constexpr (WITH_K) {
        const auto ds = E::column(dp, h);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) E::mma8(dk[dt], view.along(qt, 16 * h, dt), ds);
      }
    }
  }
  // what a key that is not valid has gathered is no number of its own: its gradient is zero
  auto put = [&](const f32x16 (&acc)[DT], void* to, const bsa_strides_t& st, float scale, int place) {
    if (plan.nseg > 1) {
      float* out = part_of<DT * 32>(part, plan.units, seg, u.unit, wave, lane) + place * DT * 16 * 64;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) out[(dt * 16 + r) * 64] = valid ? acc[dt][r] : 0.f;
    } else if (u.there) {
      T* out = static_cast<T*>(to) + u.b * st.b + u.hk * st.h + u.key * st.l;
      if (valid) store_column<T, DT>(out, acc, scale, a.d, grp);
      else store_zeros<T, DT>(out, a.d, grp);
    }
  };
  if constexpr (WITH_K) put(dk, a.dK, a.gk, a.sm_scale, 0);
  if constexpr (WITH_V) put(dv, a.dV, a.gv, 1.f, 1);
}

template <typename T, int DP>
__global__ __launch_bounds__(kThreads, 1) void cross_dkv_kernel(CrossArgs a, Plan plan, int units_of_head, const float* stat, float* part) {
  if constexpr (DP <= 128) dkv_walk<T, DP, BOTH>(a, plan, units_of_head, stat, part);
  else if (blockIdx.y == 0) dkv_walk<T, DP, ONLY_K>(a, plan, units_of_head, stat, part);
  else dkv_walk<T, DP, ONLY_V>(a, plan, units_of_head, stat, part);
}

template <typename T, int DP>
__global__ __launch_bounds__(kThreads) void cross_dkv_combine_kernel(CrossArgs a, Plan plan, int units_of_head, float* part) {
  constexpr int DT = DP / 32;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, grp = lane >> 5;
  const KeyUnit u(a, blockIdx.x, wave, lane, units_of_head);
  const bool is_v = blockIdx.y;
  f32x16 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[dt][r] = 0.f;
  for (int s = 0; s < plan.nseg; ++s) {
    const float* in = part_of<DT * 32>(part, plan.units, s, u.unit, wave, lane) + (is_v ? DT * 16 * 64 : 0);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[dt][r] += in[(dt * 16 + r) * 64];
  }
  if (!u.there) return;
  if (is_v) store_column<T, DT>(static_cast<T*>(a.dV) + u.b * a.gv.b + u.hk * a.gv.h + u.key * a.gv.l, acc, 1.f, a.d, grp);
  else store_column<T, DT>(static_cast<T*>(a.dK) + u.b * a.gk.b + u.hk * a.gk.h + u.key * a.gk.l, acc, a.sm_scale, a.d, grp);
}

// ---- host ----
static size_t part_bytes(const Plan& p, int values) { return p.nseg == 1 ? 0 : (size_t)p.nseg * p.units * kWaves * values * 64 * sizeof(float); }

size_t cross_fwd_workspace(const CrossArgs& a) { return part_bytes(rows_plan(a), padded_d(a.d) / 2 + 2); }

static size_t stat_bytes(const CrossArgs& a) { return (size_t)a.B * a.H * query_tiles(a) * 256; }

size_t cross_bwd_workspace(const CrossArgs& a) {
  return stat_bytes(a) + std::max(part_bytes(rows_plan(a), padded_d(a.d) / 2), part_bytes(keys_plan(a), padded_d(a.d)));
}

template <typename T, int DP>
static int fwd_t(const CrossArgs& a, hipStream_t st) {
  const Plan p = rows_plan(a);
  constexpr size_t lds = 4 * key_tile<T>() * DP * sizeof(T);
  if (const int rc = allow_dynamic_lds<cross_fwd_kernel<T, DP>>(lds)) return rc;
  float* part = static_cast<float*>(a.ws);
  hipLaunchKernelGGL((cross_fwd_kernel<T, DP>), dim3((unsigned)(p.units * p.nseg)), dim3(kThreads), lds, st, a, p, row_units(a), part);
  if (const int rc = check_launch()) return rc;
  if (p.nseg > 1) hipLaunchKernelGGL((cross_fwd_combine_kernel<T, DP>), dim3((unsigned)p.units), dim3(kThreads), 0, st, a, p, row_units(a), part);
  return check_launch();
}

template <typename T, int DP>
static int bwd_t(const CrossArgs& a, hipStream_t st) {
  const Plan p = rows_plan(a), k = keys_plan(a);
  constexpr size_t lds = 4 * key_tile<T>() * DP * sizeof(T), klds = 2 * (64 * DP * sizeof(T) + 256);
  if (const int rc = allow_dynamic_lds<cross_dq_kernel<T, DP>>(lds)) return rc;
  if (const int rc = allow_dynamic_lds<cross_dkv_kernel<T, DP>>(klds)) return rc;
  float* stat = static_cast<float*>(a.ws);
  float* part = stat + stat_bytes(a) / sizeof(float);
  hipLaunchKernelGGL((cross_dq_kernel<T, DP>), dim3((unsigned)(p.units * p.nseg)), dim3(kThreads), lds, st, a, p, row_units(a), stat, part);
  if (const int rc = check_launch()) return rc;
  if (p.nseg > 1) hipLaunchKernelGGL((cross_dq_combine_kernel<T, DP>), dim3((unsigned)p.units), dim3(kThreads), 0, st, a, p, row_units(a), part);
  if (const int rc = check_launch()) return rc;
  const int key_units = (a.S + kUnitRows - 1) / kUnitRows;
  hipLaunchKernelGGL((cross_dkv_kernel<T, DP>), dim3((unsigned)(k.units * k.nseg), DP > 128 ? 2 : 1), dim3(kThreads), klds, st, a, k, key_units, stat, part);
  if (const int rc = check_launch()) return rc;
  if (k.nseg > 1) hipLaunchKernelGGL((cross_dkv_combine_kernel<T, DP>), dim3((unsigned)k.units, 2), dim3(kThreads), 0, st, a, k, key_units, part);
  return check_launch();
}

int launch_cross_fwd(const CrossArgs& a, hipStream_t st) {
  const bool f = a.dtype == BSA_F32;
  switch (padded_d(a.d)) {
    case 64: return f ? fwd_t<float, 64>(a, st) : fwd_t<uint16_t, 64>(a, st);
    case 128: return f ? fwd_t<float, 128>(a, st) : fwd_t<uint16_t, 128>(a, st);
    default: return f ? fwd_t<float, 256>(a, st) : fwd_t<uint16_t, 256>(a, st);
  }
}

int launch_cross_bwd(const CrossArgs& a, hipStream_t st) {
  const bool f = a.dtype == BSA_F32;
  switch (padded_d(a.d)) {
    case 64: return f ? bwd_t<float, 64>(a, st) : bwd_t<uint16_t, 64>(a, st);
    case 128: return f ? bwd_t<float, 128>(a, st) : bwd_t<uint16_t, 128>(a, st);
    default: return f ? bwd_t<float, 256>(a, st) : bwd_t<uint16_t, 256>(a, st);
  }
}

}  // namespace bsa
