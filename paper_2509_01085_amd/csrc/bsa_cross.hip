// Cross attention: every query row attends to the valid states of an encoder.  Forward, dQ, and dK and dV, for fp32 and
// bf16, any head dimension up to 256.
//
// The G query heads that share keys are one matrix of M = G Lq rows, so shared heads cost nothing in the forward and dQ and
// their gradients come out summed.  A workgroup has four wavefronts of 32 rows (forward, dQ) or 32 keys (dK, dV); the other
// side's tiles stream through LDS in a ring of two, one barrier a tile.
//
//   S = Q K^T, P = exp(sm_scale S - LSE), O = P V;  dP = dO V^T, delta = <dO, O>, dS = P (dP - delta),
//   dQ = sm_scale dS K, dK = sm_scale dS^T Q, dV = P^T dO
//
// Softmax statistics, sums and accumulators are fp32.  bf16: P and dS are rounded once on their way into a product, as its operands are
// bf16; that and the result's own rounding are what the results are off by (O 2.0e-3 rms, gradients 2.3e-3 to 2.5e-3).
//
// What bounds them, and what they measured (512 states, 33,280 queries, 12 heads, d = 128, bf16): the forward took 137 us (105 GFLOP,
// 0.76 PFLOP/s; a library product of 8192^3 reaches 1.4), dQ 186 (157 GFLOP, 0.84), dK and dV (bsa_cross_dkv.hip) 195 and 7 for the join (209
// GFLOP, 1.04 with it).  About 30 us of the forward are the first tiles, the rows and the results, 204 MB; a further state costs 0.21 us, 0.97
// PFLOP/s, where LDS reads (42 us), matrix cores (42) and vector instructions (66) of two wavefronts a SIMD are in each other's way.  One query
// a head and 12,134 of 20,000 states in the mean, 8 entries: 80 us, the bytes at the rate of a copy 85, and 9 to join the shares.  fp32: 118
// TFLOP/s of the 154 that a library product reaches (1,200 queries, 2,000 states, 48 heads: 500, 832 and 972 us).  More than 128 channels are
// far from that: 6 heads of 256, 503, 825 and 1,018 us for the same operations.
#include <algorithm>

#include "bsa_cross.h"

namespace bsa {

constexpr int kUnitRows = 32 * kWaves;

template <typename T, int DP> constexpr int key_tile() { return sizeof(T) == 2 && DP <= 128 ? 64 : 32; }

struct RowUnit {
  int b, hk, m, g, l;  // batch entry, key head, row, its head in the group and token
  bool live, any;      // this row, any of the wavefront's exists
  __device__ inline RowUnit(Args& a, int b_, int unit /* of the entry */, int wave, int lane) : b(b_) {
    const int of_head = (a.M + kUnitRows - 1) / kUnitRows;
    hk = (int)((uint32_t)unit / (uint32_t)of_head);
    const int first = (unit - hk * of_head) * kUnitRows + 32 * wave;
    any = first < a.M;
    m = first + (lane & 31);
    live = m < a.M;
    g = live && a.G > 1 ? (int)((uint32_t)m / (uint32_t)a.Lq) : 0;
    l = live ? m - g * a.Lq : 0;
  }
  __device__ inline int head(Args& a) const { return hk * a.G + g; }
  __device__ inline int64_t offset(Args& a, const __attribute__((address_space(4))) bsa_strides_t& s) const { return b * s.b + (int64_t)head(a) * s.h + (int64_t)l * s.l; }
  __device__ inline int64_t flat(Args& a) const { return ((int64_t)b * a.H + head(a)) * a.Lq + l; }
};

__device__ inline int key_head(Args& a, int unit) { return (int)((uint32_t)unit / (uint32_t)((a.M + kUnitRows - 1) / kUnitRows)); }

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
  __device__ inline void load(const T* p_, bool live_, int d_, int grp_) {
    p = p_;
    live = live_;
    d = d_;
    grp = grp_;
    if constexpr (HELD)
#pragma unroll
      for (int s = 0; s < DS; ++s) f[s] = row_chunk(p, 2 * s + grp, live, d);
  }
  __device__ inline void arrive() {  // waited for here, not between a tile's requests and its products
    if constexpr (HELD)
#pragma unroll
      for (int s = 0; s < DS; ++s) settle(f[s]);
  }
  // D += rows row0 .. row0 + 31 of the tile times this
  __device__ inline void times(f32x16& acc, const TileView<T, DP>& view, const uint8_t* tile, int row0) const {
    if constexpr (HELD) {
      constexpr int AHEAD = sizeof(T) == 4 ? 2 : 4;  // (fp32: four products a fragment)
      typename E::Frag fr[AHEAD];
#pragma unroll
      for (int s = 0; s < AHEAD; ++s) fr[s] = view.row(tile, row0, s);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int s = 0; s < DS; ++s) {
        E::mma(acc, fr[s % AHEAD], f[s]);
        if (s + AHEAD < DS) fr[s % AHEAD] = view.row(tile, row0, s + AHEAD);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      const int n = (d / E::CE + 1) / 2;
      typename E::Frag f[2] = {row_chunk(p, grp, live, d), row_chunk(p, 2 + grp, live, d)};
      for (int s = 0; s < n; s += 2) {  // (the chunks past d are zeros on both sides)
        typename E::Frag next[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) next[i] = row_chunk(p, 2 * (s + 2 + i) + grp, live, d);
#pragma unroll
        for (int i = 0; i < 2; ++i) E::mma(acc, view.row(tile, row0, s + i), f[i]);
#pragma unroll
        for (int i = 0; i < 2; ++i) f[i] = next[i];
      }
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
// Workgroups of a CU: dQ in fp32 with 128 channels (Q, dO, dQ in registers) and the walk over several pieces of such rows have one.
template <typename T, int DP, bool LEAN> constexpr int a_cu() { return DP <= 128 && (LEAN || DP * sizeof(T) <= 256) ? 2 : 1; }
template <typename T, int DP> constexpr bool held() { return DP <= 128; }

// ---- forward ----
// O = 0 and LSE = -inf without a valid key; a row whose valid logits are all -inf has no softmax and is NaN.
__device__ inline void put_lse(Args& a, const RowUnit& u, float m, float l, bool any, int grp) {
  if (grp == 0 && u.live) a.LSE_out[u.flat(a)] = any ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}
template <typename T, int DT>
__device__ inline void finish_row(Args& a, const RowUnit& u, const f32x16 (&acc)[DT], float m, float l, bool any, int grp) {
  store_column<T, DT>(static_cast<T*>(a.O_out) + u.offset(a, a.o), acc, any ? 1.f / l : 0.f, a.d, grp, u.live);
  put_lse(a, u, m, l, any, grp);
}

// The K and V tiles of a piece on their way through the ring of two.  SUMS: V's rows are summed (forward), so that one that is not there must
// not show; elsewhere it stands beside K's, whose product with it has no weight.
template <typename T, int DP, bool SUMS>
struct KvRing {
  static constexpr int KT = key_tile<T, DP>(), TILE = KT * DP * (int)sizeof(T);
  uint8_t* smem;
  Requests<T, DP, KT, kThreads> rk, rv;
  int lane;
  __device__ inline KvRing(uint8_t* smem_, Args& a, int tid) : smem(smem_), rk(a.k.l, a.d, tid), rv(a.v.l, a.d, tid), lane(tid & 63) {
    if (a.d < DP)
      for (int k = 0; k < 4; ++k) rk.clear(smem + k * TILE);
  }
  __device__ inline const uint8_t* k_tile(int place) const { return smem + place * 2 * TILE; }
  __device__ inline const uint8_t* v_tile(int place) const { return k_tile(place) + TILE; }
  // Tile t of key head hk, whose valid keys are `there`, into a place of the ring.
  __device__ __forceinline__ uint64_t request(Args& a, uint64_t there, int b, int hk, int t, int place) const {
    const T* K = static_cast<const T*>(a.K) + b * a.k.b + hk * a.k.h + (int64_t)t * KT * a.k.l;
    const T* V = static_cast<const T*>(a.V) + b * a.v.b + hk * a.v.h + (int64_t)t * KT * a.v.l;
    uint8_t* at = smem + place * 2 * TILE;
    rk.load(at, K, a.k.l, there, a.near);
    rv.template load<SUMS>(at + TILE, V, a.v.l, there, a.near);
    return there;
  }
  static constexpr uint64_t ALL = KT == 64 ? ~0ull : (1ull << KT) - 1;
};

// A workgroup's walk over its pieces and their tiles.  While a tile is multiplied the next one is on its way, be it this piece's or the
// next one's: `place` is the multiplied tile's, the other one the requested tile's.
template <typename T, int DP, bool SUMS>
struct Walk {
  static constexpr int KT = key_tile<T, DP>();
  const KvRing<T, DP, SUMS>& ring;
  int place = 0;
  bool asked = false;  // the coming piece's first tile has been requested
  uint64_t bits = 0;   // its valid keys
  uint64_t second = 0; // those of the piece's second tile, if that is there already
  bool here = false;
  __device__ inline explicit Walk(const KvRing<T, DP, SUMS>& r) : ring(r) {}
  // Requests a piece's first tile, unless that was done while the piece before it ended.
  __device__ __forceinline__ void ask(Args& a, const Piece& pc, int hk) {
    if (!asked && pc.t0 < pc.t1) bits = ring.request(a, Keys(a, pc.b).bits(pc.t0 * KT, KT, ring.lane), pc.b, hk, pc.t0, place);
    asked = true;
  }
  // Both tiles of a piece of one or two, now.  BEHIND: pieces may have come before it, whose last tile lies where the second one goes, and
  // wavefronts may be at its products still: the last barrier was ahead of them.
  template <bool BEHIND>
  __device__ __forceinline__ void both(Args& a, const Piece& pc, int hk) {
    if (pc.t1 == 2) {
      if constexpr (BEHIND) raw_barrier();
      second = ring.request(a, Keys(a, pc.b).bits(KT, KT, ring.lane), pc.b, hk, 1, place ^ 1);
    }
    here = true;
    wait_vm<0>();
    raw_barrier();
  }
  // tile(place, valid keys) for every tile of a piece; past(place) behind it.  (No tile is passed over: a way round the products
  // would have the compiler move the accumulators at every tile.)
  template <typename F, typename G>
  __device__ __forceinline__ void operator()(Args& a, const Piece& pc, int hk, bool more, const Piece& nx, int next_hk, F tile, G past) {
    asked = false;
    const Keys keys(a, pc.b);
    for (int t = pc.t0; t < pc.t1; ++t) {
      wait_vm<0>();
      raw_barrier();  // the tile is there for all, and all are done with the other place
      const uint64_t now = bits;
      if (t + 1 < pc.t1) {
        bits = here ? second : ring.request(a, keys.bits((t + 1) * KT, KT, ring.lane), pc.b, hk, t + 1, place ^ 1);
      } else if (more && nx.t0 < nx.t1) {
        bits = ring.request(a, Keys(a, nx.b).bits(nx.t0 * KT, KT, ring.lane), nx.b, next_hk, nx.t0, place ^ 1);
        asked = true;
      }
      tile(place, now);
      past(place);
      place ^= 1;
    }
    here = false;
  }
};

// A wavefront's state in the forward walk: O^T unnormalised, the running maximum (of the scaled logits, base 2; finite from the
// start, so that logits of -inf weigh nothing wherever they stand) and the lane's share of the sum.
constexpr float kLowest = -3.4e38f;
// How far (base 2) a logit may exceed the maximum before it is moved.  fp32 probabilities may be of any size.  bf16 ones are rounded on their way
// into O, the key at the maximum not at all and those just below it least, and these weigh most: with a lag of 6 O has 1.09 to 1.15 times the error
// of P relative to the row's own maximum (300 to 512 states, logits of deviation 1.5 and 3), with one of 2 up to 1.02 times, with 1 0.98.  512 states, 33,280 queries, 12 heads, d = 128, lags of
// 6, 3, 2, 1, 0: 130, 134, 137, 140 and 140 us; 70,400 queries, 40 heads 887, 910, 920, 935 and 941.
template <typename T> constexpr float lag() { return sizeof(T) == 2 ? 1.f : 6.f; }
template <typename T, int DT>
struct Walked {
  f32x16 o[DT];
  float m = kLowest, l = 0.f;
  __device__ inline Walked() {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
  }
  // Logits -> probabilities relative to the row's maximum.  The maximum is moved, and what was gathered before brought to it, only where
  // a logit of the wavefront's rows exceeds it by the lag.
  template <int NK>
  __device__ inline void softmax(f32x16 (&s)[NK], float c) {
    float top = s[0][0];
#pragma unroll
    for (int k = 0; k < NK; ++k)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[k][r]);
    if (__builtin_amdgcn_ballot_w64(top * c > m + lag<T>())) {  // c > 0: the maximum commutes with the scaling
      const float next = fmaxf(m, pair_max(top) * c);
      const float f = __builtin_amdgcn_exp2f(m - next);
      m = next;
      l *= f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] *= f;
    }
    float sum[NK];
#pragma unroll
    for (int k = 0; k < NK; ++k) sum[k] = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int k = 0; k < NK; ++k) {
        s[k][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[k][r], c, -m));
        sum[k] += s[k][r];
      }
#pragma unroll
    for (int k = 0; k < NK; ++k) l += sum[k];
  }
};

// Logits of keys that are not valid, `own` being the tile's bits from the lane's first row on.
template <int NK>
__device__ inline void mask_logits(f32x16 (&s)[NK], uint64_t own) {
#pragma unroll
  for (int k = 0; k < NK; ++k)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (!((own >> (32 * k + d_row(r))) & 1)) s[k][r] = -INFINITY;
}


// One tile of 64 keys, bf16 and d <= 128: the LDS fragments of the tile (K, then V) run through a ring of RINGF registers
// ahead of the products, in groups of two between which nothing moves.
template <int D>
__device__ inline void fwd_tile(Walked<uint16_t, D / 32>& w, const Fragments<D>& fg, const bf16x8* q, float c, uint64_t valid, int grp) {
  constexpr int DT = D / 32, DS = D / 16, NF = 2 * DS + 4 * DT, TILE = 64 * D * 2, RINGF = 4;
  auto frag = [&](auto F) -> bf16x8 {
    constexpr int f = decltype(F)::value;
    if constexpr (f < 2 * DS) return fg.template row<0>(32 * (f / DS), f % DS);
    else return fg.template along<TILE>(16 * ((f - 2 * DS) / DT), (f - 2 * DS) % DT);
  };
  bf16x8 fr[RINGF];
  static_for<0, RINGF>([&](auto F) { fr[decltype(F)::value] = frag(F); });
  __builtin_amdgcn_sched_barrier(0);
  f32x16 s[2];
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int r = 0; r < 16; ++r) s[k][r] = 0.f;
  static_for<0, 2 * DS>([&](auto F) {
    constexpr int f = decltype(F)::value;
    s[f / DS] = mfma32(fr[f % RINGF], q[f % DS], s[f / DS]);
    if constexpr (f + RINGF < NF) fr[f % RINGF] = frag(std::integral_constant<int, f + RINGF>{});
    if constexpr (f & 1) __builtin_amdgcn_sched_barrier(0);
  });
  if (valid != ~0ull) mask_logits<2>(s, valid >> (4 * grp));
  w.template softmax<2>(s, c);
  bf16x8 p[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) p[k] = d_to_b(s[k >> 1], k & 1);
  __builtin_amdgcn_sched_barrier(0);
  static_for<2 * DS, NF>([&](auto F) {  // V^T in (key step, channel tile) order: neighbours hit different accumulators
    constexpr int f = decltype(F)::value, v = f - 2 * DS;
    w.o[v % DT] = mfma32(fr[f % RINGF], p[v / DT], w.o[v % DT]);
    if constexpr (f + RINGF < NF) fr[f % RINGF] = frag(std::integral_constant<int, f + RINGF>{});
    if constexpr (f & 1) __builtin_amdgcn_sched_barrier(0);
  });
}

// ONE: a unit a workgroup (Deal::EACH), without what the walk over several pieces needs.
template <typename T, int DP, bool ONE>
__global__ __launch_bounds__(kThreads, (a_cu<T, DP, ONE>())) void cross_fwd_kernel(CrossArgs, Deal dl, float* part) {
  using Ring = KvRing<T, DP, true>;
  constexpr int KT = key_tile<T, DP>(), NK = KT / 32, DT = DP / 32;
  extern __shared__ __align__(16) uint8_t smem[];  // [2][K tile | V tile]
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Ring ring(smem, *kernel_args(), tid);
  Walk<T, DP, true> walk(ring);
  Dealer<ONE> dealer(*kernel_args(), dl, tid & 63);
  Piece pc, nx;
  if (!dealer.next(pc)) return;
  using Rows = RowFrags<T, DP, held<T, DP>()>;
  Rows q;
  auto load_q = [&](Rows& to, Args& a, const Piece& p, int lane) {
    const RowUnit u(a, p.b, p.unit, wave, lane);
    to.load(static_cast<const T*>(a.Q) + u.offset(a, a.q), u.live, a.d, lane >> 5);
  };
  walk.ask(*kernel_args(), pc, key_head(*kernel_args(), pc.unit));
  load_q(q, *kernel_args(), pc, tid & 63);
  for (;;) {
    Args& a = *afresh(kernel_args());
    const int lane = afresh(threadIdx.x & 63), grp = lane >> 5;
    const float c = a.sm_scale * kLog2e;
    const bool more = !ONE && dealer.next(nx);
    q.arrive();
    const RowUnit u(a, pc.b, pc.unit, wave, lane);
    Walked<T, DT> w;
    bool any = false;
    if constexpr (sizeof(T) == 2 && DP <= 128) {
      Fragments<DP> fg(uniform_lds(smem) + walk.place * 2 * Ring::TILE, lane);
      auto skip = [&](int, uint64_t now) { any |= now != 0; };
      if (!u.any) walk(a, pc, u.hk, more, nx, key_head(a, nx.unit), skip, [](int) {});
      else walk(a, pc, u.hk, more, nx, key_head(a, nx.unit),
                [&](int, uint64_t now) {
                  any |= now != 0;
                  fwd_tile<DP>(w, fg, q.f, c, now, grp);
                },
                [&](int place) { fg.move(place ? -2 * Ring::TILE : 2 * Ring::TILE); });
    } else {
      const TileView<T, DP> view(lane);
      walk(a, pc, u.hk, more, nx, key_head(a, nx.unit),
           [&](int place, uint64_t now) {
             any |= now != 0;
             f32x16 s[NK];
#pragma unroll
             for (int k = 0; k < NK; ++k) {
#pragma unroll
               for (int r = 0; r < 16; ++r) s[k][r] = 0.f;
               q.times(s[k], view, ring.k_tile(place), 32 * k);
             }
             if (now != Ring::ALL) mask_logits<NK>(s, now >> (4 * grp));
             w.template softmax<NK>(s, c);
#pragma unroll
             for (int k = 0; k < NK; ++k) view.gather(w.o, ring.v_tile(place), 32 * k, s[k]);
           },
           [](int) {});
    }
    if (u.any) {
      const float l = pair_sum(w.l);
      if (pc.slot < 0) {
        finish_row<T, DT>(a, u, w.o, w.m, l, any, grp);
      } else {
        float* out = part_of<DT * 16 + 2>(part, pc.slot, wave, lane);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) out[(dt * 16 + r) * 64] = w.o[dt][r];
        out[DT * 16 * 64] = w.m;
        out[(DT * 16 + 1) * 64] = any ? l : -1.f;  // (a sum is never negative)
      }
    }
    if (!more) return;
    pc = nx;
    walk.ask(a, pc, key_head(a, pc.unit));
    load_q(q, a, pc, lane);
  }
}

// The 16 values that a wavefront's channel tile has at `at` (values before it), of eight parts from s on (the last one again where there
// are fewer): their loads are in flight together.
template <int VALUES>
__device__ inline void load_parts(float (&v)[8][16], float* part, const Parts& ps, int s, int at, int wave, int lane) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float* in = part_of<VALUES>(part, ps.slot(min(s + j, ps.n - 1)), wave, lane) + at * 64;
#pragma unroll
    for (int r = 0; r < 16; ++r) v[j][r] = in[r * 64];
  }
}
template <int VALUES>
__device__ inline f32x16 sum_parts(float* part, const Parts& ps, int at, int wave, int lane) {
  f32x16 acc;
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = 0.f;
  for (int s = 0; s < ps.n; s += 8) {
    float v[8][16];
    load_parts<VALUES>(v, part, ps, s, at, wave, lane);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (s + j < ps.n)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[r] += v[j][r];
  }
  return acc;
}

// Joins the parts of a unit, and writes the rows of the units that had no step.  A workgroup has a wavefront for every 32 channels
// of the rows of one of the walk's wavefronts (blockIdx.y).
template <typename T, int DP>
__global__ __launch_bounds__(2 * DP, 1) void cross_fwd_combine_kernel(CrossArgs, Deal dl, float* part) {
  Args& a = *kernel_args();
  constexpr int DT = DP / 32, VALUES = DT * 16 + 2;
  const int lane = threadIdx.x & 63, dt = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = blockIdx.y, grp = lane >> 5;
  const int b = (int)(blockIdx.x / (uint32_t)dl.rows), unit = (int)blockIdx.x - b * dl.rows;
  const RowUnit u(a, b, unit, wave, lane);
  if (!u.any) return;
  const Parts ps(a, dl, lane, b, unit);
  if (ps.n == 0) return;
  // one pass: what was summed is brought to the maximum of every further eight parts
  float m = kLowest, l = 0.f;
  bool any = false;
  f32x16 o[1];
#pragma unroll
  for (int r = 0; r < 16; ++r) o[0][r] = 0.f;
  for (int s = 0; s < ps.n; s += 8) {
    float v[8][16], ms[8], ls[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float* in = part_of<VALUES>(part, ps.slot(min(s + j, ps.n - 1)), wave, lane) + DT * 16 * 64;
      ms[j] = in[0];
      ls[j] = in[64];
    }
    load_parts<VALUES>(v, part, ps, s, dt * 16, wave, lane);
    float top = m;
#pragma unroll
    for (int j = 0; j < 8; ++j) {  // (the last part again changes no maximum)
      any |= ls[j] != -1.f;
      top = fmaxf(top, ls[j] == -1.f ? kLowest : ms[j]);
    }
    const float was = __builtin_amdgcn_exp2f(m - top);
    m = top;
    l *= was;
#pragma unroll
    for (int r = 0; r < 16; ++r) o[0][r] *= was;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (s + j >= ps.n || ls[j] == -1.f) continue;  // (a part without a key holds nothing)
      const float f = __builtin_amdgcn_exp2f(ms[j] - m);
      l = __builtin_fmaf(ls[j], f, l);
#pragma unroll
      for (int r = 0; r < 16; ++r) o[0][r] = __builtin_fmaf(v[j][r], f, o[0][r]);
    }
  }
  store_column<T, 1>(static_cast<T*>(a.O_out) + u.offset(a, a.o) + 32 * dt, o, any ? 1.f / l : 0.f, a.d - 32 * dt, grp, u.live);
  if (dt == 0) put_lse(a, u, m, l, any, grp);
}

// ---- dQ ----
// dQ^T += K^T dS^T over the key tiles, S^T and dP^T recomputed.  Ahead of the walk each wavefront forms delta of its rows and leaves
// (LSE, -delta) for the other kernel: per head and query tile [32] LSE log2(e), [32] -delta; places that hold no token of the tile's
// own have LSE = +inf, i.e. weights of zero.
__device__ inline void put_stat(Args& a, const RowUnit& u, float* stat, float lse2, float delta, int grp) {
  if (grp != 0 || !u.live) return;
  const int i = u.l >> 5, first = first_token(a.Lq, i), r = u.l - first;
  float* at = stat + (((int64_t)u.b * a.H + u.head(a)) * query_tiles(a.Lq) + i) * 64;
  at[r] = lse2;
  at[32 + r] = -delta;
  if (u.l == a.Lq - 1) {  // the tile's other places weigh nothing
    for (int k = 0; k < 32; ++k)
      if (k > r || first + k < 32 * i) {
        at[k] = INFINITY;
        at[32 + k] = 0.f;
      }
  }
}

// Probabilities of keys that are not valid.
__device__ inline void mask_weights(f32x16& p, uint64_t own) {
#pragma unroll
  for (int r = 0; r < 16; ++r)
    if (!((own >> d_row(r)) & 1)) p[r] = 0.f;
}

// One tile of 64 keys, bf16 and d <= 128, 32 keys at a time: fragments as in fwd_tile, K and V rows in turn, then K^T.
template <int D>
__device__ inline void dq_tile(f32x16 (&dq)[D / 32], const Fragments<D>& fg, const bf16x8* q, const bf16x8* g, float c, float lse2, float delta,
                               uint64_t valid, int grp) {
  constexpr int DT = D / 32, DS = D / 16, NF = 2 * DS + 2 * DT, TILE = 64 * D * 2, RINGF = 4;
  static_for<0, 2>([&](auto K) {
    constexpr int k = decltype(K)::value;
    auto frag = [&](auto F) -> bf16x8 {
      constexpr int f = decltype(F)::value, v = f - 2 * DS;
      if constexpr (f < 2 * DS) return fg.template row<(f & 1) * TILE>(32 * k, f >> 1);
      else return fg.template along<0>(32 * k + 16 * (v / DT), v % DT);
    };
    bf16x8 fr[RINGF];
    static_for<0, RINGF>([&](auto F) { fr[decltype(F)::value] = frag(F); });
    __builtin_amdgcn_sched_barrier(0);
    f32x16 s, dp;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
    static_for<0, 2 * DS>([&](auto F) {
      constexpr int f = decltype(F)::value;
      if constexpr (f & 1) dp = mfma32(fr[f % RINGF], g[f >> 1], dp);
      else s = mfma32(fr[f % RINGF], q[f >> 1], s);
      if constexpr (f + RINGF < NF) fr[f % RINGF] = frag(std::integral_constant<int, f + RINGF>{});
      if constexpr (f & 1) __builtin_amdgcn_sched_barrier(0);
    });
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -lse2));
    if (valid != ~0ull) mask_weights(s, valid >> (32 * k + 4 * grp));
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] *= dp[r] - delta;
    const bf16x8 d0 = d_to_b(s, 0), d1 = d_to_b(s, 1);
    __builtin_amdgcn_sched_barrier(0);
    static_for<2 * DS, NF>([&](auto F) {
      constexpr int f = decltype(F)::value, v = f - 2 * DS;
      dq[v % DT] = mfma32(fr[f % RINGF], v / DT ? d1 : d0, dq[v % DT]);
      if constexpr (f + RINGF < NF) fr[f % RINGF] = frag(std::integral_constant<int, f + RINGF>{});
      if constexpr (f & 1) __builtin_amdgcn_sched_barrier(0);
    });
  });
}

// The lane's share of delta = sum over the tile's keys of P dP, from the probabilities themselves.
template <int D>
__device__ inline float delta_tile(const Fragments<D>& fg, const bf16x8* q, const bf16x8* g, float c, float lse2, uint64_t valid, int grp) {
  constexpr int DS = D / 16, TILE = 64 * D * 2;
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    f32x16 s, dp;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
#pragma unroll
    for (int i = 0; i < DS; ++i) {
      s = mfma32(fg.template row<0>(32 * k, i), q[i], s);
      dp = mfma32(fg.template row<TILE>(32 * k, i), g[i], dp);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -lse2));
    if (valid != ~0ull) mask_weights(s, valid >> (32 * k + 4 * grp));
#pragma unroll
    for (int r = 0; r < 16; ++r) sum = __builtin_fmaf(s[r], dp[r], sum);
    __builtin_amdgcn_sched_barrier(0);
  }
  return sum;
}

template <typename T, int DP, bool ONE>
__global__ __launch_bounds__(kThreads, (a_cu<T, DP, false>())) void cross_dq_kernel(CrossArgs, Deal dl, float* stat, float* part) {
  using Ring = KvRing<T, DP, false>;
  constexpr int KT = key_tile<T, DP>(), NK = KT / 32, DT = DP / 32;
  extern __shared__ __align__(16) uint8_t smem[];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Ring ring(smem, *kernel_args(), tid);
  Walk<T, DP, false> walk(ring);
  Dealer<ONE> dealer(*kernel_args(), dl, tid & 63);
  Piece pc, nx;
  bool more = dealer.next(nx);
  while (more) {
    pc = nx;
    Args& a = *afresh(kernel_args());
    const int lane = afresh(threadIdx.x & 63), grp = lane >> 5;
    const float c = a.sm_scale * kLog2e;
    const RowUnit u(a, pc.b, pc.unit, wave, lane);
    walk.ask(a, pc, u.hk);
    RowFrags<T, DP, held<T, DP>()> q;
    RowFrags<T, DP, held<T, DP>()> gr;
    q.load(static_cast<const T*>(a.Q) + u.offset(a, a.q), u.live, a.d, grp);
    gr.load(static_cast<const T*>(a.dO) + u.offset(a, a.go), u.live, a.d, grp);
    const float lse2 = u.live ? a.LSE_in[u.flat(a)] * kLog2e : INFINITY;
    more = !ONE && dealer.next(nx);
    // A bf16 unit of no more than two tiles, which the ring holds: delta from the probabilities, a pass over both ahead of the
    // other.  With so few keys the rounding of O is what the gradients' error would mostly be (19 keys, d = 80: dQ 3.2e-3 off, rms),
    // and O is not read.  (It has to be this softmax's: for another O, as of more states than these, the two are different numbers.)
    const bool few = sizeof(T) == 2 && DP <= 128 && pc.slot < 0 && pc.t1 > 0 && pc.t1 <= 2;
    float delta = few ? 0.f : pair_sum(gr.dot(static_cast<const T*>(a.O) + u.offset(a, a.o)));
    q.arrive();
    gr.arrive();
    if (!few && pc.t0 == 0) put_stat(a, u, stat, lse2, delta, grp);
    f32x16 dq[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) dq[dt][r] = 0.f;
    if constexpr (sizeof(T) == 2 && DP <= 128) {
      Fragments<DP> fg(uniform_lds(smem) + walk.place * 2 * Ring::TILE, lane);
      auto on = [&](int place) { fg.move(place ? -2 * Ring::TILE : 2 * Ring::TILE); };
      if (few) {
        walk.template both<!ONE>(a, pc, u.hk);
        if (u.any) {
#pragma unroll 1
          for (int t = 0; t < pc.t1; ++t) {
            delta += delta_tile<DP>(fg, q.f, gr.f, c, lse2, t ? walk.second : walk.bits, grp);
            on(walk.place ^ t);
          }
          if (pc.t1 == 1) on(walk.place ^ 1);
          delta = pair_sum(delta);
          put_stat(a, u, stat, lse2, delta, grp);
        }
      }
      if (!u.any) walk(a, pc, u.hk, more, nx, key_head(a, nx.unit), [](int, uint64_t) {}, [](int) {});
      else walk(a, pc, u.hk, more, nx, key_head(a, nx.unit), [&](int, uint64_t now) { dq_tile<DP>(dq, fg, q.f, gr.f, c, lse2, delta, now, grp); }, on);
    } else {
      const TileView<T, DP> view(lane);
      walk(a, pc, u.hk, more, nx, key_head(a, nx.unit),
           [&](int place, uint64_t now) {
#pragma unroll
             for (int k = 0; k < NK; ++k) {
               f32x16 s, dp;
#pragma unroll
               for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
               q.times(s, view, ring.k_tile(place), 32 * k);
               gr.times(dp, view, ring.v_tile(place), 32 * k);
#pragma unroll
               for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -lse2));
               if (now != Ring::ALL) mask_weights(s, now >> (32 * k + 4 * grp));
#pragma unroll
               for (int r = 0; r < 16; ++r) s[r] *= dp[r] - delta;
               view.gather(dq, ring.k_tile(place), 32 * k, s);
             }
           },
           [](int) {});
    }
    if (!u.any) continue;
    if (pc.slot < 0) {
      store_column<T, DT>(static_cast<T*>(a.dQ) + u.offset(a, a.gq), dq, a.sm_scale, a.d, grp, u.live);
    } else {
      float* out = part_of<DT * 16>(part, pc.slot, wave, lane);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) out[(dt * 16 + r) * 64] = dq[dt][r];
    }
  }
}

template <typename T, int DP>
__global__ __launch_bounds__(2 * DP, 1) void cross_dq_combine_kernel(CrossArgs, Deal dl, float* part) {
  Args& a = *kernel_args();
  constexpr int DT = DP / 32;
  const int lane = threadIdx.x & 63, dt = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = blockIdx.y;
  const int b = (int)(blockIdx.x / (uint32_t)dl.rows), unit = (int)blockIdx.x - b * dl.rows;
  const RowUnit u(a, b, unit, wave, lane);
  if (!u.any) return;
  const Parts ps(a, dl, lane, b, unit);
  if (ps.n == 0) return;
  const f32x16 dq[1] = {sum_parts<DT * 16>(part, ps, dt * 16, wave, lane)};
  store_column<T, 1>(static_cast<T*>(a.dQ) + u.offset(a, a.gq) + 32 * dt, dq, a.sm_scale, a.d - 32 * dt, lane >> 5, u.live);
}

// ---- dK, dV ----
// A wavefront owns 32 keys; dV^T += dO^T P and dK^T += Q^T dS over the query tiles (32 tokens of one head) of the heads that share them.
// (Units of an entry: key tile after key tile, each for all key heads, so that those with valid keys come first.)
struct KeyUnit {
  int b, hk, first, key;
  bool there;   // the lane's key exists
  __device__ inline KeyUnit(Args& a, int b_, int unit, int wave, int lane) : b(b_) {
    const int tile = (int)((uint32_t)unit / (uint32_t)a.Hkv);
    hk = unit - tile * a.Hkv;
    first = tile * kUnitRows;
    key = first + 32 * wave + (lane & 31);
    there = key < a.S;
  }
};

// WHAT: both at once, or (256 channels, whose two accumulators would not leave the registers for the rows) dK and dV by workgroups of
// their own, which form S twice.
enum { BOTH = 0, ONLY_K = 1, ONLY_V = 2 };

template <typename T, int DP, int WHAT>
__device__ inline void dkv_walk(const Deal& dl, const float* stat, float* part) {
  constexpr int DT = DP / 32, TILE = 32 * DP * sizeof(T), STAGE = 2 * TILE + 256;
  constexpr bool WITH_K = WHAT != ONLY_V, WITH_V = WHAT != ONLY_K;
  extern __shared__ __align__(16) uint8_t smem[];  // [2][Q tile | dO tile | LSE, -delta]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), grp = lane >> 5;
  const TileView<T, DP> view(lane);
  Args& args = *kernel_args();
  const Requests<T, DP, 32, kThreads> rq(args.q.l, args.d, tid), rg(args.go.l, args.d, tid);
  if (args.d < DP)
    for (int k = 0; k < 4; ++k) rq.clear(smem + (k >> 1) * STAGE + (k & 1) * TILE);
 Dealer<false> dealer(args, dl, lane);
 Piece pc;
 while (dealer.next(pc)) {
  Args& a = *afresh(kernel_args());
  const float c = a.sm_scale * kLog2e;
  const int tiles = query_tiles(a.Lq);  // of a head
  const KeyUnit u(a, pc.b, pc.unit, wave, lane);
  const Keys keys(a, u.b);
  raw_barrier();
  const uint64_t mine = keys.bits(u.first + 32 * wave, 32, lane);                   // valid keys of the wavefront
  const bool valid = (mine >> (lane & 31)) & 1;
  const bool work = __syncthreads_or(mine != 0);                                   // of the workgroup
  const T* K = static_cast<const T*>(a.K) + u.b * a.k.b + u.hk * a.k.h + u.key * a.k.l;
  const T* V = static_cast<const T*>(a.V) + u.b * a.v.b + u.hk * a.v.h + u.key * a.v.l;
  RowFrags<T, DP, held<T, DP>()> kf, vf;
  kf.load(K, valid, a.d, grp);
  if constexpr (WITH_K) vf.load(V, valid, a.d, grp);
  kf.arrive();
  if constexpr (WITH_K) vf.arrive();
  f32x16 dk[WITH_K ? DT : 1], dv[WITH_V ? DT : 1];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      if (WITH_K) dk[dt][r] = 0.f;
      if (WITH_V) dv[dt][r] = 0.f;
    }
  const int t0 = pc.t0, t1 = work ? pc.t1 : t0;
  auto request = [&](int t) {
    const int g = t / tiles, i = t - g * tiles, head = u.hk * a.G + g;
    const int64_t first = first_token(a.Lq, i);
    const uint64_t there = a.Lq >= 32 ? 0xffffffffull : (1ull << a.Lq) - 1;
    uint8_t* at = smem + (t & 1) * STAGE;
    const T* Q = static_cast<const T*>(a.Q) + u.b * a.q.b + (int64_t)head * a.q.h + first * a.q.l;
    const T* G = static_cast<const T*>(a.dO) + u.b * a.go.b + (int64_t)head * a.go.h + first * a.go.l;
    rq.load(at, Q, a.q.l, there, a.near);
    rg.load(at + TILE, G, a.go.l, there, a.near);
    if (tid < 16) dma16(stat + (((int64_t)u.b * a.H + head) * tiles + i) * 64 + 4 * tid, at + 2 * TILE);
  };
  if (t0 < t1) request(t0);
  for (int t = t0; t < t1; ++t) {  // (a way round the products, for a wavefront without valid keys, would move the accumulators every time)
    wait_vm<0>();
    raw_barrier();
    if (t + 1 < t1) request(t + 1);
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
    if constexpr (WITH_V) view.gather(dv, gt, 0, s);
    if constexpr (WITH_K) view.gather(dk, qt, 0, dp);
  }
  // what a key that is not valid has gathered is no number of its own: its gradient is zero
  auto put = [&](const f32x16 (&acc)[DT], void* to, const __attribute__((address_space(4))) bsa_strides_t& st, float scale, int place) {
    if (pc.slot >= 0) {
      float* out = part_of<DT * 32>(part, pc.slot, wave, lane) + place * DT * 16 * 64;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) out[(dt * 16 + r) * 64] = valid ? acc[dt][r] : 0.f;
    } else {
      T* out = static_cast<T*>(to) + u.b * st.b + u.hk * st.h + u.key * st.l;
      store_column<T, DT>(out, acc, scale, a.d, grp, valid);
      if (u.there && !valid) store_zeros<T, DT>(out, a.d, grp);
    }
  };
  if constexpr (WITH_K) put(dk, a.dK, a.gk, a.sm_scale, 0);
  if constexpr (WITH_V) put(dv, a.dV, a.gv, 1.f, 1);
 }
}

template <typename T, int DP>
__global__ __launch_bounds__(kThreads, 1) void cross_dkv_kernel(CrossArgs, Deal dl, const float* stat, float* part) {
  if constexpr (DP <= 128) dkv_walk<T, DP, BOTH>(dl, stat, part);
  else if (blockIdx.y == 0) dkv_walk<T, DP, ONLY_K>(dl, stat, part);
  else dkv_walk<T, DP, ONLY_V>(dl, stat, part);
}

// Joins the parts of a unit, and writes the zeros of the units that had no step.
template <typename T, int DP>
__global__ __launch_bounds__(2 * DP, 1) void cross_dkv_combine_kernel(CrossArgs, Deal dl, float* part) {
  Args& a = *kernel_args();
  constexpr int DT = DP / 32;
  const int lane = threadIdx.x & 63, dt = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = blockIdx.y;
  const bool is_v = blockIdx.z;
  const int b = (int)(blockIdx.x / (uint32_t)dl.rows), unit = (int)blockIdx.x - b * dl.rows;
  const KeyUnit u(a, b, unit, wave, lane);
  const Parts ps(a, dl, lane, b, unit);
  if (ps.n == 0) return;
  const f32x16 acc[1] = {sum_parts<DT * 32>(part, ps, (is_v * DT + dt) * 16, wave, lane)};
  const auto& st = is_v ? a.gv : a.gk;
  store_column<T, 1>(static_cast<T*>(is_v ? a.dV : a.dK) + u.b * st.b + u.hk * st.h + u.key * st.l + 32 * dt, acc, is_v ? 1.f : a.sm_scale,
                     a.d - 32 * dt, lane >> 5, u.there);
}

// ---- host ----
static int padded_d(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

// Forward and dQ: two workgroups a CU where registers and LDS allow it.  Shares where whole units would leave slots without work for
// the time of `worth` tiles, which is what shares cost: the reckoning, the second launch, and at d = 128 a loop with fewer registers.
// bf16: about 14 us, a tile takes 1.2.  fp32: 10 to 30 us, a tile 3 to 6, and one workgroup keeps a CU's matrix cores as busy as two, so
// the CUs are counted, and shares taken only where half of them would have no unit.  4 heads of 64 channels, 700 queries, 200 states
// in fp32: 59 us whole, 36 in shares; 12 of 128, 2,520 queries, 333 states (240 units): 193 and 257; 48 of 1,200 queries, 2,000 states
// (480 units): 1,630 and 2,070.  Lengths are known on the device only and do not count here: shares for a batch of four of any length
// up to 2,000 (bf16, 480 units) took 204 us, whole units 128.
static Deal rows_deal(const CrossArgs& a) {
  const bool f32 = a.dtype == BSA_F32;
  Deal d{};
  d.tile = !f32 && a.d <= 128 ? 64 : 32;  // key_tile
  d.rows = a.Hkv * ((a.M + kUnitRows - 1) / kUnitRows);
  const int64_t units = (int64_t)d.rows * a.B, tiles = (a.S + d.tile - 1) / d.tile;
  const int slots = !f32 && a.d <= 128 ? 512 : 256, worth = f32 ? 4 : 12, least = f32 ? 1 : 4;  // (tiles of a share)
  const int64_t idle = ((units + slots - 1) / slots * slots - units) * tiles;  // of all slots together
  d.way = units < (f32 ? slots / 2 : 2 * slots) && idle > (int64_t)worth * slots ? SHARES : EACH;
  d.grid = (int)(d.way == SHARES ? std::min<int64_t>(slots, std::max<int64_t>(1, units * tiles / least)) : units);
  return d;
}

// A step is worth a share of its own: 8 steps of 2 units in fp32 took 27 us in four shares, 17 in eight, 12 in sixteen.
static Deal keys_deal(const CrossArgs& a) {
  Deal d{};
  d.by_keys = 1;
  d.tile = kUnitRows;
  d.steps = a.G * query_tiles(a.Lq);
  d.rows = a.Hkv * ((a.S + kUnitRows - 1) / kUnitRows);
  d.way = SHARES;
  d.grid = (int)std::min<int64_t>(256, (int64_t)d.rows * a.B * d.steps);
  return d;
}

static size_t part_bytes(const Deal& d, int values) { return d.way == SHARES ? (size_t)2 * d.grid * kWaves * values * 64 * sizeof(float) : 0; }

size_t cross_fwd_workspace(const CrossArgs& a) { return part_bytes(rows_deal(a), padded_d(a.d) / 2 + 2); }

static size_t stat_bytes(const CrossArgs& a) { return (size_t)a.B * a.H * query_tiles(a.Lq) * 256; }

// dK and dV on the kernel of bsa_cross_dkv.hip.  Below 32 tokens a head has no whole query tile.  (The strides may still ask for the
// kernel here, so the workspace holds either's.)
static bool fast_dkv(const CrossArgs& a) { return a.dtype == BSA_BF16 && a.d <= 128 && a.Lq >= 32; }

size_t cross_bwd_workspace(const CrossArgs& a) {
  size_t parts = std::max(part_bytes(rows_deal(a), padded_d(a.d) / 2), part_bytes(keys_deal(a), padded_d(a.d)));
  if (fast_dkv(a)) parts = std::max(parts, cross_dkv_fast_parts(a));
  return stat_bytes(a) + parts;
}

template <typename T, int DP>
static int fwd_t(const CrossArgs& a, hipStream_t st) {
  const Deal d = rows_deal(a);
  if (part_bytes(d, DP / 2 + 2) > a.ws_bytes) return BSA_ERR_WORKSPACE;
  constexpr size_t lds = 4 * key_tile<T, DP>() * DP * sizeof(T);
  const bool one = d.way == EACH;
  if (const int rc = one ? allow_dynamic_lds<cross_fwd_kernel<T, DP, true>>(lds) : allow_dynamic_lds<cross_fwd_kernel<T, DP, false>>(lds)) return rc;
  float* part = static_cast<float*>(a.ws);
  if (one) hipLaunchKernelGGL((cross_fwd_kernel<T, DP, true>), dim3(d.grid), dim3(kThreads), lds, st, a, d, part);
  else hipLaunchKernelGGL((cross_fwd_kernel<T, DP, false>), dim3(d.grid), dim3(kThreads), lds, st, a, d, part);
  if (const int rc = check_launch()) return rc;
  if (d.way == SHARES) hipLaunchKernelGGL((cross_fwd_combine_kernel<T, DP>), dim3((unsigned)d.rows * a.B, kWaves), dim3(2 * DP), 0, st, a, d, part);
  return check_launch();
}

template <typename T, int DP>
static int bwd_t(const CrossArgs& a, hipStream_t st) {
  const Deal d = rows_deal(a), k = keys_deal(a);
  if (stat_bytes(a) + std::max(part_bytes(d, DP / 2), part_bytes(k, DP)) > a.ws_bytes) return BSA_ERR_WORKSPACE;
  constexpr size_t lds = 4 * key_tile<T, DP>() * DP * sizeof(T), klds = 2 * (64 * DP * sizeof(T) + 256);
  const bool one = d.way == EACH;
  if (const int rc = one ? allow_dynamic_lds<cross_dq_kernel<T, DP, true>>(lds) : allow_dynamic_lds<cross_dq_kernel<T, DP, false>>(lds)) return rc;
  const bool fast = fast_dkv(a) && a.near;
  if (const int rc = fast ? grant_cross_dkv_fast(a) : allow_dynamic_lds<cross_dkv_kernel<T, DP>>(klds)) return rc;
  float* stat = static_cast<float*>(a.ws);
  float* part = stat + stat_bytes(a) / sizeof(float);
  if (one) hipLaunchKernelGGL((cross_dq_kernel<T, DP, true>), dim3(d.grid), dim3(kThreads), lds, st, a, d, stat, part);
  else hipLaunchKernelGGL((cross_dq_kernel<T, DP, false>), dim3(d.grid), dim3(kThreads), lds, st, a, d, stat, part);
  if (const int rc = check_launch()) return rc;
  if (d.way == SHARES) hipLaunchKernelGGL((cross_dq_combine_kernel<T, DP>), dim3((unsigned)d.rows * a.B, kWaves), dim3(2 * DP), 0, st, a, d, part);
  if (const int rc = check_launch()) return rc;
  if (fast) return launch_cross_dkv_fast(a, stat, part, st);
  hipLaunchKernelGGL((cross_dkv_kernel<T, DP>), dim3(k.grid, DP > 128 ? 2 : 1), dim3(kThreads), klds, st, a, k, stat, part);
  if (const int rc = check_launch()) return rc;
  hipLaunchKernelGGL((cross_dkv_combine_kernel<T, DP>), dim3((unsigned)k.rows * a.B, kWaves, 2), dim3(2 * DP), 0, st, a, k, part);
  return check_launch();
}

// A tile's offsets fit 31 bits.
static int is_near(const CrossArgs& a, bool backward) {
  const int64_t most = 0x7fffffffLL / (64 * (a.dtype == BSA_F32 ? 4 : 2)) - a.d;
  return a.k.l < most && a.v.l < most && (!backward || (a.q.l < most && a.go.l < most));
}

int launch_cross_fwd(const CrossArgs& given, hipStream_t st) {
  CrossArgs a = given;
  a.near = is_near(a, false);
  const bool f = a.dtype == BSA_F32;
  switch (padded_d(a.d)) {
    case 64: return f ? fwd_t<float, 64>(a, st) : fwd_t<uint16_t, 64>(a, st);
    case 128: return f ? fwd_t<float, 128>(a, st) : fwd_t<uint16_t, 128>(a, st);
    default: return f ? fwd_t<float, 256>(a, st) : fwd_t<uint16_t, 256>(a, st);
  }
}

int launch_cross_bwd(const CrossArgs& given, hipStream_t st) {
  CrossArgs a = given;
  a.near = is_near(a, true);
  const bool f = a.dtype == BSA_F32;
  switch (padded_d(a.d)) {
    case 64: return f ? bwd_t<float, 64>(a, st) : bwd_t<uint16_t, 64>(a, st);
    case 128: return f ? bwd_t<float, 128>(a, st) : bwd_t<uint16_t, 128>(a, st);
    default: return f ? bwd_t<float, 256>(a, st) : bwd_t<uint16_t, 256>(a, st);
  }
}

}  // namespace bsa
