// dK, dV of the cross attention (bf16 matrix cores, d up to 128): one workgroup owns 64 keys.
//
//   dV^T += dO^T P,  dK^T += Q^T dS,  with S = Q K^T, P = exp2(S c - LSE), dP = dO V^T,
//   dS = P (dP - delta), over the query tiles (32 tokens of a head) of the heads that share the keys.
//
// The way of bsa_attn_dkv.hip, on tensors instead of records: the four wavefronts of a workgroup take the tiles in turn, each for
// all 64 keys; K and V fragments stay in 128 registers, the dK^T and dV^T accumulators fill the 256 accumulation
// registers, Q and dO rows stream through a private LDS ring of two tiles (no barrier), every LDS fragment feeds two
// MFMAs, and the instruction order is fixed: exp2 under the dP products, dS under the dV products, the requests under the
// others.  A lane's request addresses are one instruction each, because the swizzle of a row's chunk is an exclusive or with a
// constant.  The query tiles of all units are dealt out in equal shares: 96 units (512 keys, 12 heads) of 1,040 tiles
// (33,280 tokens) have 256 workgroups walk 390 tiles each.
//
// What bounds it: the matrix cores (42 % of the time busy), and beside them the exponentials and the LDS reads: there 195 us, 1.07 PFLOP/s,
// and 7 to join the shares (1.04 with them).  See bsa_attn_dkv.hip for the waits that inline assembly needs.
#include <algorithm>

#include "bsa_cross.h"
#include "bsa_pipe.h"

namespace bsa {

// a tile's 256 bytes of row statistics: sixteen lanes
__device__ inline void dma_tail(uint64_t sbase, uint32_t lane16, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_mov_b64 exec, 0xffff\n\tglobal_load_lds_dwordx4 %0, %1\n\ts_mov_b64 exec, -1"
               :
               : "v"(lane16), "s"(sbase), "s"(lds)
               : "memory", "m0");
}

constexpr int kKeys = 64;  // of a unit

// WHOLE: d == D; else K and V are zero in the channels past d, where Q and dO rows repeat their first chunk.  (No lane is left out
// of a request: a branch between the products would have the compiler move their results before they are there.)
template <int D, bool WHOLE>
__global__ __launch_bounds__(256, 1) void cross_dkv_fast_kernel(CrossArgs, Deal dl, const float* stat, float* part) {
  using R = BwdRec<D>;
  constexpr int NH = kKeys / 32;            // 32-key halves
  constexpr int RB = D * 2, DT = D / 32, DS = D / 16, NT = NH * DT;
  constexpr int ND = 32 * RB / 1024;        // DMA instructions of a tile's Q (or dO) rows
  constexpr int CPR = RB / 16, RPI = 64 / CPR;  // chunks of a row, rows of an instruction
  constexpr int NF = 2 * DS + 4 * DT;       // fragments of a tile in order of use
  constexpr int RING = DT == 2 ? 2 : 4;     // fragments read ahead (64 cycles each)
  static_assert(NF % RING == 0 && 2 * DT - RING >= 2, "the ring wraps into the next tile");
  static_assert(8 * R::BYTES >= NT * 16 * 1024, "the tile ring doubles as the reduction buffer");
  extern __shared__ __align__(16) uint8_t smem[];  // [4 wavefronts][2 tiles]
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  Dealer<false> dealer(*kernel_args(), dl, threadIdx.x & 63);
  Piece pc;
  while (dealer.next(pc)) {
    Args& a = *afresh(kernel_args());
    const int lane = afresh(threadIdx.x & 63), grp = lane >> 5, col = lane & 31;
    const int tile = (int)((uint32_t)pc.unit / (uint32_t)a.Hkv), hk = pc.unit - tile * a.Hkv, b = pc.b, first = tile * kKeys;
    const Keys keys(a, b);
    const uint64_t valid = keys.bits(first, kKeys, lane);
    const int items = valid ? pc.t1 - pc.t0 : 0;
    const int mine = (items - wave + 3) >> 2;  // tiles t0 + wave, t0 + wave + 4, ...
    const float c2 = a.sm_scale * kLog2e;

    // K and V fragments (B operands): lane (col, grp) holds channels 16 s + 8 grp .. +7 of key 32 h + col.
    bf16x8 kf[NH][DS], vf[NH][DS];
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      const bool ok = (valid >> (32 * h + col)) & 1;
      const int64_t key = ok ? first + 32 * h + col : 0;
      const uint16_t* K = static_cast<const uint16_t*>(a.K) + b * a.k.b + hk * a.k.h + key * a.k.l;
      const uint16_t* V = static_cast<const uint16_t*>(a.V) + b * a.v.b + hk * a.v.h + key * a.v.l;
#pragma unroll
      for (int s = 0; s < DS; ++s) {
        const int ch = 16 * s + 8 * grp;
        kf[h][s] = ok && (WHOLE || ch < a.d) ? *reinterpret_cast<const bf16x8*>(K + ch) : Elt<uint16_t>::zero();
        vf[h][s] = ok && (WHOLE || ch < a.d) ? *reinterpret_cast<const bf16x8*>(V + ch) : Elt<uint16_t>::zero();
      }
    }
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int s = 0; s < DS; ++s) {  // waited for here, not in the loop
        settle(kf[h][s]);
        settle(vf[h][s]);
      }
    f32x16 dk[NH][DT], dv[NH][DT];
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) dk[h][dt][r] = dv[h][dt][r] = 0.f;

    if (mine > 0) {
      const uint32_t lds0 = uniform_lds(smem + wave * 2 * R::BYTES);
      // Requests.  LDS place n * 64 + lane of a tile is chunk position lane % CPR of row RPI n + lane / CPR and takes chunk
      // position ^ swz(row): of the row's swizzle, the part that n decides is an exclusive or with a constant.
      const int prow = lane / CPR;
      const uint32_t chunk = (uint32_t)((lane % CPR) ^ swz<D>(prow)) << 4;
      const uint32_t lane16 = D == 128 ? chunk : lane * 16;  // (of the sixteen lanes that use it)
      const uint32_t row_q = (uint32_t)(prow * a.q.l * 2), row_g = (uint32_t)(prow * a.go.l * 2);
      const int64_t step_q = RPI * a.q.l * 2, step_g = RPI * a.go.l * 2;
      auto rows = [&](uint64_t src, int64_t step, uint32_t row, uint32_t dst, auto N) {
        constexpr int n = decltype(N)::value;
        constexpr uint32_t flip = (uint32_t)swz<D>(RPI * n) << 4;
        const uint32_t ch = chunk ^ flip;
        dma16_raw(src + n * step, (WHOLE || ch < (uint32_t)a.d * 2 ? ch : 0) + row, dst + 1024 * n);
      };
      auto rows_q = [&](uint64_t src, uint32_t slot, auto N) { rows(src, step_q, row_q, slot + R::QC, N); };
      auto rows_g = [&](uint64_t src, uint32_t slot, auto N) { rows(src, step_g, row_g, slot + R::GC, N); };
      struct Tile { int g, i; };
      const int tiles = query_tiles(a.Lq);
      const int on_g = 4 / tiles, on_i = 4 - on_g * tiles;
      auto advance = [&](Tile& t, bool more) {  // four on, unless it is the last (which is then requested again); no branch
        const int i = t.i + (more ? on_i : 0), wrap = i >= tiles;
        t.i = i - (wrap ? tiles : 0);
        t.g += (more ? on_g : 0) + wrap;
      };
      auto head = [&](const Tile& t) { return hk * a.G + t.g; };
      auto source_q = [&](const Tile& t) { return uniform64(static_cast<const uint16_t*>(a.Q) + b * a.q.b + head(t) * a.q.h + first_token(a.Lq, t.i) * a.q.l); };
      auto source_g = [&](const Tile& t) { return uniform64(static_cast<const uint16_t*>(a.dO) + b * a.go.b + head(t) * a.go.h + first_token(a.Lq, t.i) * a.go.l); };
      auto source_s = [&](const Tile& t) { return uniform64(stat + (((int64_t)b * a.H + head(t)) * tiles + t.i) * 64); };
      Tile t2{(pc.t0 + wave) / tiles, (pc.t0 + wave) % tiles};
      t2.g = __builtin_amdgcn_readfirstlane(t2.g);
      t2.i = __builtin_amdgcn_readfirstlane(t2.i);
      {
        const uint64_t g0 = source_g(t2), q0 = source_q(t2);
        static_for<0, ND>([&](auto N) { rows_g(g0, lds0, N); });
        static_for<0, ND>([&](auto N) { rows_q(q0, lds0, N); });
        dma_tail(source_s(t2), lane16, lds0 + R::LS);
        advance(t2, mine > 1);
        const uint64_t g1 = source_g(t2);
        static_for<0, ND>([&](auto N) { rows_g(g1, lds0 + R::BYTES, N); });
      }
      uint64_t q1 = source_q(t2), s1 = source_s(t2);  // the next tile's
      int flip = R::BYTES;  // from the current ring slot to the other
      uint32_t cur = lds0;  // the current slot
      // LDS offsets of the fragments (see bsa_mfma.h for the swizzle): row fragments of row col,
      // transposed ones of rows 8 h + 4 grp + .., channel tile dt; row constants of this lane's rows
      int koffs[DS], voffs[2][DT], dlo = lds0 + 16 * grp;
#pragma unroll
      for (int s = 0; s < DS; ++s) koffs[s] = lds0 + col * RB + (((2 * s + grp) ^ swz<D>(col)) << 4);
      const int L16 = lane & 15, q16 = lane >> 4, rsub = L16 >> 2, jj = L16 & 3;
      const int cl = 2 * (q16 & 1) + (jj >> 1), rhi = D == 128 ? rsub : (rsub >> 1);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
          voffs[h][dt] = lds0 + (8 * h + 4 * grp + rsub) * RB + ((((dt ^ rhi) << 2) | (cl ^ (2 * h + grp))) << 4) + 8 * (jj & 1);
      // fragment f of a record: Q rows, G rows, G^T and Q^T ((16-row step, channel tile) order)
      auto frag = [&](auto F) -> bf16x8 {
        constexpr int f = decltype(F)::value;
        if constexpr (f < DS) return frag_at(koffs[f] + R::QC);
        else if constexpr (f < 2 * DS) return frag_at(koffs[f - DS] + R::GC);
        else {
          constexpr int v = f - 2 * DS, w = v % (2 * DT), dt = w % DT, base = (v < 2 * DT ? R::GC : R::QC) + 16 * (w / DT) * RB;
          return frag_tr_at(voffs[0][dt] + base, voffs[1][dt] + base);
        }
      };
      bf16x8 fr[RING];
      auto refill = [&](auto F) {  // the ring slot of fragment f takes the one RING ahead, at the end the next record's
        constexpr int f = decltype(F)::value;
        fr[f % RING] = frag(std::integral_constant<int, (f + RING) % NF>{});
      };
      wait_vm<ND>();  // the first record has landed
      static_for<0, RING>([&](auto F) { fr[decltype(F)::value] = frag(F); });
      BSA_FENCE();
      for (int i = 0; i < mine; ++i) {
        const uint32_t other = cur + flip;
        f32x16 s[NH], dp[NH];
        bf16x8 pf[NH][2], df[NH][2];
        // ---- S = Q K^T; requests of the next record's Q rows
        static_for<0, DS>([&](auto KK) {
          constexpr int k = decltype(KK)::value;
          static_for<0, NH>([&](auto HH) {
            constexpr int h = decltype(HH)::value;
            if constexpr (k == 0) mfma_first(s[h], fr[k % RING], kf[h][k]);
            else mfma_next(s[h], fr[k % RING], kf[h][k]);
            if constexpr (h == 0) {  // (behind an MFMA of its own: a request may wait for the vector memory port)
              BSA_FENCE();
              static_for<k * ND / DS, (k + 1) * ND / DS>([&](auto N) { rows_q(q1, other, N); });
              BSA_FENCE();
            }
          });
          refill(KK);
          if constexpr (k == DS - 1) dma_tail(s1, lane16, other + R::LS);
          if constexpr (k == DS - 2) {
            int own[2] = {dlo, dlo};
            asm("" : "+v"(own[1]));
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
#pragma unroll
              for (int h = 0; h < NH; ++h) {  // one read each: a copy of the other's registers would cost vector instructions
                const f32x4 v = f4_at(own[h] + R::DL + 32 * r4);
#pragma unroll
                for (int e = 0; e < 4; ++e) dp[h][4 * r4 + e] = v[e];
              }
            }
          }
          BSA_FENCE();
        });
        // ---- dP - delta = G V^T - delta; P under it
        static_for<0, DS>([&](auto KK) {
          constexpr int k = decltype(KK)::value, ra = 16 * k / DS, rz = 16 * (k + 1) / DS;
          const std::integral_constant<int, DS + k> F{};
          float lse[rz - ra];
#pragma unroll
          for (int r = ra; r < rz; ++r) {
            if (r == ra || r % 4 == 0) {
              const f32x4 v = f4_at(dlo + R::LS + 32 * (r / 4));
#pragma unroll
              for (int q = r; q < rz && q < (r / 4) * 4 + 4; ++q)
                lse[q - ra] = v[q % 4];
            }
          }
#pragma unroll
          for (int h = 0; h < NH; ++h) {
            if (k == 0) mfma_next(dp[h], fr[F % RING], vf[h][k], s[h]);
            else mfma_next(dp[h], fr[F % RING], vf[h][k]);
#pragma unroll
            for (int r = ra; r < rz; ++r) s[h][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h][r], c2, -lse[r - ra]));
          }
          if (k == DS - 2) {
#pragma unroll
            for (int h = 0; h < NH; ++h) pf[h][0] = d_to_b(s[h], 0);
          }
          refill(F);
          BSA_FENCE();
        });
        // ---- dV^T += G^T P; dS under it
        static_for<0, 2 * DT>([&](auto VV) {
          constexpr int v = decltype(VV)::value, dt = v % DT, ra = 16 * v / (2 * DT), rz = 16 * (v + 1) / (2 * DT);
          const std::integral_constant<int, 2 * DS + v> F{};
          static_for<0, NH>([&](auto HH) {
            constexpr int h = decltype(HH)::value;
            mfma_acc<h == 0 && v % DT == 0>(dv[h][dt], fr[F % RING], pf[h][v / DT]);
            if (v == 0) order_behind(dp[h]);
#pragma unroll
            for (int r = ra; r < rz; ++r) dp[h][r] = s[h][r] * dp[h][r];
          });
          if (v == 0) {
#pragma unroll
            for (int h = 0; h < NH; ++h) pf[h][1] = d_to_b(s[h], 1);
          }
          if (v == 2 * DT - 2) {
#pragma unroll
            for (int h = 0; h < NH; ++h) df[h][0] = d_to_b(dp[h], 0);
          }
          refill(F);
          BSA_FENCE();
        });
        // ---- dK^T += Q^T dS; requests of the G rows two records ahead (this record's are free now)
        advance(t2, i + 2 < mine);
        const uint64_t g2 = source_g(t2);
        static_for<0, 2 * DT>([&](auto VV) {
          constexpr int v = decltype(VV)::value, dt = v % DT;
          const std::integral_constant<int, 2 * DS + 2 * DT + v> F{};
          if constexpr (v == 2 * DT - RING) {  // the next record has landed once only these G rows are outstanding
            wait_vm<(2 * DT - RING) * ND / (2 * DT)>();
#pragma unroll
            for (int q = 0; q < DS; ++q) koffs[q] += flip;
          }
          static_for<0, NH>([&](auto HH) {
            constexpr int h = decltype(HH)::value;
            mfma_acc<h == 0 && v % DT == 0>(dk[h][dt], fr[F % RING], df[h][v / DT]);
            if constexpr (h == 0) {
              BSA_FENCE();
              static_for<v * ND / (2 * DT), (v + 1) * ND / (2 * DT)>([&](auto N) { rows_g(g2, cur, N); });
              BSA_FENCE();
            }
          });
          if (v == 0) {
#pragma unroll
            for (int h = 0; h < NH; ++h) df[h][1] = d_to_b(dp[h], 1);
          }
          refill(F);
          BSA_FENCE();
        });
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) voffs[h][dt] += flip;
        dlo += flip;
        cur = other;
        flip = -flip;
        q1 = source_q(t2);
        s1 = source_s(t2);
      }
      BSA_WAIT_VM(0);
      asm volatile("s_nop 15\n\ts_nop 15");  // the last accumulations land before anything reads them
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) asm volatile("" : "+a"(dk[h][dt]), "+a"(dv[h][dt]));
    }

    // sum of the four wavefronts, in order, through the idle ring: dK then dV
    f32x4* red = reinterpret_cast<f32x4*>(smem) + lane;  // [tile][wavefront][4][64]
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
      __syncthreads();
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const f32x16& acc = pass ? dv[h][dt] : dk[h][dt];
#pragma unroll
          for (int r4 = 0; r4 < 4; ++r4)
            red[(((h * DT + dt) * 4 + wave) * 4 + r4) * 64] = f32x4{acc[4 * r4], acc[4 * r4 + 1], acc[4 * r4 + 2], acc[4 * r4 + 3]};
        }
      __syncthreads();
      const auto& st = pass ? a.gv : a.gk;
      uint16_t* out = static_cast<uint16_t*>(pass ? a.dV : a.dK) + b * st.b + hk * st.h;
      const float scale = pass ? 1.f : a.sm_scale;
      for (int t = wave * NT / 4; t < (wave + 1) * NT / 4; ++t) {
        const int h = t / DT, key = first + 32 * h + col;
        f32x16 v[1];
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          f32x4 x = red[(t * 16 + r4) * 64];
#pragma unroll
          for (int w = 1; w < 4; ++w) x += red[(t * 16 + 4 * w + r4) * 64];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[0][4 * r4 + e] = (valid >> (32 * h + col)) & 1 ? x[e] : 0.f;  // no key, no gradient
        }
        if (pc.slot < 0) {
          store_column<uint16_t, 1>(out + key * st.l + 32 * (t % DT), v, scale, a.d - 32 * (t % DT), grp, key < a.S);
        } else {
          float* to = part + (((int64_t)pc.slot * 2 + pass) * NT + t) * 1024 + lane;
#pragma unroll
          for (int r = 0; r < 16; ++r) to[r * 64] = v[0][r];
        }
      }
    }
    __syncthreads();  // the ring is free
  }
}

// Joins the parts of a unit, and writes the zeros of the units that had no step.  A wavefront has 32 channels of 32 keys.
template <int D>
__global__ __launch_bounds__(2 * D, 1) void cross_dkv_fast_combine_kernel(CrossArgs, Deal dl, const float* part) {
  Args& a = *kernel_args();
  constexpr int DT = D / 32, NT = 2 * DT;
  const int lane = threadIdx.x & 63, dt = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = blockIdx.y, pass = blockIdx.z;
  const int b = (int)(blockIdx.x / (uint32_t)dl.rows), unit = (int)blockIdx.x - b * dl.rows;
  const Parts ps(a, dl, lane, b, unit);
  if (ps.n == 0) return;
  const int tile = (int)((uint32_t)unit / (uint32_t)a.Hkv), hk = unit - tile * a.Hkv, key = tile * kKeys + 32 * h + (lane & 31);
  f32x16 acc[1];
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[0][r] = 0.f;
  for (int s = 0; s < ps.n; s += 8) {
    float v[8][16];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float* in = part + (((int64_t)ps.slot(min(s + j, ps.n - 1)) * 2 + pass) * NT + h * DT + dt) * 1024 + lane;
#pragma unroll
      for (int r = 0; r < 16; ++r) v[j][r] = in[r * 64];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (s + j < ps.n)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[0][r] += v[j][r];
  }
  const auto& st = pass ? a.gv : a.gk;
  uint16_t* out = static_cast<uint16_t*>(pass ? a.dV : a.dK) + b * st.b + hk * st.h + key * st.l + 32 * dt;
  store_column<uint16_t, 1>(out, acc, pass ? 1.f : a.sm_scale, a.d - 32 * dt, lane >> 5, key < a.S);
}

// One workgroup a CU; a share of sixteen tiles (four a wavefront) at least, or a piece's loads and sums are all that it does.
static Deal fast_deal(const CrossArgs& a) {
  Deal d{};
  d.by_keys = 1;
  d.way = SHARES;
  d.tile = kKeys;
  d.steps = a.G * query_tiles(a.Lq);
  d.rows = a.Hkv * ((a.S + kKeys - 1) / kKeys);
  d.grid = (int)std::min<int64_t>(256, std::max<int64_t>(1, (int64_t)d.rows * a.B * d.steps / 16));
  return d;
}

size_t cross_dkv_fast_parts(const CrossArgs& a) { return (size_t)fast_deal(a).grid * 2 * 2 * kKeys * (a.d <= 64 ? 64 : 128) * sizeof(float); }

template <int D> static constexpr size_t lds_bytes() { return (size_t)8 * BwdRec<D>::BYTES; }

template <int D>
static int launch_t(const CrossArgs& a, const float* stat, float* part, hipStream_t st) {
  const Deal d = fast_deal(a);
  if (a.d == D) hipLaunchKernelGGL((cross_dkv_fast_kernel<D, true>), dim3(d.grid), dim3(256), lds_bytes<D>(), st, a, d, stat, part);
  else hipLaunchKernelGGL((cross_dkv_fast_kernel<D, false>), dim3(d.grid), dim3(256), lds_bytes<D>(), st, a, d, stat, part);
  if (const int rc = check_launch()) return rc;
  hipLaunchKernelGGL((cross_dkv_fast_combine_kernel<D>), dim3((unsigned)d.rows * a.B, 2, 2), dim3(2 * D), 0, st, a, d, part);
  return check_launch();
}

template <int D>
static int grant_t(const CrossArgs& a) {
  return a.d == D ? allow_dynamic_lds<cross_dkv_fast_kernel<D, true>>(lds_bytes<D>()) : allow_dynamic_lds<cross_dkv_fast_kernel<D, false>>(lds_bytes<D>());
}
int grant_cross_dkv_fast(const CrossArgs& a) { return a.d <= 64 ? grant_t<64>(a) : grant_t<128>(a); }

int launch_cross_dkv_fast(const CrossArgs& a, const float* stat, float* part, hipStream_t st) {
  return a.d <= 64 ? launch_t<64>(a, stat, part, st) : launch_t<128>(a, stat, part, st);
}

}  // namespace bsa
