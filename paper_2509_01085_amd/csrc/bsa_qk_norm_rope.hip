// Per-head RMS norm of queries and keys and their rotation by grid position, from the projection's output [B, L, H, d] to the
// attention's [B, H, L, d] (raster or block-major), values moved along; and the backward.
//
//   xhat = x r, r = 1 / sqrt(mean(x^2) + eps);  y = R (w xhat)
//   u = R^T dy;  dw = sum u xhat;  g = w u;  dx = r (g - xhat mean(g xhat))
//
// What bounds it: memory.  Every element is read once and written once (backward: x and dy read, dx written), some ten
// operations each.  A row (the d channels of a head's token) lies in 2^k lanes, eight channels each, so a wavefront holds
// 64 / 2^k rows: consecutive tokens of the result, whose writes are one run.  A lane keeps its tokens' cosines and sines in
// registers for all heads, and the row sums are register exchanges.  Of queries, keys and values a workgroup has one: with all three
// the backward held two sets of weights and sums, which left three wavefronts a SIMD (33,280 tokens, 12 heads, d = 128, bf16: 197 us,
// now 170).
//
// Measured there: forward 117 us for 614 MB (5.2 TB/s), backward 170 for 818 MB (4.8); a copy reaches 4.7.  70,400 tokens, 40 heads,
// block-major: 857 us for 4.3 GB (5.1).  fp32: 242 and 332 us (5.1 and 4.9).  d = 72 leaves seven of sixteen lanes without channels: two batch
// entries of 32,760 tokens, 4 heads, 44 and 80 us (5.1 and 3.8 TB/s).
#include "bsa_common.h"

namespace bsa {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;

// ---- eight channels of a lane, in two pieces of four at p + o0 and p + o1 (elements) ----
template <bool SPLIT>
__device__ inline void load8(const uint16_t* p, int o0, int o1, float x[8]) {
  u32x4 v;
  if (SPLIT) {
    const u32x2 a = *reinterpret_cast<const u32x2*>(p + o0), b = *reinterpret_cast<const u32x2*>(p + o1);
    v = u32x4{a.x, a.y, b.x, b.y};
  } else {
    v = *reinterpret_cast<const u32x4*>(p + o0);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(v[i] << 16);
    x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
  }
}
template <bool SPLIT>
__device__ inline void load8(const float* p, int o0, int o1, float x[8]) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p + o0), b = *reinterpret_cast<const f32x4*>(p + o1);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = a[i];
    x[4 + i] = b[i];
  }
}
__device__ inline uint32_t pack2(float lo, float hi) {
  typedef __attribute__((ext_vector_type(2))) float f32x2;
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  const f32x2 v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
template <bool SPLIT>
__device__ inline void store8(uint16_t* p, int o0, int o1, const float x[8]) {
  const u32x4 v = {pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])};
  if (SPLIT) {
    *reinterpret_cast<u32x2*>(p + o0) = u32x2{v.x, v.y};
    *reinterpret_cast<u32x2*>(p + o1) = u32x2{v.z, v.w};
  } else {
    *reinterpret_cast<u32x4*>(p + o0) = v;
  }
}
template <bool SPLIT>
__device__ inline void store8(float* p, int o0, int o1, const float x[8]) {
  *reinterpret_cast<f32x4*>(p + o0) = f32x4{x[0], x[1], x[2], x[3]};
  *reinterpret_cast<f32x4*>(p + o1) = f32x4{x[4], x[5], x[6], x[7]};
}

// Sum over the LPR lanes of a row, the same value in all of them: lane exchanges by data-parallel primitives.
template <int CTRL>
__device__ inline float dpp_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int LPR>
__device__ inline float row_sum(float v) {
  v = dpp_add<0xB1>(v);                       // lane ^ 1
  v = dpp_add<0x4E>(v);                       // lane ^ 2
  if (LPR >= 8) v = dpp_add<0x141>(v);        // mirrored within 8: the other four
  if (LPR >= 16) v = dpp_add<0x140>(v);       // mirrored within 16: the other eight
  if (LPR >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return v;
}

// What a lane knows of its place: which channels, and how they turn.
template <int LPR, bool HALVES>
struct Place {
  int c, o0, o1, rows_at;
  bool live, turns;
  int pair[4], axis;  // of the lane's four pairs: number on its axis; axes, two bits each

  __device__ inline Place(const Geom& g, const RopeArgs& a, int lane) {
    c = lane & (LPR - 1);
    rows_at = lane / LPR;
    live = 8 * c < g.d;
    const int np = a.nt + a.nh + a.nw;
    turns = live && 4 * c < np;
    o0 = live ? 8 * c : 0;  // (lanes past d take part in the sums, with nothing)
    o1 = o0 + 4;
    if (HALVES && turns) {
      o0 = 4 * c;
      o1 = np + o0;
    }
    axis = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = 4 * c + i, x = p < a.nt ? 0 : p < a.nt + a.nh ? 1 : 2;
      axis |= x << (2 * i);
      pair[i] = p - (x == 0 ? 0 : x == 1 ? a.nt : a.nt + a.nh);
    }
  }
  __device__ inline void weights(const float* from, float w[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = from ? from[(i < 4 ? o0 : o1 - 4) + i] : 1.f;
  }
  // cosines and sines of raster token n (unturned: 1, 0)
  __device__ inline void angles(const Geom& g, const RopeArgs& a, int n, float cs[4], float sn[4]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) { cs[i] = 1.f; sn[i] = 0.f; }
    if (!turns) return;
    const uint32_t th = (uint32_t)n / (uint32_t)g.Ws, t = th / (uint32_t)g.Hs;
    const int w = n - (int)th * g.Ws, h = (int)(th - t * (uint32_t)g.Hs);
    const int64_t at[3] = {(int64_t)t * a.nt, (int64_t)g.T * a.nt + (int64_t)h * a.nh,
                           (int64_t)g.T * a.nt + (int64_t)g.Hs * a.nh + (int64_t)w * a.nw};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int x = (axis >> (2 * i)) & 3;
      const float2 v = reinterpret_cast<const float2*>(a.table)[(x == 0 ? at[0] : x == 1 ? at[1] : at[2]) + pair[i]];
      cs[i] = v.x;
      sn[i] = v.y;
    }
  }
};

template <bool HALVES>
__device__ inline void turn(float x[8], const float cs[4], const float sn[4], float sign) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int lo = HALVES ? i : 2 * i, hi = HALVES ? 4 + i : 2 * i + 1;
    const float u = x[lo], v = x[hi], s = sign * sn[i];
    x[lo] = __builtin_fmaf(u, cs[i], -(v * s));
    x[hi] = __builtin_fmaf(u, s, v * cs[i]);
  }
}

// Raster token of row m of a result in the shape's order.
__device__ inline int raster_token(const Geom& g, int m) {
  if (!g.tiled) return m;
  const int i = m / g.Bk, k = m - i * g.Bk;
  const int bw = i % g.Nw, bh = (i / g.Nw) % g.Nh, bt = i / (g.Nw * g.Nh);
  const int cw = k % g.Cw, ch = (k / g.Cw) % g.Ch, ct = k / (g.Cw * g.Ch);
  return ((bt * g.Ct + ct) * g.Hs + (bh * g.Ch + ch)) * g.Ws + (bw * g.Cw + cw);
}

// Rows of the values, which are only moved: HB heads of them in flight.
template <typename T, int HB>
__device__ inline void move_rows(const T* from, int64_t fs, T* to, int64_t ts, int h0, int h1) {
  constexpr int NV = sizeof(T) * 8 / 16;
  for (int h = h0; h < h1; h += HB) {
    u32x4 v[HB][NV];
#pragma unroll
    for (int j = 0; j < HB; ++j)
#pragma unroll
      for (int i = 0; i < NV; ++i) v[j][i] = reinterpret_cast<const u32x4*>(from + min(h + j, h1 - 1) * fs)[i];
#pragma unroll
    for (int j = 0; j < HB; ++j)
      if (h + j < h1)
#pragma unroll
        for (int i = 0; i < NV; ++i) reinterpret_cast<u32x4*>(to + (h + j) * ts)[i] = v[j][i];
  }
}

// A workgroup has one of the tensors (blockIdx.z counts those that are there), 4 * 64 / LPR rows of the result and a range of heads (blockIdx.y).
__device__ inline int tensor_of(int have) {  // the blockIdx.z-th bit
  int z = blockIdx.z;
  for (int i = 0; i < 3; ++i)
    if ((have >> i) & 1 && z-- == 0) return i;
  return 0;
}
template <typename P>
__device__ inline P pick(P const (&p)[3], int z) { return z == 0 ? p[0] : z == 1 ? p[1] : p[2]; }

template <typename T, int LPR, bool HALVES>
__global__ __launch_bounds__(256) void rope_fwd_kernel(Geom g, RopeArgs a, int heads, int have) {
  constexpr int RPW = 64 / LPR, HB = 4;  // rows of a wavefront, heads in flight
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, z = tensor_of(have);
  const Place<LPR, HALVES> pl(g, a, lane);
  const int64_t at = ((int64_t)blockIdx.x * 4 + wave) * RPW + pl.rows_at;  // row of the results, over the batch
  if (at >= (int64_t)g.B * g.L) return;                                   // (a row's lanes leave together)
  const int b = (int)((uint32_t)at / (uint32_t)g.L), m = (int)at - b * g.L, n = raster_token(g, m);
  const int h0 = blockIdx.y * heads, h1 = min(h0 + heads, g.H);
  const T* X = static_cast<const T*>(pick(a.X, z)) + b * a.x.b + n * a.x.l;
  T* Y = static_cast<T*>(pick(a.Y, z)) + ((int64_t)b * g.H * g.L + m) * g.d;
  const int64_t ys = (int64_t)g.L * g.d;
  if (z == 2) {
    if (pl.live) move_rows<T, HB>(X + 8 * pl.c, a.x.h, Y + 8 * pl.c, ys, h0, h1);
    return;
  }
  float cs[4], sn[4], w[8];
  pl.angles(g, a, n, cs, sn);
  pl.weights(z ? a.w[1] : a.w[0], w);
  const float inv_d = 1.f / g.d;
  for (int h = h0; h < h1; h += HB) {
    float x[HB][8];
#pragma unroll
    for (int j = 0; j < HB; ++j) load8<HALVES>(X + min(h + j, h1 - 1) * a.x.h, pl.o0, pl.o1, x[j]);
#pragma unroll
    for (int j = 0; j < HB; ++j) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) s = __builtin_fmaf(x[j][i], x[j][i], s);
      const float r = __builtin_amdgcn_rsqf(__builtin_fmaf(row_sum<LPR>(pl.live ? s : 0.f), inv_d, a.eps));
#pragma unroll
      for (int i = 0; i < 8; ++i) x[j][i] = x[j][i] * r * w[i];
      if (pl.turns) turn<HALVES>(x[j], cs, sn, 1.f);
      if (pl.live && h + j < h1) store8<HALVES>(Y + (h + j) * ys, pl.o0, pl.o1, x[j]);
    }
  }
}

// Backward.  A workgroup takes groups of rows in turn and keeps its share of its tensor's dw in registers; the workgroups' shares
// are added up by a second launch, in a fixed order.
template <typename T, int LPR, bool HALVES>
__global__ __launch_bounds__(256) void rope_bwd_kernel(Geom g, RopeArgs a, int heads, int have) {
  constexpr int RPW = 64 / LPR, HB = 2;
  __shared__ float red[4][64][8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, z = tensor_of(have);
  const Place<LPR, HALVES> pl(g, a, lane);
  const int h0 = blockIdx.y * heads, h1 = min(h0 + heads, g.H);
  const float inv_d = 1.f / g.d;
  const int64_t rows = (int64_t)g.B * g.L, ys = (int64_t)g.L * g.d;
  const T* dYz = static_cast<const T*>(pick(a.dY, z));
  T* dXz = static_cast<T*>(pick(a.dX, z));
  const T* Xz = static_cast<const T*>(z == 0 ? a.X[0] : a.X[1]);
  float dw[8], w[8];
  if (z < 2) pl.weights(z ? a.w[1] : a.w[0], w);
#pragma unroll
  for (int i = 0; i < 8; ++i) dw[i] = 0.f;
  for (int64_t first = ((int64_t)blockIdx.x * 4 + wave) * RPW; first < rows; first += (int64_t)gridDim.x * 4 * RPW) {
    const int64_t at = first + pl.rows_at;
    if (at >= rows) continue;
    const int b = (int)((uint32_t)at / (uint32_t)g.L), m = (int)at - b * g.L, n = raster_token(g, m);
    const T* dY = dYz + ((int64_t)b * g.H * g.L + m) * g.d;
    T* dX = dXz + b * a.dx.b + n * a.dx.l;
    if (z == 2) {
      if (pl.live) move_rows<T, 4>(dY + 8 * pl.c, ys, dX + 8 * pl.c, a.dx.h, h0, h1);
      continue;
    }
    const T* X = Xz + b * a.x.b + n * a.x.l;
    float cs[4], sn[4];
    pl.angles(g, a, n, cs, sn);
    for (int h = h0; h < h1; h += HB) {
      float x[HB][8], u[HB][8];
#pragma unroll
      for (int j = 0; j < HB; ++j) {
        load8<HALVES>(X + min(h + j, h1 - 1) * a.x.h, pl.o0, pl.o1, x[j]);
        load8<HALVES>(dY + min(h + j, h1 - 1) * ys, pl.o0, pl.o1, u[j]);
      }
#pragma unroll
      for (int j = 0; j < HB; ++j) {
        if (pl.turns) turn<HALVES>(u[j], cs, sn, -1.f);
        const bool there = pl.live && h + j < h1;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s = __builtin_fmaf(x[j][i], x[j][i], s);
        const float r = __builtin_amdgcn_rsqf(__builtin_fmaf(row_sum<LPR>(pl.live ? s : 0.f), inv_d, a.eps));
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[j][i] *= r;
          if (there) dw[i] = __builtin_fmaf(u[j][i], x[j][i], dw[i]);
          u[j][i] *= w[i];
          t = __builtin_fmaf(u[j][i], x[j][i], t);
        }
        t = row_sum<LPR>(pl.live ? t : 0.f) * inv_d;
#pragma unroll
        for (int i = 0; i < 8; ++i) u[j][i] = r * __builtin_fmaf(-x[j][i], t, u[j][i]);
        if (there) store8<HALVES>(dX + (h + j) * a.dx.h, pl.o0, pl.o1, u[j]);
      }
    }
  }
  if (z == 2 || !(z ? a.dw[1] : a.dw[0])) return;
  // the workgroup's sums: its 4 * RPW row slots in a fixed order
#pragma unroll
  for (int i = 0; i < 8; ++i) red[wave][lane][i] = dw[i];
  __syncthreads();
  if (threadIdx.x < LPR && pl.live) {
    const int64_t wg = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    float* out = a.part + (wg * 2 + z) * g.d;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float s = 0.f;
#pragma unroll 1
      for (int v = 0; v < 4; ++v)
        for (int k = 0; k < RPW; ++k) s += red[v][k * LPR + lane][i];
      out[(i < 4 ? pl.o0 : pl.o1 - 4) + i] = s;
    }
  }
}

// dw: sums over the workgroups' shares, fp64.  16 channels and 64 shares a workgroup at a time.
__global__ __launch_bounds__(1024) void rope_dw_kernel(const float* part, int n, int d, float* dwq, float* dwk) {
  __shared__ double red[64][16];
  float* out = blockIdx.y ? dwk : dwq;
  if (!out) return;
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), k = threadIdx.x >> 4;
  double s = 0.;
  if (c < d)
#pragma unroll 8
    for (int i = k; i < n; i += 64) s += part[((int64_t)i * 2 + blockIdx.y) * d + c];
  red[k][threadIdx.x & 15] = s;
  __syncthreads();
  if (k < 8) {
    for (int i = 1; i < 8; ++i) s += red[8 * i + k][threadIdx.x & 15];
    red[k][threadIdx.x & 15] = s;  // (row k is read by this thread alone above)
  }
  __syncthreads();
  if (k == 0 && c < d) {
    for (int i = 1; i < 8; ++i) s += red[i][threadIdx.x & 15];
    out[c] = (float)s;
  }
}

__global__ __launch_bounds__(256) void rope_table_kernel(Geom g, int nt, int nh, int nw, double log_theta, double t0, double h0,
                                                         double w0, float2* table) {
  const int64_t a = (int64_t)g.T * nt, b = a + (int64_t)g.Hs * nh, all = b + (int64_t)g.Ws * nw;
  for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < all; k += (int64_t)gridDim.x * 256) {
    const int n = k < a ? nt : k < b ? nh : nw;
    const int64_t at = k - (k < a ? 0 : k < b ? a : b);
    const double pos = (k < a ? t0 : k < b ? h0 : w0) + (double)(at / n);
    const double angle = pos * exp(-log_theta * (double)(at % n) / n);
    table[k] = make_float2((float)cos(angle), (float)sin(angle));
  }
}

constexpr int kBwdGroups = 1024;  // workgroups of a tensor's backward at most: each leaves d sums

// Heads of a workgroup and workgroups along them: all heads, unless that leaves the chip short of wavefronts.
static int head_split(int64_t groups, int H) {
  const int64_t want = (1024 + groups - 1) / groups;
  const int parts = (int)(want < 1 ? 1 : want > H ? H : want);
  return (H + parts - 1) / parts;
}

static int lanes_of(int d) { return d <= 32 ? 4 : d <= 64 ? 8 : d <= 128 ? 16 : 32; }

bool rope_fits(const Geom& g) { return (int64_t)g.B * g.L * lanes_of(g.d) < 0xffffff00LL; }  // a launch has fewer than 2^32 threads

static dim3 bwd_grid(const Geom& g, int* heads) {
  const int rpw = 64 / lanes_of(g.d);
  const int64_t groups = ((int64_t)g.B * g.L + 4 * rpw - 1) / (4 * rpw);
  *heads = head_split(groups, g.H);
  const int parts = (g.H + *heads - 1) / *heads;
  const int64_t most = kBwdGroups / parts;  // (head_split leaves parts > 1 only where groups * parts is about 1024)
  return dim3((unsigned)(groups < most ? groups : most < 1 ? 1 : most), parts);
}

size_t rope_bwd_workspace(const Geom& g) {
  int heads;
  const dim3 n = bwd_grid(g, &heads);
  return (size_t)n.x * n.y * 2 * g.d * sizeof(float);
}

template <typename T, int LPR, bool HALVES>
static int launch_t(const Geom& g, const RopeArgs& a, bool backward, hipStream_t st) {
  int heads, have = 0, tensors = 0;
  for (int i = 0; i < 3; ++i)
    if (backward ? a.dY[i] != nullptr : a.X[i] != nullptr) {
      have |= 1 << i;
      ++tensors;
    }
  if (backward) {
    dim3 grid = bwd_grid(g, &heads);
    const int shares = (int)(grid.x * grid.y);
    grid.z = tensors;
    hipLaunchKernelGGL((rope_bwd_kernel<T, LPR, HALVES>), grid, dim3(256), 0, st, g, a, heads, have);
    if (const int rc = check_launch()) return rc;
    if (!a.dw[0] && !a.dw[1]) return BSA_OK;
    hipLaunchKernelGGL(rope_dw_kernel, dim3((g.d + 15) / 16, 2), dim3(1024), 0, st, a.part, shares, g.d, a.dw[0], a.dw[1]);
    return check_launch();
  }
  constexpr int RPW = 64 / LPR;
  const int64_t groups = ((int64_t)g.B * g.L + 4 * RPW - 1) / (4 * RPW);
  heads = head_split(groups, g.H);
  hipLaunchKernelGGL((rope_fwd_kernel<T, LPR, HALVES>), dim3((unsigned)groups, (g.H + heads - 1) / heads, tensors), dim3(256), 0, st, g, a, heads, have);
  return check_launch();
}

template <typename T>
static int launch(const Geom& g, const RopeArgs& a, bool backward, hipStream_t st) {
  switch (lanes_of(g.d)) {
    case 4: return a.halves ? launch_t<T, 4, true>(g, a, backward, st) : launch_t<T, 4, false>(g, a, backward, st);
    case 8: return a.halves ? launch_t<T, 8, true>(g, a, backward, st) : launch_t<T, 8, false>(g, a, backward, st);
    case 16: return a.halves ? launch_t<T, 16, true>(g, a, backward, st) : launch_t<T, 16, false>(g, a, backward, st);
    default: return a.halves ? launch_t<T, 32, true>(g, a, backward, st) : launch_t<T, 32, false>(g, a, backward, st);
  }
}

int launch_rope_fwd(const Geom& g, int dtype, const RopeArgs& a, hipStream_t st) {
  return dtype == BSA_F32 ? launch<float>(g, a, false, st) : launch<uint16_t>(g, a, false, st);
}

int launch_rope_bwd(const Geom& g, int dtype, const RopeArgs& a, hipStream_t st) {
  return dtype == BSA_F32 ? launch<float>(g, a, true, st) : launch<uint16_t>(g, a, true, st);
}

int launch_rope_table(const Geom& g, const RopeArgs& a, double theta, const double origin[3], float* table, hipStream_t st) {
  const int64_t n = (int64_t)g.T * a.nt + (int64_t)g.Hs * a.nh + (int64_t)g.Ws * a.nw;
  if (n == 0) return BSA_OK;
  const int64_t grid = (n + 255) / 256;
  hipLaunchKernelGGL(rope_table_kernel, dim3((unsigned)(grid < 4096 ? grid : 4096)), dim3(256), 0, st, g, a.nt, a.nh, a.nw, log(theta),
                     origin[0], origin[1], origin[2], reinterpret_cast<float2*>(table));
  return check_launch();
}

}  // namespace bsa
