// The first half of a gated MLP: act(x gate) * (x up), and its gradients, as products in tiles (g10_tile.h).
//
// Bound by the matrix unit with many tokens, by the weights' bytes with few.  Forward both products are one kernel: a tile's two
// panels are the same columns of both weights, and the activation and the product are taken from the sums in the registers; neither
// factor goes to memory.  Backward the same kernel makes g and u again and turns dh into dg and du (rounded to 16 bits: the next products take
// them so), then one kernel makes dx (its sum goes over gate's columns and on over up's) and one the gradients of both weights.
// Where the tiles are too few to fill the chip the sum over k is cut into shares: these go to memory in 32 bits, and a second kernel
// adds them in order and does what the tiles' end would have done.
#include "g10_tile.h"

enum { END_GATED = 0, END_BACK = 1, END_PLAIN = 2 };

struct GatedArgs {
  const void *a[2], *b[2];         // the first factor's sources; the second one's (gate and up)
  void* out[2];                    // h | dg, du | the product (the gradients of both weights: one each)
  const void* dh;
  int64_t as, bs, os, dhs;         // strides of rows
  u32 m, n, k, sources;            // rows, columns (of each of two panels where gated), values of k in a source
  u32 n8;                          // columns up to a multiple of 8, which all inputs' rows go on to
  u32 tiles_m, tiles_n;
  u32 products, shares, per;       // products of their own (both weights' gradients); shares of the sum over k, of `per` steps
  u32 act;
  float* part;                     // [product][share][m][columns]
};

// h's activation and its slope.
struct Act { float a, slope; };
__device__ __forceinline__ Act activation(float g, u32 act, bool slope) {
  if (act == G10_ACT_SILU) {
    const float s = __builtin_amdgcn_rcpf(1.0f + exp2_fast(-g * G10_LOG2E));
    return {g * s, slope ? s * (1.0f + g * (1.0f - s)) : 0.0f};
  }
  const float s = 0.5f * erfcf(-0.70710678118654752f * g);
  return {g * s, slope ? s + g * 0.3989422804014327f * exp2_fast(-0.5f * G10_LOG2E * g * g) : 0.0f};
}

// What comes of N neighbouring columns of a row: both panels' sums in g and u (END_PLAIN: g alone), to column c.  d: dh there.  Outputs may lie
// anywhere and end where they like (accesses to memory need not be aligned); dg and du go on to n8, with the zeros of dh.
template <class T, int END, int N>
struct Ends {
  typedef T V __attribute__((ext_vector_type(N), aligned(sizeof(T))));
  static __device__ __forceinline__ V dh_at(const GatedArgs& a, u32 row, u32 c) {
    const bool in = row < a.m && c < a.n8;
    return *(const V*)((const T*)a.dh + (in ? (int64_t)row * a.dhs + c : 0));
  }
  static __device__ __forceinline__ void store(const GatedArgs& a, u32 which, u32 row, u32 c, const V& w) {
    T* to = (T*)(which ? a.out[1] : a.out[0]) + (int64_t)row * a.os + c;
    if (END == END_BACK || c + N <= a.n) {
      *(V*)to = w;
    } else {
#pragma unroll
      for (int r = 0; r < N; ++r)
        if (c + r < a.n) to[r] = w[r];
    }
  }
  static __device__ __forceinline__ void put(const GatedArgs& a, u32 which, u32 row, u32 c, const float (&g)[N], const float (&u)[N], const V& d) {
    if (row >= a.m || c >= (END == END_BACK ? a.n8 : a.n)) return;
    V w0, w1;
#pragma unroll
    for (int r = 0; r < N; ++r) {
      if constexpr (END == END_GATED) {
        w0[r] = (T)(activation(g[r], a.act, false).a * u[r]);
      } else if constexpr (END == END_BACK) {
        const Act t = activation(g[r], a.act, true);
        w0[r] = (T)((float)d[r] * u[r] * t.slope);
        w1[r] = (T)((float)d[r] * t.a);
      } else {
        w0[r] = (T)g[r];
      }
    }
    store(a, END == END_PLAIN ? which : 0, row, c, w0);
    if constexpr (END == END_BACK) store(a, 1, row, c, w1);
  }
};
// A result's registers 8 q .. 8 q + 7 hold a row's columns 16 q + 4 h .. + 3 and 16 q + 8 + 4 h .. + 3 in the halves h of a wavefront; exchanged, eight
// neighbouring ones from 16 q + 8 h on.
__device__ __forceinline__ void neighbours(const f32x16& x, int q, float (&y)[8]) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const u32x2 s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x[8 * q + r]), __float_as_uint(x[8 * q + 4 + r]), false, false);
    y[r] = __uint_as_float(s[0]);
    y[4 + r] = __uint_as_float(s[1]);
  }
}

template <class T, int LA, int LB, int WM, int WN, int TM, int KS, int STAGES, int END>
__global__ __launch_bounds__(64 * WM * WN, (WM * WN == 8 || Tile<T, LA, LB, WM, WN, TM, KS, STAGES>::LDS <= 80 * 1024 ? 2 : 1)) void k_gated(const GatedArgs a) {
  typedef Tile<T, LA, LB, WM, WN, TM, KS, STAGES> Tl;
  typedef typename Tl::PA PA;
  typedef typename Tl::PB PB;
  constexpr bool GATED = END != END_PLAIN;
  constexpr u32 WIDE = Tl::WIDE;                                       // columns of a panel
  __shared__ __attribute__((aligned(256))) char lds[Tl::LDS];
  // Workgroups go round the 8 XCDs by their number: each XCD gets a run of tiles, eight tiles of rows side by side, so that the panels that its 32
  // units read at a time lie in its L2.
  const u32 tiles = a.tiles_m * a.tiles_n, all = tiles * a.products * a.shares, each = (all + 7) / 8;
  const u32 id = (blockIdx.x % 8) * each + blockIdx.x / 8;
  if (blockIdx.x / 8 >= each || id >= all) return;
  const u32 group = id / tiles, t = id % tiles, band = t / (8 * a.tiles_n), high = a.tiles_m - band * 8 < 8 ? a.tiles_m - band * 8 : 8;
  const u32 in = t - band * 8 * a.tiles_n, m0 = (band * 8 + in % high) * Tl::BM, n0 = in / high * (GATED ? WIDE : 2 * WIDE);
  const u32 which = group / a.shares, share = group % a.shares;
  const u32 nk = (a.k + KS - 1) / KS, first = share * a.per, last = first + a.per < nk * a.sources ? first + a.per : nk * a.sources;
  PA pa[Tl::APANELS];
  PB pb[2];
  u32 am[Tl::APANELS], bn[2];
#pragma unroll
  for (int i = 0; i < Tl::APANELS; ++i) {
    am[i] = m0 + i * 128 < a.m ? m0 + i * 128 : 0;                     // (a panel with nothing in it: the first one, which nobody keeps)
    pa[i].init(threadIdx.x, a.as, am[i], a.m);
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    bn[j] = GATED ? n0 : n0 + j * WIDE < a.n ? n0 + j * WIDE : 0;
    pb[j].init(threadIdx.x, a.bs, bn[j], a.n);
  }
  // (a sum over two sources takes both factors from the second one there; products of their own differ in one factor)
  typename Tl::Walk w;
  u32 src = first >= nk;
  auto place = [&](typename Tl::Walk& w, u32 step) {
    const void* pa0 = a.a[a.sources > 1 ? src : which];
#pragma unroll
    for (int i = 0; i < Tl::APANELS; ++i) w.a[i] = PA::start(pa0, a.as, am[i], step);
#pragma unroll
    for (int j = 0; j < 2; ++j) w.b[j] = PB::start(a.b[GATED ? (u32)j : a.sources > 1 ? src : which], a.bs, bn[j], step);
    w.left = a.k - step * KS;
  };
  place(w, first - src * nk);
  const u32 l = lane_id(), wave = uniform(wave_id()), row0 = m0 + (wave / WN) * 32 * TM + (l & 31), c0 = n0 + (wave % WN) * 32 + 8 * (l >> 5);
  typedef Ends<T, END, 8> E;
  // (dh is on its way while the tile's first panels are: at the end its latency would be all there is to do)
  typename E::V dh[END == END_BACK ? TM : 1][2];
  if constexpr (END == END_BACK) {
    if (a.shares == 1) {
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int q = 0; q < 2; ++q) dh[i][q] = E::dh_at(a, row0 + 32 * i, c0 + 16 * q);
    }
  }
  f32x16 acc[2][TM] = {};
  Tl::run(acc, lds_addr(lds), (int)(last - first), pa, pb, w, PA::bytes(a.as), PB::bytes(a.bs), a.sources == 1 || a.k % KS == 0, [&](typename Tl::Walk& w) {
    src = 1;
    if (a.sources > 1) place(w, 0);
  });
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const u32 row = row0 + 32 * i;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const u32 c = c0 + 16 * q;
      float g[8], u[8];
      neighbours(acc[0][i], q, g);
      neighbours(acc[1][i], q, u);
      if (a.shares > 1) {
        const u64 wide = GATED ? 2ull * a.n8 : a.n8;
        float* to = a.part + ((u64)group * a.m + row) * wide + c;
#pragma unroll
        for (int r = 0; r < 8; r += 4) {
          if (row < a.m && c < a.n8) *(f32x4*)(to + r) = f32x4{g[r], g[r + 1], g[r + 2], g[r + 3]};
          if (row < a.m && (GATED ? c : c + WIDE) < a.n8) *(f32x4*)(to + (GATED ? a.n8 : WIDE) + r) = f32x4{u[r], u[r + 1], u[r + 2], u[r + 3]};
        }
      } else {
        E::put(a, which, row, c, g, u, dh[END == END_BACK ? i : 0][q]);
        if (!GATED) E::put(a, which, row, c + WIDE, u, g, dh[0][q]);
      }
    }
  }
}

// The shares of four columns added in order.
template <class T, int END>
__global__ __launch_bounds__(256) void k_gated_join(const GatedArgs a) {
  const u64 quads = a.n8 / 4, one = (u64)a.m * quads, all = one * a.products, wide = END == END_PLAIN ? a.n8 : 2ull * a.n8;
  for (u64 e = (u64)blockIdx.x * 256 + threadIdx.x; e < all; e += (u64)gridDim.x * 256) {
    const u32 which = (u32)(e / one), row = (u32)(e % one / quads), c = (u32)(e % quads) * 4;
    f32x4 g = {}, u = {};
    const float* p = a.part + ((u64)which * a.shares * a.m + row) * wide + c;
#pragma unroll 4
    for (u32 s = 0; s < a.shares; ++s, p += (u64)a.m * wide) {
      g += *(const f32x4*)p;
      if (END != END_PLAIN) u += *(const f32x4*)(p + a.n8);
    }
    typedef Ends<T, END, 4> E;
    typename E::V d = {};
    if constexpr (END == END_BACK) d = E::dh_at(a, row, c);
    const float gs[4] = {g[0], g[1], g[2], g[3]}, us[4] = {u[0], u[1], u[2], u[3]};
    E::put(a, which, row, c, gs, us, d);
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------------------------------
// How a product's tiles are cut, by what they cost: us of 64 values of k with every unit full, and of a tile's beginning and end.  Measured in bfloat16:
// 2048 tokens, 4096 -> 16384, forward 464 us in tiles of 256 rows, 497 of 128, 501 of 256 with steps half as long and twice the stages (more barriers; loads
// further ahead do not help); 5001 tokens, 1000 -> 2744, 78 and 88; the weights' gradients of 16384 tokens, 768 -> 2048, 376 in 48 tiles of 256 rows, 333 in
// 96 of 128, 165 with the sum of the former in three shares, 121 in five.  Few tokens are bound by the weights' bytes and by the way from memory to LDS and
// back: panels of 64 columns and six stages are more workgroups with more on their way (16 tokens, 512 -> 2048: 8 us for 9.7; 64 tokens, 4096 -> 16384:
// 56 for 63).
struct TileCut { u32 rows, wide, ks, slots; float step, ends; };      // wide: columns of a panel
static const TileCut CUTS[4] = {{256, 128, 64, 256, 1.65f, 9.0f}, {128, 128, 32, 512, 1.85f, 7.0f}, {64, 128, 64, 512, 1.1f, 6.0f}, {64, 64, 64, 256, 0.9f, 4.5f}};

// One product, or two of one shape: the cut of its tiles and the shares of its sum.
struct ProductPlan { u32 cut, shares, per; u64 part; };

static u32 ceil_div(u64 a, u64 b) { return (u32)((a + b - 1) / b); }

// across: the first factor lies across k; along: the second one along it
static ProductPlan product_plan(u64 m, u64 n, u64 k, u32 sources, u32 products, bool gated, bool across, bool along) {
  ProductPlan best{};
  float least = 3e38f;
  const u64 n8 = (n + 7) & ~7ull, wide = gated ? 2 * n8 : n8;
  const float bytes = (float)(k * sources) * (float)(m + wide) * (float)products * 2 / 5.2e6f;      // us that reading both factors once takes
  for (u32 c = 0; c < 4; ++c) {
    const TileCut& cut = CUTS[c];
    if (c >= 2 && across) continue;                                    // (panels of 128 rows)
    if (m <= 64 ? c < 2 && !across : c == 3) continue;                 // (the larger ones are for more rows, the last one for few)
    const u64 tiles = (u64)ceil_div(m, cut.rows) * ceil_div(n, gated ? cut.wide : 2 * cut.wide) * products, steps = (u64)ceil_div(k, cut.ks) * sources;
    for (u32 want = 1; want <= 32; ++want) {
      if (want > 1 && want > steps * cut.ks / 256) break;              // (a share has 256 values of k at least)
      const u32 per = ceil_div(steps, want), shares = per ? ceil_div(steps, per) : 1;
      const u64 part = shares > 1 ? (u64)products * shares * m * wide * 4 : 0;
      if (part > 1ull << 30) break;
      const u64 all = tiles * shares, rounds = all / cut.slots, left = all % cut.slots;
      // (one workgroup alone on a unit that could hold two of 128 rows takes 0.72 of the time; with six stages a step of few workgroups is short)
      const float work = (float)rounds + (left ? (c == 1 && left <= 256 ? 0.72f : 1.0f) : 0.0f);
      const float step = c == 3 && all < 256 ? 0.3f + 0.6f * (float)all / 256 : cut.step;
      float t = work * ((float)per * cut.ks / 64 * step + cut.ends);
      // (rows along k are read in pieces of 128 bytes: that takes more workgroups, or longer; 8 tokens, 4096 -> 16384: 50 us with 512, 69 with 256)
      const float slow = c == 3 ? (along ? 1.15f : 1.05f) : c == 2 && along && all < 512 ? 1.3f : 1.0f;
      if (t < bytes * slow + cut.ends) t = bytes * slow + cut.ends;
      if (shares > 1) t += 2.5f + (float)part * 2 / 5e6f;
      if (t < least) { least = t; best = {c, shares, per, part}; }
    }
  }
  return best;
}

// whether a product's tiles fit into a launch (wide: a tile's columns)
static bool fits(const ProductPlan& p, const GatedArgs& a, u32 wide, u32 products) {
  const TileCut& cut = CUTS[p.cut];
  return (u64)ceil_div(a.m, cut.rows) * ceil_div(a.n, wide * cut.wide / 128) * products * p.shares <= G10_GROUPS_MOST / 2 - 8;
}

template <class T, int LA, int LB, int END>
static int product(GatedArgs a, const ProductPlan& p, u32 products, void* part, hipStream_t s) {
  a.tiles_m = ceil_div(a.m, CUTS[p.cut].rows);
  a.tiles_n = ceil_div(a.n, CUTS[p.cut].wide * (END == END_PLAIN ? 2 : 1));
  a.n8 = (a.n + 7) & ~7u;
  a.products = products; a.per = p.per; a.shares = p.shares; a.part = (float*)part;
  const u64 all = (u64)a.tiles_m * a.tiles_n * products * p.shares;
  const u32 grid = ceil_div(all, 8) * 8;
  if (p.cut == 0) k_gated<T, LA, LB, 2, 4, 4, 64, 2, END><<<grid, 512, 0, s>>>(a);
  else if (p.cut == 1) k_gated<T, LA, LB, 1, 4, 4, 32, 3, END><<<grid, 256, 0, s>>>(a);
  else if constexpr (LA == ALONG) {
    if (p.cut == 2) k_gated<T, LA, LB, 1, 4, 2, 64, 2, END><<<grid, 256, 0, s>>>(a);
    else k_gated<T, LA, LB, 2, 2, 1, 64, 6, END><<<grid, 256, 0, s>>>(a);
  }
  if (p.shares > 1) {
    const u64 groups = ((u64)a.m * (a.n8 / 4) * products + 255) / 256;
    k_gated_join<T, END><<<(u32)(groups < 65536 ? groups : 65536), 256, 0, s>>>(a);
  }
  return G10_OK;
}

// The tiles are loaded in pieces of 16 bytes: rows have to begin and end at multiples of 8 values.  Inputs that do not are laid out so in the
// workspace first, all in one launch, rows ending in zeros.
struct Lay { const void* from; void* to; int64_t fs, ts; u32 rows, columns; };
struct LayArgs { Lay t[4]; u32 count; };
template <class T>
__global__ __launch_bounds__(256) void k_gated_lay(const LayArgs a) {
  typedef T V __attribute__((ext_vector_type(8), aligned(sizeof(T))));
  for (u32 i = 0; i < a.count; ++i) {
    const Lay& t = a.t[i];
    const u32 per = (u32)(t.ts / 8);
    const u64 all = (u64)t.rows * per;
    for (u64 e = (u64)blockIdx.x * 256 + threadIdx.x; e < all; e += (u64)gridDim.x * 256) {
      const u64 row = e / per;
      const u32 c = (u32)(e % per) * 8;
      const T* p = (const T*)t.from + (int64_t)row * t.fs + c;
      V v = {};
      if (c + 8 <= t.columns) {
        v = *(const V*)p;
      } else {
#pragma unroll
        for (int r = 0; r < 8; ++r)
          if (c + r < t.columns) v[r] = p[r];
      }
      *(V*)((T*)t.to + (int64_t)row * t.ts + c) = v;
    }
  }
}

static bool lies_well(const void* p, int64_t stride, u32 columns) {
  return !((uintptr_t)p & 15) && stride % 8 == 0 && columns % 8 == 0 && stride >= (int64_t)columns && stride <= (1 << 22);
}
static bool there(const void* p, int64_t stride, u32 columns) { return p && !((uintptr_t)p & 1) && stride >= (int64_t)columns; }

static int gated_check(const g10_gated_args* g, bool back) {
  if (!g || (g->type != G10_F16 && g->type != G10_BF16) || g->act > G10_ACT_GELU || g->out_in > 1) return G10_EINVAL;
  if (!g->dim || !g->inner || g->dim > 1u << 20 || g->inner > 1u << 20 || g->tokens >= 0x80000000u) return G10_EINVAL;
  const u32 wrow = g->out_in ? g->dim : g->inner;
  if (!there(g->gate, g->gate_stride, wrow) || !there(g->up, g->up_stride, wrow)) return G10_EINVAL;
  if (g->tokens && !there(g->x, g->x_stride, g->dim)) return G10_EINVAL;
  if (!back) return !g->tokens || there(g->h, g->h_stride, g->inner) ? G10_OK : G10_EINVAL;
  if (g->tokens && (!there(g->dh, g->dh_stride, g->inner) || !there(g->dx, g->dx_stride, g->dim))) return G10_EINVAL;
  return there(g->dgate, g->dw_stride, wrow) && there(g->dup, g->dw_stride, wrow) ? G10_OK : G10_EINVAL;
}

// The inputs as the products read them, and where the workspace goes on behind those that are laid out in it.
struct Inputs {
  const void *x, *gate, *up, *dh;
  int64_t xs, ws, dhs;
  LayArgs lay;
  u64 bytes;
};
static Inputs inputs_of(const g10_gated_args* g, bool back, char* room) {
  Inputs in{};
  const u32 rows = g->out_in ? g->inner : g->dim, columns = g->out_in ? g->dim : g->inner;
  auto take = [&](const void* p, int64_t stride, u32 n, u32 width, int64_t& out_stride, bool copy) {
    if (!copy) { out_stride = stride; return p; }
    out_stride = (width + 7) & ~7u;
    void* to = room + in.bytes;
    in.bytes += ((u64)n * out_stride * 2 + 255) & ~255ull;
    in.lay.t[in.lay.count++] = {p, to, stride, out_stride, n, width};
    return (const void*)to;
  };
  const bool weights = !lies_well(g->gate, g->gate_stride, columns) || !lies_well(g->up, g->up_stride, columns) || g->gate_stride != g->up_stride;
  in.x = take(g->x, g->x_stride, g->tokens, g->dim, in.xs, g->tokens && !lies_well(g->x, g->x_stride, g->dim));
  in.gate = take(g->gate, g->gate_stride, rows, columns, in.ws, g->tokens && weights);
  in.up = take(g->up, g->up_stride, rows, columns, in.ws, g->tokens && weights);
  if (back) in.dh = take(g->dh, g->dh_stride, g->tokens, g->inner, in.dhs, g->tokens && !lies_well(g->dh, g->dh_stride, g->inner));
  return in;
}
template <class T>
static void lay_out(const Inputs& in, hipStream_t s) {
  if (!in.lay.count) return;
  u64 most = 0;
  for (u32 i = 0; i < in.lay.count; ++i) {
    const u64 n = (u64)in.lay.t[i].rows * (u64)(in.lay.t[i].ts / 8);
    most = n > most ? n : most;
  }
  const u64 groups = (most + 255) / 256;
  k_gated_lay<T><<<(u32)(groups < 16384 ? groups : 16384), 256, 0, s>>>(in.lay);
}

extern "C" int g10_gated_workspace(const g10_gated_args* g, uint64_t* bytes) {
  if (!bytes) return G10_EINVAL;
  G10_TRY(gated_check(g, false));
  *bytes = g->tokens ? inputs_of(g, false, nullptr).bytes + product_plan(g->tokens, g->inner, g->dim, 1, 1, true, false, g->out_in).part : 0;
  return G10_OK;
}

template <class T>
static int gated_forward(const g10_gated_args* g, char* ws, hipStream_t s) {
  const Inputs in = inputs_of(g, false, ws);
  GatedArgs a{};
  a.a[0] = a.a[1] = in.x; a.b[0] = in.gate; a.b[1] = in.up; a.out[0] = g->h;
  a.as = in.xs; a.bs = in.ws; a.os = g->h_stride;
  a.m = g->tokens; a.n = g->inner; a.k = g->dim; a.sources = 1; a.act = g->act;
  const ProductPlan p = product_plan(a.m, a.n, a.k, 1, 1, true, false, g->out_in);
  if (!fits(p, a, 128, 1)) return G10_EINVAL;
  lay_out<T>(in, s);
  return g->out_in ? product<T, ALONG, ALONG, END_GATED>(a, p, 1, ws + in.bytes, s) : product<T, ALONG, ACROSS, END_GATED>(a, p, 1, ws + in.bytes, s);
}

extern "C" int g10_gated(const g10_gated_args* g, void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  uint64_t n = 0;
  G10_TRY(g10_gated_workspace(g, &n));
  if (n && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < n)) return G10_EINVAL;
  if (!g->tokens) return G10_OK;
  G10_TRY((g->type == G10_F16 ? gated_forward<_Float16> : gated_forward<__bf16>)(g, (char*)workspace, (hipStream_t)hip_stream));
  G10_HIP(hipGetLastError());
  return G10_OK;
}

// Backward: inputs laid out, dg and du, and behind them room for the shares of one product at a time.
struct BackPlan { ProductPlan gated, dx, dw; u64 row, at_dg, at_du, at_part, bytes; };
static BackPlan back_plan(const g10_gated_args* g, u64 laid) {
  BackPlan b{};
  const u32 wm = g->out_in ? g->inner : g->dim, wn = g->out_in ? g->dim : g->inner;
  b.gated = product_plan(g->tokens, g->inner, g->dim, 1, 1, true, false, g->out_in);
  b.dx = product_plan(g->tokens, g->dim, g->inner, 2, 1, false, false, !g->out_in);
  b.dw = product_plan(wm, wn, g->tokens, 1, 2, false, true, false);
  u64 part = b.gated.part > b.dx.part ? b.gated.part : b.dx.part;
  if (b.dw.part > part) part = b.dw.part;
  b.row = (g->inner + 7) & ~7u;
  const u64 one = ((u64)g->tokens * b.row * 2 + 255) & ~255ull;
  b.at_dg = laid;
  b.at_du = laid + one;
  b.at_part = laid + 2 * one;
  b.bytes = b.at_part + part;
  return b;
}

extern "C" int g10_gated_backward_workspace(const g10_gated_args* g, uint64_t* bytes) {
  if (!bytes) return G10_EINVAL;
  G10_TRY(gated_check(g, true));
  *bytes = back_plan(g, inputs_of(g, true, nullptr).bytes).bytes;
  return G10_OK;
}

template <class T>
static int gated_back(const g10_gated_args* g, char* ws, hipStream_t s) {
  const Inputs in = inputs_of(g, true, ws);
  const BackPlan b = back_plan(g, in.bytes);
  void *dg = ws + b.at_dg, *du = ws + b.at_du, *part = ws + b.at_part;
  GatedArgs first{}, second{}, third{};
  first.a[0] = first.a[1] = in.x; first.b[0] = in.gate; first.b[1] = in.up; first.out[0] = dg; first.out[1] = du; first.dh = in.dh;
  first.as = in.xs; first.bs = in.ws; first.os = (int64_t)b.row; first.dhs = in.dhs;
  first.m = g->tokens; first.n = g->inner; first.k = g->dim; first.sources = 1; first.act = g->act;
  second.a[0] = dg; second.a[1] = du; second.b[0] = in.gate; second.b[1] = in.up; second.out[0] = g->dx;
  second.as = (int64_t)b.row; second.bs = in.ws; second.os = g->dx_stride;
  second.m = g->tokens; second.n = g->dim; second.k = g->inner; second.sources = 2;
  third.out[0] = g->dgate; third.out[1] = g->dup; third.os = g->dw_stride;
  third.k = g->tokens; third.sources = 1;
  if (g->out_in) { third.a[0] = dg; third.a[1] = du; third.as = (int64_t)b.row; third.b[0] = third.b[1] = in.x; third.bs = in.xs; third.m = g->inner; third.n = g->dim; }
  else { third.a[0] = third.a[1] = in.x; third.as = in.xs; third.b[0] = dg; third.b[1] = du; third.bs = (int64_t)b.row; third.m = g->dim; third.n = g->inner; }
  if (!fits(b.gated, first, 128, 1) || !fits(b.dx, second, 256, 1) || !fits(b.dw, third, 256, 2)) return G10_EINVAL;      // (before anything is launched)
  if (g->tokens) {
    lay_out<T>(in, s);
    G10_TRY((g->out_in ? product<T, ALONG, ALONG, END_BACK> : product<T, ALONG, ACROSS, END_BACK>)(first, b.gated, 1, part, s));
    G10_TRY((g->out_in ? product<T, ALONG, ACROSS, END_PLAIN> : product<T, ALONG, ALONG, END_PLAIN>)(second, b.dx, 1, part, s));
  }
  return product<T, ACROSS, ACROSS, END_PLAIN>(third, b.dw, 2, part, s);  // (without tokens: zeros)
}

extern "C" int g10_gated_backward(const g10_gated_args* g, void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  uint64_t n = 0;
  G10_TRY(g10_gated_backward_workspace(g, &n));
  if (n && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < n)) return G10_EINVAL;
  G10_TRY((g->type == G10_F16 ? gated_back<_Float16> : gated_back<__bf16>)(g, (char*)workspace, (hipStream_t)hip_stream));
  G10_HIP(hipGetLastError());
  return G10_OK;
}
