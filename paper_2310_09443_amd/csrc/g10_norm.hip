// Norms of rows, centred or not, forward and backward.
//
// Bound by memory: forward a value is read and written once, backward it is read with its gradient and written once.  A row lies in the
// registers of a part of a wavefront (up to 256 values), of a wavefront (up to 1024) or of a workgroup, 8 values to a lane and step, so
// that the statistics are taken from the values themselves: the mean first, then the squares of what is left (the squares' mean less the
// mean's square would lose what a large mean leaves over).  Backward the statistics are worked out again from x, which has to be read in
// any case.  The gradients of weight and bias are sums over rows: a lane keeps its columns' over all rows that its group takes, and the
// groups' sums are joined in one order and 64 bits by a second kernel.  Backward a row's four arrays of values do not fit the 128 registers that 1024 threads have
// from 8193 values on (36 to 96 bytes of scratch a lane in whole rows of up to 16384 values in bf16 and fp32, 0.15 to 1.4 KB above; forward from 16385 in
// rows that are no multiple of 8, from 32769 in all): 8192 rows of 12288 in bf16 62 us forward and 131 backward, 5033 of 20000 79 and 306.
#include "g10_internal.h"
#include "g10_ops.h"

#include <math.h>

struct NormArgs {
  const void *x, *dy, *w, *b;
  void *out, *dw, *db;
  int64_t xs, dys, os;
  u32 rows, dim, w32, center;
  float eps;
  float* partial;                  // backward: [groups][2][dim]
};


template <int CTRL>
__device__ __forceinline__ float dpp_plus(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
// sum over an aligned group of L lanes, in each of them
template <int L>
__device__ __forceinline__ float lanes_sum(float x) {
  x = dpp_plus<0xb1>(x);                                            // lanes 1, 0, 3, 2 of a quad
  x = dpp_plus<0x4e>(x);                                            // lanes 2, 3, 0, 1
  x = dpp_plus<0x141>(x);                                           // eight lanes mirrored
  if (L >= 16) x = dpp_plus<0x140>(x);                              // sixteen lanes mirrored
  if (L >= 32) x += __shfl_xor(x, 16, 64);
  if (L >= 64) x += __shfl_xor(x, 32, 64);
  return x;
}
// Sums over the L lanes or W wavefronts of a row, in each lane.  `room`: LDS of the call's own (the next call takes another one, so that
// one barrier a call is enough).
template <int W, int L, int N>
__device__ __forceinline__ void row_sums(float (&x)[N], float* room) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = lanes_sum<L>(x[i]);
  if constexpr (W > 1) {
    if (lane_id() == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) room[i * W + wave_id()] = x[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = room[i * W];
#pragma unroll
      for (int w = 1; w < W; ++w) x[i] += room[i * W + w];
    }
  }
}

// Eight values side by side, at any address of a value: accesses to memory need not be aligned, only a row's last eight may be fewer.
template <class T> struct Eight { typedef T x8 __attribute__((ext_vector_type(8), aligned(sizeof(T)))); };

// WHOLE: rows of a multiple of 8 values.
template <class T, bool WHOLE>
__device__ __forceinline__ void get8(const T* p, u32 d, u32 dim, float (&v)[8]) {
  if (WHOLE || d + 8 <= dim) {
    typedef typename Eight<T>::x8 x8;
    const x8 r = *(const x8*)(p + d);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = (float)r[k];
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = d + k < dim ? (float)p[d + k] : 0.0f;
  }
}
template <class T, bool WHOLE>
__device__ __forceinline__ void put8(T* p, u32 d, u32 dim, const float (&v)[8]) {
  if (WHOLE || d + 8 <= dim) {
    typedef typename Eight<T>::x8 x8;
    x8 r;
#pragma unroll
    for (int k = 0; k < 8; ++k) r[k] = (T)v[k];
    __builtin_nontemporal_store(r, (x8*)(p + d));                      // (past the L2)
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (d + k < dim) p[d + k] = (T)v[k];
  }
}
template <class T, bool WHOLE>
__device__ __forceinline__ void weights8(const void* w, u32 w32, u32 d, u32 dim, float none, float (&v)[8]) {
  if (!w) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = none;
  } else if (w32) {
    get8<float, WHOLE>((const float*)w, d, dim, v);
  } else {
    get8<T, WHOLE>((const T*)w, d, dim, v);
  }
}

// W wavefronts to a row, NV steps of 8 values a lane; a workgroup holds one row (W = 4, 8, 16) or four wavefronts' (W = 1), of which each has
// 64 / L: rows of up to 256 values lie side by side in a wavefront (100000 x 128 in bf16: 7.3 us forward and 19 backward, with a wavefront to
// each row 24 and 47; 14021 x 69: 4.1 and 10.6 for 7.1 and 18.5).
template <class T, int W, int L, int NV, bool WHOLE, bool BACK>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void k_norm(const NormArgs a) {
  constexpr u32 BESIDE = 64 / L, ROWS = W == 1 ? 4 * BESIDE : 1, LANES = L * W;
  __shared__ float room[4][2 * W];
  const u32 l = W == 1 ? lane_id() % L : threadIdx.x, mine = L < 64 ? lane_id() / L : 0;
  const u64 first = (u64)blockIdx.x * ROWS + (W == 1 ? wave_id() * BESIDE : 0), step = (u64)gridDim.x * ROWS;      // (the same in all lanes)
  auto row_of = [&](u64 base) { return L == 64 || base + mine < a.rows ? base + mine : (u64)a.rows - 1; };
  const float inv = 1.0f / (float)a.dim;
  float dw[BACK ? NV : 1][8] = {}, db[BACK ? NV : 1][8] = {};
  u32 turn = 0;
  // backward with a few steps a row, the next row is on its way while this one is worked on
  constexpr bool AHEAD = BACK && WHOLE && NV <= 2;
  typedef typename Eight<T>::x8 x8;
  x8 nx[AHEAD ? NV : 1], ny[AHEAD ? NV : 1];
  auto fetch = [&](u64 row) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const u32 d = (i * LANES + l) * 8, at = d < a.dim ? d : 0;
      nx[AHEAD ? i : 0] = *(const x8*)((const T*)a.x + (int64_t)row * a.xs + at);
      ny[AHEAD ? i : 0] = *(const x8*)((const T*)a.dy + (int64_t)row * a.dys + at);
    }
  };
  if constexpr (AHEAD) {
    if (first < a.rows) fetch(row_of(first));
  }
  // A lane's columns are the same in every row: with a few steps their weights stay in registers (16384 rows of 768 forward 11.5 -> 9.8 us; not where
  // a workgroup has one row: 32768 of 4096 89 -> 96, fewer wavefronts fit).
  constexpr bool KEPT = NV <= 2 && (BACK || W == 1);
  float kw[KEPT ? NV : 1][8], kb[KEPT && !BACK ? NV : 1][8];
  if constexpr (KEPT) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const u32 d = (i * LANES + l) * 8;
      if (d >= a.dim) continue;
      weights8<T, WHOLE>(a.w, a.w32, d, a.dim, 1.0f, kw[i]);
      if constexpr (!BACK) weights8<T, WHOLE>(a.b, a.w32, d, a.dim, 0.0f, kb[i]);
    }
  }
  auto weights = [&](int i, u32 d, float (&w)[8]) {
    if constexpr (KEPT) {
#pragma unroll
      for (int k = 0; k < 8; ++k) w[k] = kw[i][k];
    } else {
      weights8<T, WHOLE>(a.w, a.w32, d, a.dim, 1.0f, w);
    }
  };
  for (u64 base = first; base < a.rows; base += step) {
    const u64 row = row_of(base);
    const bool on = L == 64 || base + mine < a.rows;                // (lanes of rows past the last one repeat it, and neither write nor add)
    const T* x = (const T*)a.x + (int64_t)row * a.xs;
    const T* y = BACK ? (const T*)a.dy + (int64_t)row * a.dys : nullptr;
    T* out = (T*)a.out + (int64_t)row * a.os;
    float v[NV][8], g[BACK ? NV : 1][8];
    if constexpr (AHEAD) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const bool in = (i * LANES + l) * 8 < a.dim;
#pragma unroll
        for (int k = 0; k < 8; ++k) { v[i][k] = in ? (float)nx[i][k] : 0.0f; g[i][k] = in ? (float)ny[i][k] : 0.0f; }
      }
      fetch(base + step < a.rows ? row_of(base + step) : row);
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const u32 d = (i * LANES + l) * 8;
        if (d < a.dim) {
          get8<T, WHOLE>(x, d, a.dim, v[i]);
          if constexpr (BACK) get8<T, WHOLE>(y, d, a.dim, g[i]);
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) { v[i][k] = 0.0f; if constexpr (BACK) g[i][k] = 0.0f; }
        }
      }
    }
    float mean = 0.0f;
    if (a.center) {
      float s[1] = {};
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) s[0] += v[i][k];
      row_sums<W, L>(s, room[turn]);
      turn = (turn + 1) & 3;
      mean = s[0] * inv;
    }
    float s[1] = {};
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const u32 d = (i * LANES + l) * 8 + k;
        v[i][k] = d < a.dim ? v[i][k] - mean : 0.0f;
        s[0] += v[i][k] * v[i][k];
      }
    row_sums<W, L>(s, room[turn]);
    turn = (turn + 1) & 3;
    const float r = 1.0f / sqrtf(s[0] * inv + a.eps);
    if constexpr (!BACK) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const u32 d = (i * LANES + l) * 8;
        if (d >= a.dim) continue;
        float w[8], b[8];
        weights(i, d, w);
        if constexpr (!KEPT) weights8<T, WHOLE>(a.b, a.w32, d, a.dim, 0.0f, b);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[i][k] = v[i][k] * r * w[k] + (KEPT ? kb[KEPT ? i : 0][k] : b[k]);
        if (on) put8<T, WHOLE>(out, d, a.dim, v[i]);
      }
    } else {
      float t[2] = {};                                              // sums of u n and of u
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const u32 d = (i * LANES + l) * 8;
        if (d >= a.dim) continue;
        float w[8];
        weights(i, d, w);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          v[i][k] *= r;
          dw[i][k] += on ? g[i][k] * v[i][k] : 0.0f;
          db[i][k] += on ? g[i][k] : 0.0f;
          g[i][k] *= w[k];
          t[0] += g[i][k] * v[i][k];
          t[1] += g[i][k];
        }
      }
      row_sums<W, L>(t, room[turn]);
      turn = (turn + 1) & 3;
      const float dot = t[0] * inv, off = a.center ? t[1] * inv : 0.0f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const u32 d = (i * LANES + l) * 8;
        if (d >= a.dim) continue;
#pragma unroll
        for (int k = 0; k < 8; ++k) g[i][k] = r * (g[i][k] - v[i][k] * dot - off);
        if (on) put8<T, WHOLE>(out, d, a.dim, g[i]);
      }
    }
  }
  if constexpr (BACK) {
    if (!a.partial) return;
    float* to = a.partial + (u64)blockIdx.x * 2 * a.dim;
    if constexpr (W == 1) {                                         // the four wavefronts' sums, step by step
      constexpr u32 WIDE = 8 * L;
      __shared__ float sums[2][4][WIDE];
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          float w = dw[i][k], b = db[i][k];
#pragma unroll
          for (int d = L; d < 64; d *= 2) { w += __shfl_xor(w, d, 64); b += __shfl_xor(b, d, 64); }
          if (mine == 0) { sums[0][wave_id()][l * 8 + k] = w; sums[1][wave_id()][l * 8 + k] = b; }
        }
        __syncthreads();
        for (u32 e = threadIdx.x; e < 2 * WIDE; e += 256) {
          const u32 which = e / WIDE, c = e % WIDE, d = i * WIDE + c;
          if (d < a.dim) to[which * a.dim + d] = (sums[which][0][c] + sums[which][1][c]) + (sums[which][2][c] + sums[which][3][c]);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const u32 d = (i * LANES + l) * 8 + k;
          if (d < a.dim) { to[d] = dw[i][k]; to[a.dim + d] = db[i][k]; }
        }
    }
  }
}

// The groups' sums of 16 columns to a workgroup, in one order and 64 bits.
template <class T>
__global__ __launch_bounds__(1024) void k_norm_weights(const NormArgs a, u32 groups) {
  __shared__ double sums[64][17];
  const u32 e = blockIdx.x * 16 + threadIdx.x % 16, w = threadIdx.x / 16;
  const u64 all = 2ull * a.dim;
  double t = 0.0;
  if (e < all) {
#pragma unroll 8
    for (u32 i = w; i < groups; i += 64) t += (double)a.partial[i * all + e];
  }
  sums[w][threadIdx.x % 16] = t;
  __syncthreads();
  if (w || e >= all) return;
  for (u32 i = 1; i < 64; ++i) t += sums[i][threadIdx.x];
  const u32 d = e % a.dim;
  void* to = e / a.dim ? a.db : a.dw;
  if (!to) return;
  if (a.w32) ((float*)to)[d] = (float)t;
  else ((T*)to)[d] = (T)(float)t;
}

// ---------------------------------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------------------------------
struct NormPlan { u32 grid, waves, lanes, steps; bool whole, weights; };

static int norm_args(const g10_norm_args* g, bool back, NormArgs& a, NormPlan& p) {
  if (!g) return G10_EINVAL;
  if (g->type > G10_BF16 || (g->weight_type != g->type && g->weight_type != G10_F32) || g->center > 1) return G10_EINVAL;
  if (!g->dim || g->dim > 65536 || g->rows >= 0x80000000u || !(g->eps >= 0.0f) || isinf(g->eps)) return G10_EINVAL;
  const u32 e = g->type == G10_F32 ? 4 : 2, we = g->weight_type == G10_F32 ? 4 : 2;
  if (g->rows && (!g->x || !g->out || (back && !g->dy))) return G10_EINVAL;
  if (back && g->dweight && !g->weight) return G10_EINVAL;
  for (const void* q : {g->x, (const void*)g->out, back ? g->dy : nullptr})
    if ((uintptr_t)q % e) return G10_EINVAL;
  const void* ws[4] = {g->weight, g->bias, back ? g->dweight : nullptr, back ? g->dbias : nullptr};
  for (const void* q : ws)
    if ((uintptr_t)q % we) return G10_EINVAL;
  a = NormArgs{};
  a.x = g->x; a.dy = g->dy; a.w = g->weight; a.b = g->bias; a.out = g->out;
  a.dw = back ? g->dweight : nullptr; a.db = back ? g->dbias : nullptr;
  a.xs = g->x_stride; a.dys = g->dy_stride; a.os = g->out_stride;
  a.rows = g->rows; a.dim = g->dim; a.w32 = g->weight_type == G10_F32; a.center = g->center; a.eps = g->eps;
  p.weights = a.dw || a.db;
  p.whole = g->dim % 8 == 0;
  const u32 lanes = (g->dim + 7) / 8;
  p.waves = lanes <= 128 ? 1 : lanes <= 512 ? 4 : lanes <= 1024 ? 8 : 16;
  p.lanes = lanes <= 8 ? 8 : lanes <= 16 ? 16 : lanes <= 32 ? 32 : 64;
  p.steps = (lanes + 64 * p.waves - 1) / (64 * p.waves);
  if (p.steps == 3) p.steps = 4;
  if (p.steps > 4) p.steps = 8;
  const u32 rows_each = p.waves == 1 ? 4 * (64 / p.lanes) : 1;
  const u64 groups = ((u64)a.rows + rows_each - 1) / rows_each;
  const u32 most = back ? (p.waves == 16 ? 256u : 512u) : 1u << 16;
  p.grid = (u32)(groups < most ? groups : most);
  return G10_OK;
}

template <class T, bool WHOLE, bool BACK>
static void norm_launch(const NormArgs& a, const NormPlan& p, hipStream_t s) {
  auto go = [&](auto w, auto nv) {
    constexpr int W = decltype(w)::value, NV = decltype(nv)::value;
    k_norm<T, W, 64, NV, WHOLE, BACK><<<p.grid, W == 1 ? 256 : 64 * W, 0, s>>>(a);
  };
  using std::integral_constant;
  auto pick = [&](auto w) {
    if (p.steps == 2) go(w, integral_constant<int, 2>{});
    else if (p.steps == 4) go(w, integral_constant<int, 4>{});
    else go(w, integral_constant<int, 8>{});
  };
  if (p.lanes == 8) k_norm<T, 1, 8, 1, WHOLE, BACK><<<p.grid, 256, 0, s>>>(a);
  else if (p.lanes == 16) k_norm<T, 1, 16, 1, WHOLE, BACK><<<p.grid, 256, 0, s>>>(a);
  else if (p.lanes == 32) k_norm<T, 1, 32, 1, WHOLE, BACK><<<p.grid, 256, 0, s>>>(a);
  else if (p.waves == 1) { if (p.steps == 1) go(integral_constant<int, 1>{}, integral_constant<int, 1>{}); else go(integral_constant<int, 1>{}, integral_constant<int, 2>{}); }
  else if (p.waves == 4) { if (p.steps == 1) go(integral_constant<int, 4>{}, integral_constant<int, 1>{}); else go(integral_constant<int, 4>{}, integral_constant<int, 2>{}); }
  else if (p.waves == 8) go(integral_constant<int, 8>{}, integral_constant<int, 2>{});
  else pick(integral_constant<int, 16>{});
}

template <bool BACK>
static void norm_typed(const g10_norm_args* g, const NormArgs& a, const NormPlan& p, hipStream_t s) {
  if (g->type == G10_F32) { if (p.whole) norm_launch<float, true, BACK>(a, p, s); else norm_launch<float, false, BACK>(a, p, s); }
  else if (g->type == G10_F16) { if (p.whole) norm_launch<_Float16, true, BACK>(a, p, s); else norm_launch<_Float16, false, BACK>(a, p, s); }
  else { if (p.whole) norm_launch<__bf16, true, BACK>(a, p, s); else norm_launch<__bf16, false, BACK>(a, p, s); }
}

extern "C" int g10_norm(const g10_norm_args* g, void* hip_stream) {
  NormArgs a; NormPlan p;
  G10_TRY(norm_args(g, false, a, p));
  if (!p.grid) return G10_OK;
  norm_typed<false>(g, a, p, (hipStream_t)hip_stream);
  G10_HIP(hipGetLastError());
  return G10_OK;
}

extern "C" int g10_norm_backward_workspace(const g10_norm_args* g, uint64_t* bytes) {
  if (!bytes) return G10_EINVAL;
  NormArgs a; NormPlan p;
  G10_TRY(norm_args(g, true, a, p));
  *bytes = p.weights ? (uint64_t)p.grid * 2 * a.dim * 4 : 0;
  return G10_OK;
}

extern "C" int g10_norm_backward(const g10_norm_args* g, void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  NormArgs a; NormPlan p;
  G10_TRY(norm_args(g, true, a, p));
  hipStream_t s = (hipStream_t)hip_stream;
  if (p.weights && p.grid) {
    if (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < (uint64_t)p.grid * 2 * a.dim * 4) return G10_EINVAL;
    a.partial = (float*)workspace;
  }
  if (p.grid) norm_typed<true>(g, a, p, s);
  if (p.weights) {                                                   // (without rows: zeros)
    const u32 grid = (2 * a.dim + 15) / 16;
    if (g->type == G10_F32) k_norm_weights<float><<<grid, 1024, 0, s>>>(a, p.grid);
    else if (g->type == G10_F16) k_norm_weights<_Float16><<<grid, 1024, 0, s>>>(a, p.grid);
    else k_norm_weights<__bf16><<<grid, 1024, 0, s>>>(a, p.grid);
  }
  G10_HIP(hipGetLastError());
  return G10_OK;
}
