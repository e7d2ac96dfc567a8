// The norms of queries and keys with the rotation by position, one pass over both; forward and backward.
//
// Bound by memory: a value is read once and written once (backward: read with its gradient, written once), some 20
// operations between them.  A row (token, head) lies in the registers of a group of 8, 16 or 32 lanes, 8 values to a lane, which
// are four pairs: neighbours lie side by side, halves as 4 values of the lower and the same 4 of the upper half, so that no value
// has to change lanes for its rotation.  Sums are DPP steps inside the group.  A group keeps the cosines and sines of its token for
// several heads (the table's values are four times a 16-bit head's) and has the next four heads on their way while it works.
#include "g10_internal.h"
#include "g10_ops.h"

#include <math.h>

struct RopeArgs {
  const void *x[2], *dy[2], *w[2];
  void *out[2], *dw[2];
  int64_t xs[2][3], dys[2][3], os[2][3];
  u32 heads[2], all_heads;
  u32 seq, dim, rot, n_pos;
  u64 tokens;
  const float* table;
  const void* positions;
  float eps;
  u32 w32, pos64, per[2];           // heads to a task
  u32 chunks[2], all_chunks;        // tasks to a token: of queries, of keys
  float* partial;                   // backward: [workgroups][2][dim]
};

template <class T> __device__ __forceinline__ float to_f(T x) { return (float)x; }

// Eight values as they come from memory: two runs of four.
template <class T>
struct Raw {
  typedef T x4 __attribute__((ext_vector_type(4)));
  x4 a, b;
  __device__ __forceinline__ void load(const T* p, u32 d0, u32 d1) { a = *(const x4*)(p + d0); b = *(const x4*)(p + d1); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = (float)a[i]; v[4 + i] = (float)b[i]; }
  }
};
// (Past the L2, which would write them back when the kernel ends: 32768 tokens of 64 heads of 128 218 -> 210 us, 5001 of 20 heads of 80 in 32 bits,
// forward and backward, 55 -> 48.)
template <class T>
__device__ __forceinline__ void store8(T* p, u32 d0, u32 d1, const float (&v)[8]) {
  typedef T x4 __attribute__((ext_vector_type(4)));
  x4 a, b;
#pragma unroll
  for (int i = 0; i < 4; ++i) { a[i] = (T)v[i]; b[i] = (T)v[4 + i]; }
  __builtin_nontemporal_store(a, (x4*)(p + d0));
  __builtin_nontemporal_store(b, (x4*)(p + d1));
}

template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
// sum over an aligned group of G lanes, in each of them
template <int G>
__device__ __forceinline__ float group_sum(float x) {
  x = dpp_add<0xb1>(x);                                             // lanes 1, 0, 3, 2 of a quad
  x = dpp_add<0x4e>(x);                                             // lanes 2, 3, 0, 1
  x = dpp_add<0x141>(x);                                            // eight lanes mirrored
  if (G >= 16) x = dpp_add<0x140>(x);                               // sixteen lanes mirrored
  if (G >= 32) x += __shfl_xor(x, 16, 64);
  if (G >= 64) x += __shfl_xor(x, 32, 64);
  return x;
}

__device__ __forceinline__ int64_t position(const RopeArgs& a, u64 tok) {
  return a.pos64 ? ((const int64_t*)a.positions)[tok] : (int64_t)((const int*)a.positions)[tok];
}
template <class T>
__device__ __forceinline__ float weight(const RopeArgs& a, int part, u32 d) {
  if (!a.w[part]) return 1.0f;
  return a.w32 ? ((const float*)a.w[part])[d] : to_f(((const T*)a.w[part])[d]);
}

// A lane's four pairs turned by their angles; BACK: by the angles' opposites.
template <bool PAIRS, bool BACK>
__device__ __forceinline__ void turn(float (&v)[8], const float4& c4, const float4& s4) {
  const float c[4] = {c4.x, c4.y, c4.z, c4.w}, s[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int i = PAIRS ? 2 * k : k, j = PAIRS ? 2 * k + 1 : k + 4;
    const float x = v[i], y = v[j], t = BACK ? -s[k] : s[k];
    v[i] = x * c[k] - y * t;
    v[j] = y * c[k] + x * t;
  }
}

// Where a task's rows lie: token, and up to `per` heads of the queries or the keys.
struct Task {
  u64 tok;
  int64_t b, i;
  u32 h0, n;                        // first head, heads (0: no task)
  int part;
};
__device__ __forceinline__ Task task_of(const RopeArgs& a, u64 task, u64 tasks) {
  Task t;
  const bool real = task < tasks;
  t.tok = real ? task / a.all_chunks : 0;
  u32 c = real ? (u32)(task % a.all_chunks) : 0u;
  t.part = c >= a.chunks[0];
  if (t.part) c -= a.chunks[0];
  const u32 per = t.part ? a.per[1] : a.per[0];
  t.h0 = c * per;
  const u32 left = (t.part ? a.heads[1] : a.heads[0]) - t.h0;
  t.n = real ? (left < per ? left : per) : 0u;
  t.b = (int64_t)(t.tok / a.seq);
  t.i = (int64_t)(t.tok % a.seq);
  return t;
}

template <class T, int G, bool PAIRS, bool BACK>
__global__ __launch_bounds__(256) void k_rope(const RopeArgs a) {
  constexpr bool AHEAD = !BACK;                                     // (backward, the registers are worth more: 38 -> 34 us for 16384 tokens of 24 heads of 64)
  const u32 l = lane_id() % G, half = a.rot / 2;
  const bool has = 8 * l < a.dim, in = 8 * l < a.rot;
  const u32 dl = has ? 8 * l : 0u;                                  // (lanes without values read the first ones, and write nothing)
  const u32 d0 = !PAIRS && in ? 4 * l : dl, d1 = !PAIRS && in ? half + 4 * l : dl + 4;
  const u32 at = in ? 4 * l : 0u;                                   // its angles
  const float inv_dim = 1.0f / (float)a.dim;
  float w[2][8], dw[2][8] = {};
#pragma unroll
  for (int part = 0; part < 2; ++part)
#pragma unroll
    for (int k = 0; k < 8; ++k) w[part][k] = has ? weight<T>(a, part, (k < 4 ? d0 + k : d1 + k - 4)) : 0.0f;
  const u32 per = a.per[0] > a.per[1] ? a.per[0] : a.per[1];        // (the same in every lane)
  const u64 tasks = a.tokens * a.all_chunks, step = (u64)gridDim.x * (256 / G);
  // (whole wavefronts stay in the loop: the sums below go over lanes)
  for (u64 first = (u64)blockIdx.x * (256 / G) + wave_id() * (64 / G); first < tasks; first += step) {
    const Task t = task_of(a, first + lane_id() / G, tasks);
    const int p = t.part;
    const int64_t pos = position(a, t.tok);
    const int64_t xh = p ? a.xs[1][2] : a.xs[0][2], yh = p ? a.dys[1][2] : a.dys[0][2], oh = p ? a.os[1][2] : a.os[0][2];
    const T* x = (const T*)(p ? a.x[1] : a.x[0]) + t.b * (p ? a.xs[1][0] : a.xs[0][0]) + t.i * (p ? a.xs[1][1] : a.xs[0][1]) + t.h0 * xh;
    const T* y = nullptr;
    if (BACK) y = (const T*)(p ? a.dy[1] : a.dy[0]) + t.b * (p ? a.dys[1][0] : a.dys[0][0]) + t.i * (p ? a.dys[1][1] : a.dys[0][1]) + t.h0 * yh;
    T* out = (T*)(p ? a.out[1] : a.out[0]) + t.b * (p ? a.os[1][0] : a.os[0][0]) + t.i * (p ? a.os[1][1] : a.os[0][1]) + t.h0 * oh;
    const u32 last = t.n ? t.n - 1 : 0u;                            // (heads past the task's repeat its last)
    Raw<T> rx[4], ry[4];
#pragma unroll
    for (u32 u = 0; u < 4; ++u) {
      const u32 h = u < last ? u : last;
      rx[u].load(x + h * xh, d0, d1);
      if (BACK) ry[u].load(y + h * yh, d0, d1);
    }
    const bool fine = pos >= 0 && pos < (int64_t)a.n_pos;
    const float* tab = a.table + (fine ? pos : 0) * a.rot;
    float4 c = make_float4(1.0f, 1.0f, 1.0f, 1.0f), s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (in) { c = *(const float4*)(tab + at); s = *(const float4*)(tab + half + at); }
    float sw[8], sdw[8] = {};
#pragma unroll
    for (int k = 0; k < 8; ++k) sw[k] = p ? w[1][k] : w[0][k];
    for (u32 q = 0; q < per; q += 4) {
      Raw<T> nx[4], ny[4];
      if (AHEAD && q + 4 < per) {
#pragma unroll
        for (u32 u = 0; u < 4; ++u) {
          const u32 h = q + 4 + u < last ? q + 4 + u : last;
          nx[u].load(x + h * xh, d0, d1);
          if (BACK) ny[u].load(y + h * yh, d0, d1);
        }
      }
#pragma unroll
      for (u32 u = 0; u < 4; ++u) {
        if (q + u >= per) break;                                    // (the same in every lane)
        const bool on = q + u < t.n && has;
        float v[8], sum = 0.0f;
        rx[u].get(v);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += v[k] * v[k];
        sum = group_sum<G>(has ? sum : 0.0f);
        const float r = fine ? 1.0f / sqrtf(sum * inv_dim + a.eps) : __builtin_nanf("");
        if constexpr (!BACK) {
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] = v[k] * r * sw[k];
          turn<PAIRS, false>(v, c, s);
        } else {
          float g[8], dot = 0.0f;
          ry[u].get(g);
          turn<PAIRS, true>(g, c, s);
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            v[k] *= r;
            sdw[k] += on ? g[k] * v[k] : 0.0f;
            g[k] *= sw[k];
            dot += g[k] * v[k];
          }
          dot = group_sum<G>(has ? dot : 0.0f) * inv_dim;
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] = r * (g[k] - v[k] * dot);
        }
        if (on) store8(out + (q + u) * oh, d0, d1, v);
      }
      if (AHEAD) {
#pragma unroll
        for (u32 u = 0; u < 4; ++u) { rx[u] = nx[u]; ry[u] = ny[u]; }
      } else if (q + 4 < per) {
#pragma unroll
        for (u32 u = 0; u < 4; ++u) {
          const u32 h = q + 4 + u < last ? q + 4 + u : last;
          rx[u].load(x + h * xh, d0, d1);
          if (BACK) ry[u].load(y + h * yh, d0, d1);
        }
      }
    }
    if (BACK) {
#pragma unroll
      for (int k = 0; k < 8; ++k) { dw[0][k] += p ? 0.0f : sdw[k]; dw[1][k] += p ? sdw[k] : 0.0f; }
    }
  }
  if constexpr (BACK) {
    if (!a.partial) return;
    __shared__ float sums[4][2][8 * G];
#pragma unroll
    for (int part = 0; part < 2; ++part)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        float t = dw[part][k];
#pragma unroll
        for (int d = G; d < 64; d *= 2) t += __shfl_xor(t, d, 64);
        if (lane_id() < G && has) sums[wave_id()][part][k < 4 ? d0 + k : d1 + k - 4] = t;
      }
    __syncthreads();
    for (u32 e = threadIdx.x; e < 2 * a.dim; e += 256) {
      const u32 part = e / a.dim, d = e % a.dim;
      a.partial[(u64)blockIdx.x * 2 * a.dim + e] = (sums[0][part][d] + sums[1][part][d]) + (sums[2][part][d] + sums[3][part][d]);
    }
  }
}

// Any dimension, alignment and rotation: a wavefront to a row, one value at a time, values lane, lane + 64, ...
template <class T, bool BACK>
__global__ __launch_bounds__(256) void k_rope_any(const RopeArgs a, u32 pairs) {
  const u32 l = lane_id();
  const float inv_dim = 1.0f / (float)a.dim;
  float dw[2][4] = {};
  const u64 rows = a.tokens * a.all_heads;
  for (u64 row = (u64)blockIdx.x * 4 + wave_id(); row < rows; row += (u64)gridDim.x * 4) {
    const u64 tok = row / a.all_heads;
    u32 h = (u32)(row % a.all_heads);
    const int part = h >= a.heads[0];
    if (part) h -= a.heads[0];
    const int64_t pos = position(a, tok), b = (int64_t)(tok / a.seq), i = (int64_t)(tok % a.seq);
    const bool fine = pos >= 0 && pos < (int64_t)a.n_pos;
    const float* t = a.table + (fine ? pos : 0) * a.rot;
    const T* x = (const T*)a.x[part] + b * a.xs[part][0] + i * a.xs[part][1] + h * a.xs[part][2];
    const T* dy = BACK ? (const T*)a.dy[part] + b * a.dys[part][0] + i * a.dys[part][1] + h * a.dys[part][2] : nullptr;
    T* out = (T*)a.out[part] + b * a.os[part][0] + i * a.os[part][1] + h * a.os[part][2];
    float v[4] = {}, e[4] = {}, sum = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const u32 d = l + 64 * k;
      if (d >= a.dim) continue;
      const float own = to_f(x[d]);
      sum += own * own;
      float c = 1.0f, s = 0.0f;                                     // y = v c + (pair's other value) s
      u32 o = d;
      if (d < a.rot) {
        const u32 half = a.rot / 2, at = pairs ? d / 2 : d % half;
        const bool low = pairs ? !(d & 1) : d < half;
        o = pairs ? d ^ 1 : low ? d + half : d - half;
        c = t[at];
        s = low ? -t[half + at] : t[half + at];
      }
      if constexpr (BACK) {
        e[k] = to_f(dy[d]) * c - to_f(dy[o]) * s;                   // the gradient turned back
        v[k] = own;
      } else {
        v[k] = own * weight<T>(a, part, d) * c + to_f(x[o]) * weight<T>(a, part, o) * s;
      }
    }
    sum = group_sum<64>(sum);
    const float r = fine ? 1.0f / sqrtf(sum * inv_dim + a.eps) : __builtin_nanf("");
    float dot = 0.0f;
    if constexpr (BACK) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const u32 d = l + 64 * k;
        if (d >= a.dim) continue;
        const float n = v[k] * r;
        v[k] = n;
        if (part) dw[1][k] += e[k] * n; else dw[0][k] += e[k] * n;
        e[k] *= weight<T>(a, part, d);
        dot += e[k] * n;
      }
      dot = group_sum<64>(dot) * inv_dim;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const u32 d = l + 64 * k;
      if (d < a.dim) out[d] = (T)(BACK ? r * (e[k] - v[k] * dot) : r * v[k]);
    }
  }
  if constexpr (BACK) {
    if (!a.partial) return;
    __shared__ float sums[4][2][256];
#pragma unroll
    for (int part = 0; part < 2; ++part)
#pragma unroll
      for (int k = 0; k < 4; ++k) sums[wave_id()][part][l + 64 * k] = dw[part][k];
    __syncthreads();
    for (u32 e = threadIdx.x; e < 2 * a.dim; e += 256) {
      const u32 part = e / a.dim, d = e % a.dim;
      a.partial[(u64)blockIdx.x * 2 * a.dim + e] = (sums[0][part][d] + sums[1][part][d]) + (sums[2][part][d] + sums[3][part][d]);
    }
  }
}

// Gradients of the weights: the workgroups' sums, 16 values to a workgroup, in one order and 64 bits.
template <class T>
__global__ __launch_bounds__(1024) void k_rope_weights(const RopeArgs a, u32 n) {
  __shared__ double sums[64][16];
  const u32 e = blockIdx.x * 16 + threadIdx.x % 16, w = threadIdx.x / 16;
  double t = 0.0;
  if (e < 2 * a.dim) {
#pragma unroll 8
    for (u32 i = w; i < n; i += 64) t += (double)a.partial[(u64)i * 2 * a.dim + e];
  }
  sums[w][threadIdx.x % 16] = t;
  __syncthreads();
  if (w || e >= 2 * a.dim) return;
  for (u32 i = 1; i < 64; ++i) t += sums[i][threadIdx.x];
  const u32 part = e / a.dim, d = e % a.dim;
  if (!a.dw[part]) return;
  if (a.w32) ((float*)a.dw[part])[d] = (float)t;
  else ((T*)a.dw[part])[d] = (T)(float)t;
}

// ---------------------------------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------------------------------
#define ROPE_GROUPS 1024           // workgroups of a backward pass: 4 on each of 256 compute units

struct RopePlan { u32 grid, lanes; bool any, weights; };

static int rope_args(const g10_rope_args* g, bool back, RopeArgs& a, RopePlan& p) {
  if (!g) return G10_EINVAL;
  if (g->type > G10_BF16 || (g->weight_type != g->type && g->weight_type != G10_F32)) return G10_EINVAL;
  if (!g->dim || g->dim > 256 || g->rot % 2 || g->rot > g->dim) return G10_EINVAL;
  if (!(g->eps >= 0.0f) || (g->flags & ~(G10_ROPE_INTERLEAVED | G10_ROPE_POSITIONS_64))) return G10_EINVAL;
  a = RopeArgs{};
  a.tokens = (u64)g->batch * g->seq;
  const u64 heads = (u64)g->part[0].heads + g->part[1].heads;
  if (heads > 65536 || a.tokens * (heads ? heads : 1) >= (1ull << 40)) return G10_EINVAL;
  const bool some = a.tokens && heads;
  if (some && (!g->positions || !g->n_positions || (g->rot && !g->table))) return G10_EINVAL;
  const u32 e = g->type == G10_F32 ? 4 : 2, step = 16 / e;          // elements of 16 bytes
  p.weights = false;
  p.any = g->dim % 8 || g->rot % 8 || ((uintptr_t)g->table & 15);
  for (int k = 0; k < 2; ++k) {
    const g10_rope_part& s = g->part[k];
    a.heads[k] = s.heads;
    a.x[k] = s.x; a.w[k] = s.weight; a.dy[k] = s.dy; a.out[k] = s.out; a.dw[k] = back ? s.dweight : nullptr;
    for (int i = 0; i < 3; ++i) { a.xs[k][i] = s.x_stride[i]; a.dys[k][i] = s.dy_stride[i]; a.os[k][i] = s.out_stride[i]; }
    if (back && s.dweight && !s.weight) return G10_EINVAL;
    if (back && s.dweight) p.weights = true;
    if (!a.tokens || !s.heads) continue;
    if (!s.x || !s.out || (back && !s.dy)) return G10_EINVAL;
    for (const void* q : {s.x, (const void*)s.out, back ? s.dy : nullptr}) {
      if ((uintptr_t)q % e) return G10_EINVAL;
      if ((uintptr_t)q & 15) p.any = true;
    }
    for (int i = 0; i < 3; ++i)
      if (s.x_stride[i] % step || s.out_stride[i] % step || (back && s.dy_stride[i] % step)) p.any = true;
  }
  a.all_heads = (u32)heads;
  a.seq = g->seq; a.dim = g->dim; a.rot = g->rot; a.n_pos = g->n_positions;
  a.table = g->table; a.positions = g->positions; a.eps = g->eps;
  a.w32 = g->weight_type == G10_F32; a.pos64 = (g->flags & G10_ROPE_POSITIONS_64) != 0;
  p.lanes = g->dim <= 64 ? 8 : g->dim <= 128 ? 16 : 32;
  // A task takes 4, 8 or 12 heads where that still fills the chip, as many as leave the fewest places empty; else one: with few tokens a
  // row's way from memory and back is all there is.
  const u64 rows = a.tokens * heads;
  for (int k = 0; k < 2; ++k) {
    a.per[k] = 1;
    if (rows / 8 * p.lanes >= 256ull * 8 * 64) {
      u32 best = ~0u;
      for (const u32 per : {8u, 12u, 4u}) {
        const u32 places = (a.heads[k] + per - 1) / per * per;
        if (places < best) { best = places; a.per[k] = per; }
      }
    }
    a.chunks[k] = some ? (a.heads[k] + a.per[k] - 1) / a.per[k] : 0;
  }
  a.all_chunks = a.chunks[0] + a.chunks[1];
  const u64 groups = p.any ? (rows + 3) / 4 : (a.tokens * a.all_chunks + 256 / p.lanes - 1) / (256 / p.lanes);
  p.grid = (u32)(back ? (groups < ROPE_GROUPS ? groups : ROPE_GROUPS) : (groups < G10_GROUPS_MOST ? groups : G10_GROUPS_MOST));
  return G10_OK;
}

template <class T, bool BACK>
static void rope_launch(const RopeArgs& a, const RopePlan& p, bool pairs, hipStream_t s) {
  if (p.any) { k_rope_any<T, BACK><<<p.grid, 256, 0, s>>>(a, pairs); return; }
  if (pairs) {
    if (p.lanes == 8) k_rope<T, 8, true, BACK><<<p.grid, 256, 0, s>>>(a);
    else if (p.lanes == 16) k_rope<T, 16, true, BACK><<<p.grid, 256, 0, s>>>(a);
    else k_rope<T, 32, true, BACK><<<p.grid, 256, 0, s>>>(a);
  } else {
    if (p.lanes == 8) k_rope<T, 8, false, BACK><<<p.grid, 256, 0, s>>>(a);
    else if (p.lanes == 16) k_rope<T, 16, false, BACK><<<p.grid, 256, 0, s>>>(a);
    else k_rope<T, 32, false, BACK><<<p.grid, 256, 0, s>>>(a);
  }
}

extern "C" int g10_norm_rope(const g10_rope_args* g, void* hip_stream) {
  RopeArgs a; RopePlan p;
  G10_TRY(rope_args(g, false, a, p));
  if (!p.grid) return G10_OK;
  const bool pairs = g->flags & G10_ROPE_INTERLEAVED;
  if (g->type == G10_F32) rope_launch<float, false>(a, p, pairs, (hipStream_t)hip_stream);
  else if (g->type == G10_F16) rope_launch<_Float16, false>(a, p, pairs, (hipStream_t)hip_stream);
  else rope_launch<__bf16, false>(a, p, pairs, (hipStream_t)hip_stream);
  G10_HIP(hipGetLastError());
  return G10_OK;
}

extern "C" int g10_norm_rope_workspace(const g10_rope_args* g, uint64_t* bytes) {
  if (!bytes) return G10_EINVAL;
  RopeArgs a; RopePlan p;
  G10_TRY(rope_args(g, true, a, p));
  *bytes = p.weights ? (uint64_t)p.grid * 2 * a.dim * 4 : 0;
  return G10_OK;
}

extern "C" int g10_norm_rope_backward(const g10_rope_args* g, void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  RopeArgs a; RopePlan p;
  G10_TRY(rope_args(g, true, a, p));
  hipStream_t s = (hipStream_t)hip_stream;
  if (p.weights && p.grid) {
    if (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < (uint64_t)p.grid * 2 * a.dim * 4) return G10_EINVAL;
    a.partial = (float*)workspace;
  }
  const bool pairs = g->flags & G10_ROPE_INTERLEAVED;
  if (p.grid) {
    if (g->type == G10_F32) rope_launch<float, true>(a, p, pairs, s);
    else if (g->type == G10_F16) rope_launch<_Float16, true>(a, p, pairs, s);
    else rope_launch<__bf16, true>(a, p, pairs, s);
  }
  if (p.weights) {                                                   // (without tokens: zeros)
    const u32 grid = (2 * a.dim + 15) / 16;
    if (g->type == G10_F32) k_rope_weights<float><<<grid, 1024, 0, s>>>(a, p.grid);
    else if (g->type == G10_F16) k_rope_weights<_Float16><<<grid, 1024, 0, s>>>(a, p.grid);
    else k_rope_weights<__bf16><<<grid, 1024, 0, s>>>(a, p.grid);
  }
  G10_HIP(hipGetLastError());
  return G10_OK;
}
