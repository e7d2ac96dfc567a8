// The norms of queries and keys with the rotation by position, one pass over both; forward and backward.
//
// Bound by memory: a value is read once and written once (backward: read with its gradient, written once), some 20
// operations between them.  A row (token, head) lies in the registers of a group of 8, 16 or 32 lanes, 8 values to a lane; its sums
// are DPP steps inside the group, pairs of the rotation are values of one lane or of two lanes of the group.  A group keeps the
// cosines and sines of its token for several heads (the table's values are four times a 16-bit head's).
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
  u32 w32, pos64, chunks, per;      // per heads to a task, chunks tasks to a token
  float* partial;                   // backward: [workgroups][2][dim]
};

template <class T> __device__ __forceinline__ float to_f(T x) { return (float)x; }

template <class T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
    const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
    typedef T x8 __attribute__((ext_vector_type(8)));
    const x8 a = *(const x8*)p;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)a[i];
  }
}
template <class T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
    *(float4*)p = make_float4(v[0], v[1], v[2], v[3]);
    *(float4*)(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    typedef T x8 __attribute__((ext_vector_type(8)));
    x8 a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = (T)v[i];
    *(x8*)p = a;
  }
}

// sum over an aligned group of G lanes, in each of them
template <int G>
__device__ __forceinline__ float group_sum(float x) {
#pragma unroll
  for (int d = 1; d < G; d *= 2) x += __shfl_xor(x, d, 64);
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

// The cosines and sines that a lane's values 8 lane .. + 7 meet.  Values past `rot` meet 1 and 0.
template <bool PAIRS>
__device__ __forceinline__ void angles(const RopeArgs& a, int64_t pos, u32 d0, float (&c)[8], float (&s)[8]) {
  const bool in = d0 < a.rot;
  const float* t = a.table + pos * a.rot;
  if constexpr (PAIRS) {
    const u32 i = in ? d0 / 2 : 0u;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float x = in ? t[i + k] : 1.0f, y = in ? t[a.rot / 2 + i + k] : 0.0f;
      c[2 * k] = c[2 * k + 1] = x; s[2 * k] = s[2 * k + 1] = y;
    }
  } else {
    const u32 i = in ? d0 % (a.rot / 2) : 0u;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      c[k] = in ? t[i + k] : 1.0f;
      s[k] = in ? t[a.rot / 2 + i + k] : 0.0f;
    }
  }
}
// Values turned by their angles; `back`: by the angles' opposites.  Lane l's values are 8 (l % G) .. + 7 of the row.
template <bool PAIRS, bool BACK>
__device__ __forceinline__ void turn(const RopeArgs& a, u32 d0, float (&v)[8], const float (&c)[8], const float (&s)[8]) {
  if constexpr (PAIRS) {
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
      const float x = v[k], y = v[k + 1], t = BACK ? -s[k] : s[k];
      v[k] = x * c[k] - y * t;
      v[k + 1] = y * c[k] + x * t;
    }
  } else {
    const u32 half = a.rot / 16;                                    // lanes between the two values of a pair
    const bool low = d0 < a.rot / 2, in = d0 < a.rot;
    const int other = (int)lane_id() + (in ? (low ? (int)half : -(int)half) : 0);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float y = __shfl(v[k], other, 64);
      const float t = low != BACK ? -s[k] : s[k];
      v[k] = v[k] * c[k] + y * t;
    }
  }
}

template <class T, int G, bool PAIRS, bool BACK>
__global__ __launch_bounds__(256) void k_rope(const RopeArgs a) {
  const u32 l = lane_id() % G, d0 = 8 * l;
  const bool has = d0 < a.dim;
  const float inv_dim = 1.0f / (float)a.dim;
  float w[2][8], dw[2][8] = {};
#pragma unroll
  for (int part = 0; part < 2; ++part)
#pragma unroll
    for (int k = 0; k < 8; ++k) w[part][k] = has ? weight<T>(a, part, d0 + k) : 0.0f;
  const u64 tasks = a.tokens * a.chunks, step = (u64)gridDim.x * (256 / G);
  // (whole wavefronts stay in the loop: the sums below go over lanes)
  for (u64 first = (u64)blockIdx.x * (256 / G) + wave_id() * (64 / G); first < tasks; first += step) {
    const u64 task = first + lane_id() / G;
    const bool real = task < tasks;
    const u64 tok = real ? task / a.chunks : 0;
    const u32 h0 = real ? (u32)(task % a.chunks) * a.per : 0u;
    const u32 h1 = real ? (h0 + a.per < a.all_heads ? h0 + a.per : a.all_heads) : 0u;
    const int64_t pos = position(a, tok), b = (int64_t)(tok / a.seq), i = (int64_t)(tok % a.seq);
    const bool fine = pos >= 0 && pos < (int64_t)a.n_pos;
    float c[8], s[8];
    angles<PAIRS>(a, fine ? pos : 0, d0, c, s);
    for (u32 q = 0; q < a.per; q += 4) {
      float x[4][8], dy[4][8];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const u32 h = h0 + q + u;
        const bool on = h < h1 && q + u < a.per && has;
        const int part = h >= a.heads[0];
        const u32 hh = part ? h - a.heads[0] : h;
#pragma unroll
        for (int k = 0; k < 8; ++k) { x[u][k] = 0.0f; if (BACK) dy[u][k] = 0.0f; }
        if (on) {
          load8((const T*)a.x[part] + b * a.xs[part][0] + i * a.xs[part][1] + hh * a.xs[part][2] + d0, x[u]);
          if (BACK) load8((const T*)a.dy[part] + b * a.dys[part][0] + i * a.dys[part][1] + hh * a.dys[part][2] + d0, dy[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const u32 h = h0 + q + u;
        if (q + u >= a.per) break;                                  // (the same in every lane)
        const bool on = h < h1 && has;
        const int part = h >= a.heads[0];
        const u32 hh = part ? h - a.heads[0] : h;
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += x[u][k] * x[u][k];
        sum = group_sum<G>(sum);
        const float r = fine ? 1.0f / sqrtf(sum * inv_dim + a.eps) : __builtin_nanf("");
        float v[8];
        if constexpr (!BACK) {
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] = x[u][k] * r * (part ? w[1][k] : w[0][k]);
          turn<PAIRS, false>(a, d0, v, c, s);
        } else {
          float dot = 0.0f;
          turn<PAIRS, true>(a, d0, dy[u], c, s);
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float n = x[u][k] * r, g = dy[u][k];
            x[u][k] = n;
            v[k] = g * (part ? w[1][k] : w[0][k]);
            dot += v[k] * n;
            if (on) { if (part) dw[1][k] += g * n; else dw[0][k] += g * n; }
          }
          dot = group_sum<G>(dot) * inv_dim;
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] = r * (v[k] - x[u][k] * dot);
        }
        if (on) store8((T*)a.out[part] + b * a.os[part][0] + i * a.os[part][1] + hh * a.os[part][2] + d0, v);
      }
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
        if (lane_id() < G) sums[wave_id()][part][d0 + k] = t;
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

// Gradients of the weights: the workgroups' sums, 32 values to a workgroup, in one order and 64 bits.
template <class T>
__global__ __launch_bounds__(256) void k_rope_weights(const RopeArgs a, u32 n) {
  __shared__ double sums[8][32];
  const u32 e = blockIdx.x * 32 + threadIdx.x % 32, w = threadIdx.x / 32;
  double t = 0.0;
  if (e < 2 * a.dim)
    for (u32 i = w; i < n; i += 8) t += (double)a.partial[(u64)i * 2 * a.dim + e];
  sums[w][threadIdx.x % 32] = t;
  __syncthreads();
  if (w || e >= 2 * a.dim) return;
  for (u32 i = 1; i < 8; ++i) t += sums[i][threadIdx.x];
  const u32 part = e / a.dim, d = e % a.dim;
  if (!a.dw[part]) return;
  if (a.w32) ((float*)a.dw[part])[d] = (float)t;
  else ((T*)a.dw[part])[d] = (T)(float)t;
}

// ---------------------------------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------------------------------
#define ROPE_GROUPS 2048           // workgroups of a backward pass: 8 on each of 256 compute units

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
  const bool pairs = g->flags & G10_ROPE_INTERLEAVED;
  const u32 e = g->type == G10_F32 ? 4 : 2, step = 16 / e;          // elements of 16 bytes
  p.weights = false;
  p.any = g->dim % 8 || (pairs ? g->rot % 8 : g->rot % 16) || ((uintptr_t)g->table & 15);
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
  // A task takes 8 heads where that still fills the chip, else one: with few tokens a row's way from memory and back is all there is.
  const u64 rows = a.tokens * heads;
  a.per = rows / 8 * p.lanes >= 256ull * 8 * 64 ? 8 : 1;
  a.chunks = some ? (u32)((heads + a.per - 1) / a.per) : 0;
  const u64 groups = p.any ? (rows + 3) / 4 : (a.tokens * a.chunks + 256 / p.lanes - 1) / (256 / p.lanes);
  p.grid = (u32)(back ? (groups < ROPE_GROUPS ? groups : ROPE_GROUPS) : (groups < (1u << 30) ? groups : (1u << 30)));
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
    const u32 grid = (2 * a.dim + 31) / 32;
    if (g->type == G10_F32) k_rope_weights<float><<<grid, 256, 0, s>>>(a, p.grid);
    else if (g->type == G10_F16) k_rope_weights<_Float16><<<grid, 256, 0, s>>>(a, p.grid);
    else k_rope_weights<__bf16><<<grid, 256, 0, s>>>(a, p.grid);
  }
  G10_HIP(hipGetLastError());
  return G10_OK;
}
