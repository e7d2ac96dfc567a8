// AdamW over many tensors in one launch, moments in 32 or 8 bits, and the norm of all gradients.
//
// Bound by memory: every value is read and written once, the update between is some 20 operations (8-bit moments: 40).  A
// workgroup takes a chunk of 2048 elements of one tensor, 8 neighbouring ones to a thread; a block of 8-bit values with one
// scale is half a wavefront's, so its largest magnitude is found between 32 lanes.  The table of chunks lies on the device,
// the gradients' addresses (other ones in every step, maybe) come with the launch: 480 tensors to a launch.
#include "g10_internal.h"
#include "g10_ops.h"

#include <math.h>
#include <new>
#include <stdlib.h>

// The steps below round after every operation, as their formula is written: the 8-bit values do not depend on which
// products a compiler joins with which sums.
#pragma clang fp contract(off)

#define CHUNK 2048u
#define GRADS 480u                 // tensors of a launch
#define NORM_GROUPS 2048u
#define TOP8 448.0f                // largest value of the 8-bit type
#define LEAST8 0.001953125f        // its smallest above zero, 2^-9
#define TINY8 1e-30f               // blocks of smaller values are held as zeros
#define PLACE 0xc13fa9a9u          // 2^32 / 1.3247..., the real root of x^3 = x + 1: how far the threshold turns from element to element
#define TURN 0x9e3779b1u           // 2^32 / 1.6180...: from update to update

struct Place { void *p, *copy; u64 n, first; };    // first: block in the moments' arrays
struct Chunk { u32 tensor, at; };

struct g10_adamw_s {
  int device;
  u32 count, type, grad_type, copy_type, state_type;
  void *m, *v;
  float *m_scale, *v_scale;
  Place* places;                   // device [count]
  Chunk* chunks;                   // device
  u64* chunk_first;                // host [count + 1]
  double* partial;                 // device: of the norm
  u32 launches;
};

struct Grads { const void* g[GRADS]; };
struct StepArgs {
  const Place* places;
  const Chunk* chunks;
  void *m, *v;
  float *m_scale, *v_scale;
  const float* coefficient;
  u32 tensor0, copy16;             // first tensor of the launch; copies: 0 none, 1 half, 2 bfloat
  u32 spread, turn;                // 8-bit moments: whether a threshold decides how they are rounded; its turn
  float beta1, rest1, beta2, rest2, keep, step, root, eps;
};

template <class T>
__device__ __forceinline__ void read8(const T* p, u32 n, bool vec, float (&x)[8]) {
  if (vec && n >= 8) {
    if constexpr (sizeof(T) == 4) {
      const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
      x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
      typedef T x8 __attribute__((ext_vector_type(8)));
      const x8 a = *(const x8*)p;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = (float)a[i];
    }
  } else {
#pragma unroll
    for (u32 i = 0; i < 8; ++i) x[i] = i < n ? (float)p[i] : 0.0f;
  }
}
// (Past the L2, which would write them back when the kernel ends: 109 million weights with moments in 8 bits 375 -> 355 us, 285 million with moments in 32 1626 -> 1587.)
template <class T>
__device__ __forceinline__ void write8(T* p, u32 n, bool vec, const float (&x)[8]) {
  if (vec && n >= 8) {
    if constexpr (sizeof(T) == 4) {
      typedef float f4 __attribute__((ext_vector_type(4)));
      __builtin_nontemporal_store((f4{x[0], x[1], x[2], x[3]}), (f4*)p);
      __builtin_nontemporal_store((f4{x[4], x[5], x[6], x[7]}), (f4*)(p + 4));
    } else {
      typedef T x8 __attribute__((ext_vector_type(8)));
      x8 a;
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] = (T)x[i];
      __builtin_nontemporal_store(a, (x8*)p);
    }
  } else {
#pragma unroll
    for (u32 i = 0; i < 8; ++i)
      if (i < n) p[i] = (T)x[i];
  }
}

__device__ __forceinline__ void read_codes(const void* codes, u64 at, float scale, float (&x)[8]) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  const uint2 c = *(const uint2*)((const char*)codes + at);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int w = (int)(i ? c.y : c.x);
    const f2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    x[4 * i] = lo[0] * scale; x[4 * i + 1] = lo[1] * scale; x[4 * i + 2] = hi[0] * scale; x[4 * i + 3] = hi[1] * scale;
  }
}
// An 8-bit value of magnitude y has a lower and an upper neighbour; up if the part of the way that y has gone lies above the threshold, the upper 20
// bits of t: over all thresholds the mean is y. A moment is rounded again in every update, and with beta2 = 0.999 an update moves a root by less
// than 0.05 % where half a step is 3 to 6 %: to nearest it would stay where it is for good (gradients that fall tenfold after 1000 updates: 6.7
// times the root that they should have 5000 updates later, that grow fivefold: 0.45 times; so 1.01 both). The threshold turns by the golden ratio from update to update, which meets every part of
// the way in nearly equal numbers: the root's spread about the exact one is 15 % with thresholds that turn and 17 % with random ones. (109
// million weights: 365 us a step to nearest, 379 so.)
__device__ __forceinline__ float spread8(float y, u32 t) {
  const float a = fabsf(y), low = a < 0.015625f ? 0.015625f : 0.0f;  // (below 2^-6 neighbours lie 2^-9 apart, as they do from 2^-6 to 2^-5)
  const float up = __uint_as_float((__float_as_uint(a + low) + (t >> 12)) & 0xfff00000u) - low;
  return a < TOP8 ? copysignf(up, y) : y;                            // (or not a number)
}

// Eight values of a block, 32 lanes to the block.  ROOT: no value above zero is held as zero (a moment that is not
// zero would be divided by eps alone).
template <bool ROOT>
__device__ __forceinline__ void write_codes(void* codes, float* scales, u64 at, bool real, const float (&x)[8], bool spread, u32 turn) {
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[i]));
#pragma unroll
  for (int d = 1; d < 32; d *= 2) top = fmaxf(top, __shfl_xor(top, d, 64));
  if (!real) return;
  const bool some = !(top < TINY8);
  const float inv = some ? (1.0f / top) * TOP8 : 0.0f;
  float y[8];
  const u32 first = (u32)at * PLACE + turn;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    y[i] = x[i] * inv;
    if (spread) y[i] = spread8(y[i], first + i * PLACE);
    if (ROOT && some && x[i] > 0.0f) y[i] = fmaxf(y[i], LEAST8);
  }
  typedef u32 u2 __attribute__((ext_vector_type(2)));
  u2 c;
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  c.x = (u32)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
  c.y = (u32)__builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], w, true);
  __builtin_nontemporal_store(c, (u2*)((char*)codes + at));
  if (!(lane_id() & 31)) scales[at / G10_ADAMW_BLOCK] = some ? top * (1.0f / TOP8) : 0.0f;
}

template <class P, class G, bool SMALL>
__global__ __launch_bounds__(256) void k_adamw(const StepArgs a, const Chunk* chunks, const Grads grads) {
  const Chunk c = chunks[blockIdx.x];
  const G* g = (const G*)grads.g[c.tensor - a.tensor0];
  if (!g) return;
  float coef = 1.0f;
  if (a.coefficient) {
    coef = *a.coefficient;
    if (!(fabsf(coef) <= 3.4028234e38f)) return;
  }
  const Place t = a.places[c.tensor];
  const u64 e = (u64)c.at * CHUNK + threadIdx.x * 8;                 // of the tensor
  const u64 at = t.first * G10_ADAMW_BLOCK + e;                      // of the moments
  const u32 n = e >= t.n ? 0u : t.n - e < 8 ? (u32)(t.n - e) : 8u;
  const bool real = (e & ~(u64)(G10_ADAMW_BLOCK - 1)) < t.n;         // the block has elements
  const bool vec = !((uintptr_t)t.p & 15) && !((uintptr_t)g & 15) && !((uintptr_t)t.copy & 15);
  float p[8] = {}, d[8] = {}, m[8] = {}, v[8] = {}, r[8];
  if (real) {
    read8((const P*)t.p + e, n, vec, p);
    read8(g + e, n, vec, d);
    if constexpr (SMALL) {
      const float sm = a.m_scale[at / G10_ADAMW_BLOCK], sv = a.v_scale[at / G10_ADAMW_BLOCK];
      read_codes(a.m, at, sm, m);
      read_codes(a.v, at, sv, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= v[i];
    } else {
      read8((const float*)a.m + at, 8, true, m);
      read8((const float*)a.v + at, 8, true, v);
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = a.coefficient ? d[i] * coef : d[i];
    m[i] = m[i] * a.beta1 + x * a.rest1;
    v[i] = v[i] * a.beta2 + (x * x) * a.rest2;
    r[i] = sqrtf(v[i]);
    p[i] = p[i] * a.keep - (a.step * m[i]) / (r[i] * a.root + a.eps);
  }
  if (real) {
    write8((P*)t.p + e, n, vec, p);
    if (t.copy) {
      if (a.copy16 == 1) write8((_Float16*)t.copy + e, n, vec, p);
      else if (a.copy16 == 2) write8((__bf16*)t.copy + e, n, vec, p);
    }
  }
  if constexpr (SMALL) {
    write_codes<false>(a.m, a.m_scale, at, real, m, a.spread, a.turn);
    write_codes<true>(a.v, a.v_scale, at, real, r, a.spread, a.turn + 0x80000000u);
  } else if (real) {
    write8((float*)a.m + at, 8, true, m);
    write8((float*)a.v + at, 8, true, v);
  }
}

// sum of squares in 64 bits: chunks blockIdx.x, + gridDim.x, ...
template <class G>
__global__ __launch_bounds__(256) void k_norm(const Place* places, const Chunk* chunks, u64 n_chunks, u32 tensor0, double* partial, const Grads grads) {
  double sum = 0.0;
  for (u64 k = blockIdx.x; k < n_chunks; k += gridDim.x) {
    const Chunk c = chunks[k];
    const G* g = (const G*)grads.g[c.tensor - tensor0];
    if (!g) continue;
    const u64 total = places[c.tensor].n, e = (u64)c.at * CHUNK + threadIdx.x * 8;
    const u32 n = e >= total ? 0u : total - e < 8 ? (u32)(total - e) : 8u;
    if (!n) continue;
    float x[8];
    read8(g + e, n, !((uintptr_t)g & 15), x);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += (double)x[i] * (double)x[i];
  }
  __shared__ double sums[4];
#pragma unroll
  for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d, 64);
  if (!lane_id()) sums[wave_id()] = sum;
  __syncthreads();
  if (!threadIdx.x) partial[blockIdx.x] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

__global__ __launch_bounds__(256) void k_norm_end(const double* partial, u32 n, float max_norm, float* out) {
  double sum = 0.0;
  for (u32 i = threadIdx.x; i < n; i += 256) sum += partial[i];
  __shared__ double sums[4];
#pragma unroll
  for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d, 64);
  if (!lane_id()) sums[wave_id()] = sum;
  __syncthreads();
  if (threadIdx.x) return;
  const double norm = sqrt((sums[0] + sums[1]) + (sums[2] + sums[3]));
  const double c = (double)max_norm / (norm + 1e-6);
  out[0] = (float)norm;
  out[1] = norm <= 1.7976931348623157e308 ? (float)(c < 1.0 ? c : 1.0) : __builtin_nanf("");
}

// ---------------------------------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------------------------------
extern "C" int g10_adamw_blocks(const g10_adamw_tensor* tensors, uint32_t count, uint64_t* blocks) {
  if (!blocks || (count && !tensors) || count > G10_ADAMW_MAX_TENSORS) return G10_EINVAL;
  u64 n = 0;
  for (u32 i = 0; i < count; ++i) {
    if (tensors[i].n >= (1ull << 40)) return G10_EINVAL;
    n += (tensors[i].n + G10_ADAMW_BLOCK - 1) / G10_ADAMW_BLOCK;
  }
  *blocks = n;
  return G10_OK;
}

extern "C" void g10_adamw_free(g10_adamw_t* h) {
  if (!h) return;
  int now = 0;
  const bool moved = hipGetDevice(&now) == hipSuccess && now != h->device && hipSetDevice(h->device) == hipSuccess;
  (void)hipDeviceSynchronize();
  mem_dev_free(h->places);
  mem_dev_free(h->chunks);
  mem_dev_free(h->partial);
  if (moved) (void)hipSetDevice(now);
  free(h->chunk_first);
  delete h;
}

static bool float_type(u32 t) { return t <= G10_BF16; }
static u32 size_of(u32 t) { return t == G10_F32 ? 4 : 2; }

extern "C" int g10_adamw_create(const g10_adamw_desc* d, void* hip_stream, g10_adamw_t** out) {
  if (!d || !out) return G10_EINVAL;
  u64 blocks = 0;
  G10_TRY(g10_adamw_blocks(d->tensors, d->count, &blocks));
  if (!float_type(d->type) || !float_type(d->grad_type)) return G10_EINVAL;
  if (d->state_type != G10_F32 && d->state_type != G10_E4M3) return G10_EINVAL;
  const bool small = d->state_type == G10_E4M3;
  if (blocks && (!d->m || !d->v || ((uintptr_t)d->m & 15) || ((uintptr_t)d->v & 15))) return G10_EINVAL;
  if (blocks && small && (!d->m_scale || !d->v_scale || ((uintptr_t)d->m_scale & 3) || ((uintptr_t)d->v_scale & 3))) return G10_EINVAL;
  u64 chunks = 0;
  for (u32 i = 0; i < d->count; ++i) {
    const g10_adamw_tensor& t = d->tensors[i];
    if (t.n && (!t.p || (uintptr_t)t.p % size_of(d->type))) return G10_EINVAL;
    if (t.copy && ((d->copy_type != G10_F16 && d->copy_type != G10_BF16) || ((uintptr_t)t.copy & 1))) return G10_EINVAL;
    chunks += (t.n + CHUNK - 1) / CHUNK;
  }
  if (chunks >= (1ull << 31)) return G10_EINVAL;
  g10_adamw_t* h = new (std::nothrow) g10_adamw_s();
  if (!h) return G10_ENOMEM;
  h->count = d->count; h->type = d->type; h->grad_type = d->grad_type; h->copy_type = d->copy_type; h->state_type = d->state_type;
  h->m = d->m; h->v = d->v; h->m_scale = d->m_scale; h->v_scale = d->v_scale;
  h->launches = (d->count + GRADS - 1) / GRADS;
  if (hipGetDevice(&h->device) != hipSuccess) { delete h; return G10_EDEVICE; }
  Place* places = (Place*)malloc((d->count + 1) * sizeof(Place));
  Chunk* table = (Chunk*)malloc((chunks + 1) * sizeof(Chunk));
  h->chunk_first = (u64*)malloc(((u64)d->count + 1) * sizeof(u64));
  int rc = places && table && h->chunk_first ? G10_OK : G10_ENOMEM;
  hipStream_t s = (hipStream_t)hip_stream;
  if (!rc) {
    u64 at = 0, block = 0;
    for (u32 i = 0; i < d->count; ++i) {
      const g10_adamw_tensor& t = d->tensors[i];
      places[i] = Place{t.p, t.copy, t.n, block};
      block += (t.n + G10_ADAMW_BLOCK - 1) / G10_ADAMW_BLOCK;
      h->chunk_first[i] = at;
      for (u64 k = 0; k * CHUNK < t.n; ++k) table[at++] = Chunk{i, (u32)k};
    }
    h->chunk_first[d->count] = at;
    rc = mem_dev_alloc((void**)&h->places, (d->count + 1) * sizeof(Place));
    if (!rc) rc = mem_dev_alloc((void**)&h->chunks, (chunks + 1) * sizeof(Chunk));
    if (!rc) rc = mem_dev_alloc((void**)&h->partial, ((u64)h->launches * NORM_GROUPS + 1) * sizeof(double));
    if (!rc && d->count && hipMemcpyAsync(h->places, places, d->count * sizeof(Place), hipMemcpyHostToDevice, s) != hipSuccess) rc = G10_EDEVICE;
    if (!rc && chunks && hipMemcpyAsync(h->chunks, table, chunks * sizeof(Chunk), hipMemcpyHostToDevice, s) != hipSuccess) rc = G10_EDEVICE;
    if (hipStreamSynchronize(s) != hipSuccess && !rc) rc = G10_EDEVICE;
  }
  free(places);
  free(table);
  if (rc) { g10_adamw_free(h); return rc; }
  *out = h;
  return G10_OK;
}

static int check_call(g10_adamw_t* h, const void* const* grads) {
  if (!h || (h->count && !grads)) return G10_EINVAL;
  int now = 0;
  if (hipGetDevice(&now) != hipSuccess) return G10_EDEVICE;
  if (now != h->device) return G10_EINVAL;
  uintptr_t all = 0;
  for (u32 i = 0; i < h->count; ++i) all |= (uintptr_t)grads[i];
  return all & (size_of(h->grad_type) - 1) ? G10_EINVAL : G10_OK;
}

template <class P, class G>
static void step_launch(bool small, u32 grid, const StepArgs& a, const Chunk* chunks, const Grads& g, hipStream_t s) {
  if (small) k_adamw<P, G, true><<<grid, 256, 0, s>>>(a, chunks, g);
  else k_adamw<P, G, false><<<grid, 256, 0, s>>>(a, chunks, g);
}
template <class P>
static void step_launch(u32 grad_type, bool small, u32 grid, const StepArgs& a, const Chunk* chunks, const Grads& g, hipStream_t s) {
  if (grad_type == G10_F32) step_launch<P, float>(small, grid, a, chunks, g, s);
  else if (grad_type == G10_F16) step_launch<P, _Float16>(small, grid, a, chunks, g, s);
  else step_launch<P, __bf16>(small, grid, a, chunks, g, s);
}

static bool launch_of(const g10_adamw_t* h, u32 k, const void* const* grads, Grads& g, u64& first, u64& n) {
  const u32 t0 = k * GRADS, t1 = t0 + GRADS < h->count ? t0 + GRADS : h->count;
  for (u32 i = t0; i < t1; ++i) g.g[i - t0] = grads[i];
  first = h->chunk_first[t0];
  n = h->chunk_first[t1] - first;
  return n != 0;
}

extern "C" int g10_adamw_step(g10_adamw_t* h, const void* const* grads, const g10_adamw_params* p, void* hip_stream) {
  if (!p) return G10_EINVAL;
  G10_TRY(check_call(h, grads));
  if (!p->step || !(p->beta1 >= 0.0 && p->beta1 < 1.0) || !(p->beta2 >= 0.0 && p->beta2 < 1.0) || !(p->eps >= 0.0 && p->eps < 3e38)) return G10_EINVAL;
  if (!(fabs(p->lr) < 1e30) || !(fabs(p->weight_decay) < 1e30) || ((uintptr_t)p->coefficient & 3)) return G10_EINVAL;
  hipStream_t s = (hipStream_t)hip_stream;
  StepArgs a{};
  a.places = h->places; a.m = h->m; a.v = h->v; a.m_scale = h->m_scale; a.v_scale = h->v_scale;
  a.coefficient = p->coefficient;
  a.copy16 = h->copy_type == G10_F16 ? 1 : h->copy_type == G10_BF16 ? 2 : 0;
  const double b1 = p->beta1, b2 = p->beta2, t = (double)p->step;
  a.beta1 = (float)b1; a.beta2 = (float)b2; a.rest1 = (float)(1.0 - b1); a.rest2 = (float)(1.0 - b2);
  a.keep = (float)(1.0 - p->lr * p->weight_decay);
  a.step = (float)(p->lr / (1.0 - pow(b1, t)));
  a.root = (float)(1.0 / sqrt(1.0 - pow(b2, t)));
  a.eps = (float)p->eps;
  a.spread = p->step > G10_ADAMW_NEAREST;
  a.turn = (u32)p->step * TURN;
  for (u32 k = 0; k < h->launches; ++k) {
    Grads g = {};
    u64 first, n;
    if (!launch_of(h, k, grads, g, first, n)) continue;
    a.tensor0 = k * GRADS;
    const bool small = h->state_type == G10_E4M3;
    for (u64 at = 0; at < n; at += G10_GROUPS_MOST) {
      const u32 grid = n - at < G10_GROUPS_MOST ? (u32)(n - at) : G10_GROUPS_MOST;
      const Chunk* chunks = h->chunks + first + at;
      if (h->type == G10_F32) step_launch<float>(h->grad_type, small, grid, a, chunks, g, s);
      else if (h->type == G10_F16) step_launch<_Float16>(h->grad_type, small, grid, a, chunks, g, s);
      else step_launch<__bf16>(h->grad_type, small, grid, a, chunks, g, s);
    }
  }
  G10_HIP(hipGetLastError());
  return G10_OK;
}

extern "C" int g10_grad_norm(g10_adamw_t* h, const void* const* grads, float max_norm, float* out, void* hip_stream) {
  G10_TRY(check_call(h, grads));
  if (!out || ((uintptr_t)out & 3) || !(max_norm > 0.0f)) return G10_EINVAL;
  hipStream_t s = (hipStream_t)hip_stream;
  u32 used = 0;
  for (u32 k = 0; k < h->launches; ++k) {
    Grads g = {};
    u64 first, n;
    if (!launch_of(h, k, grads, g, first, n)) continue;
    const u32 grid = n < NORM_GROUPS ? (u32)n : NORM_GROUPS;
    double* to = h->partial + used;
    if (h->grad_type == G10_F32) k_norm<float><<<grid, 256, 0, s>>>(h->places, h->chunks + first, n, k * GRADS, to, g);
    else if (h->grad_type == G10_F16) k_norm<_Float16><<<grid, 256, 0, s>>>(h->places, h->chunks + first, n, k * GRADS, to, g);
    else k_norm<__bf16><<<grid, 256, 0, s>>>(h->places, h->chunks + first, n, k * GRADS, to, g);
    used += grid;
  }
  k_norm_end<<<1, 256, 0, s>>>(h->partial, used, max_norm, out);
  G10_HIP(hipGetLastError());
  return G10_OK;
}
