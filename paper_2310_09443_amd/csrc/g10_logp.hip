// Log probabilities of given tokens, entropy, the likeliest tokens of each row, and the gradient of the logits.
//
// Bound by memory: forward a logit is read once, backward read and written once.  A workgroup takes a row in one pass: each thread keeps
// its own running maximum m, sum s of exp(z - m) and sum t of exp(z - m) (z - m), which are scaled when the maximum moves and joined
// at the end:  lse = m + log s,  entropy = log s - t / s.  Differences are taken before the product with the scale: z - m is then as
// exact as the logits.
//
// The `top` likeliest: beside the sums each thread remembers its own largest logit.  The top-th largest of the 64 that a wavefront's lanes
// remember is no larger than the row's top-th largest, so the largest such bound of all wavefronts leaves few candidates, and they lie with
// the threads whose own largest passes it: these read theirs again (from the cache), and a candidate's rank is the number of
// candidates above it.  Keys are the logit's bits in order with the complement of its place below them: no two are equal, and of equal
// logits the first comes first.  Where there are more candidates than room, or a NaN, the row is read once for each of the top.
#include "g10_internal.h"
#include "g10_ops.h"

#include <math.h>

struct LogpArgs {
  const void *logits, *tokens;
  float *logp, *lse, *entropy, *top_logp;
  int64_t* top_ids;
  const float *dlogp, *dentropy;
  void* dlogits;
  int64_t ls, ds, ignore;
  u32 rows, vocab, top;
  float scale, scale2;             // scale2: in powers of two
};

#define LOGP_LOG2E 1.4426950408889634f
#define LOGP_LN2 0.6931471805599453f
#define LOGP_NEG_INF (-__builtin_inff())
#define LOGP_ROOM 1024u            // candidates of a row
#define LOGP_NAN 0xfffffffeu

// A product that is 0 where p is, whatever x is (v_mul_legacy_f32, which the compiler knows by this name only).
extern "C" __device__ float logp_times(float p, float x) __asm("llvm.amdgcn.fmul.legacy");

// Bits in the order of the numbers, NaN above all, both zeros alike.
__device__ __forceinline__ u32 in_order(float x) {
  if (x != x) return LOGP_NAN;
  const u32 b = __float_as_uint(x + 0.0f);
  return b ^ (u32)(((int)b >> 31) | (int)0x80000000);
}
__device__ __forceinline__ float out_of_order(u32 k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
__device__ __forceinline__ u64 key_of(float x, u32 place) { return ((u64)in_order(x) << 32) | (u32)~place; }

struct Sums { float m, s, t; };
__device__ __forceinline__ Sums join(const Sums& a, const Sums& b, float scale2) {
  const float m = fmaxf(a.m, b.m);
  if (m == LOGP_NEG_INF) return {m, a.s + b.s, a.t + b.t};            // (nothing yet, or NaN)
  const float da = (a.m - m) * scale2, db = (b.m - m) * scale2;
  const float fa = __builtin_amdgcn_exp2f(da), fb = __builtin_amdgcn_exp2f(db);
  return {m, a.s * fa + b.s * fb, logp_times(fa, a.t + logp_times(a.s, da)) + logp_times(fb, b.t + logp_times(b.s, db))};
}

// A row in pieces of 16 bytes: values up to the first whole piece, the pieces, and what is left.
template <class T>
struct Row {
  static constexpr u32 N = 16 / sizeof(T);
  typedef T V __attribute__((ext_vector_type(N)));
  const T* p;
  u32 n, head, pieces;
  __device__ __forceinline__ Row(const T* row, u32 vocab) : p(row), n(vocab) {
    head = (u32)((0 - (uintptr_t)row) & 15) / (u32)sizeof(T);
    if (head > n) head = n;
    pieces = (n - head) / N;
  }
  __device__ __forceinline__ V piece(u32 i) const { return *(const V*)(p + head + (u64)i * N); }
  __device__ __forceinline__ u32 place(u32 i) const { return head + i * N; }
  __device__ __forceinline__ u32 tail() const { return head + pieces * N; }
  // f(value, place) for a thread's value before the pieces, and behind them
  template <class F>
  __device__ __forceinline__ void first(u32 tid, F&& f) const {
    if (tid < head) f((float)p[tid], tid);
  }
  template <class F>
  __device__ __forceinline__ void last(u32 tid, F&& f) const {
    const u32 at = tail() + tid;
    if (tid < N && at < n) f((float)p[at], at);
  }
  // and for all of a thread's values
  template <u32 NT, class F>
  __device__ __forceinline__ void each(u32 tid, F&& f) const {
    first(tid, f);
    last(tid, f);
    for (u32 i = tid; i < pieces; i += NT) {
      const V v = piece(i);
#pragma unroll
      for (u32 k = 0; k < N; ++k) f((float)v[k], place(i) + k);
    }
  }
};

template <class T, int NT, bool TOP>
__global__ __launch_bounds__(NT) void k_logp(const LogpArgs a) {
  constexpr u32 W = NT / 64, AHEAD = 4, N = Row<T>::N;
  typedef typename Row<T>::V V;
  __shared__ Sums sums[W];
  __shared__ u64 bounds[W];
  __shared__ u64 list[TOP ? LOGP_ROOM : 1];
  __shared__ u32 listed;
  const u32 tid = threadIdx.x;
  for (u64 row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const Row<T> r((const T*)a.logits + (int64_t)row * a.ls, a.vocab);
    Sums me = {LOGP_NEG_INF, 0.0f, 0.0f};
    float best = LOGP_NEG_INF;
    u64 mine = 0;                                                     // the largest key
    auto one = [&](float x, u32 place) {
      const Sums b = {x, x == x && x != LOGP_NEG_INF ? 1.0f : x != x ? x : 0.0f, 0.0f};
      me = join(me, b, a.scale2);
      if (TOP) {
        const u64 k = key_of(x, place);
        if (k > mine) { mine = k; best = x; }
      }
    };
    auto take = [&](const V& v, u32 place) {
      float x[N], top = LOGP_NEG_INF;
#pragma unroll
      for (u32 k = 0; k < N; ++k) { x[k] = (float)v[k]; top = fmaxf(top, x[k]); }
      if (TOP && (top > best || mine == 0)) {
#pragma unroll
        for (u32 k = 0; k < N; ++k) {
          const u64 key = key_of(x[k], place + k);
          if (key > mine) mine = key;
        }
        best = top;
      }
      if (top > me.m) {
        const float d = (me.m - top) * a.scale2, f = __builtin_amdgcn_exp2f(d);
        me.t = logp_times(f, me.t + logp_times(me.s, d));                // (d may be -infinity: logits apart by more than 32 bits hold)
        me.s *= f;
        me.m = top;
      }
      const float m = me.m == LOGP_NEG_INF ? 0.0f : me.m;
#pragma unroll
      for (u32 k = 0; k < N; ++k) {
        const float d = (x[k] - m) * a.scale2, e = __builtin_amdgcn_exp2f(d);
        me.s += e;
        me.t += logp_times(e, d);
      }
    };
    r.first(tid, one);                                                // (places in their order: of equal logits a thread keeps the first)
    u32 i = tid;
    for (; i + (AHEAD - 1) * NT < r.pieces; i += AHEAD * NT) {
      V v[AHEAD];
#pragma unroll
      for (u32 u = 0; u < AHEAD; ++u) v[u] = r.piece(i + u * NT);
#pragma unroll
      for (u32 u = 0; u < AHEAD; ++u) take(v[u], r.place(i + u * NT));
    }
    for (; i < r.pieces; i += NT) take(r.piece(i), r.place(i));
    r.last(tid, one);
    // the row's sums
#pragma unroll
    for (u32 d = 1; d < 64; d *= 2) {
      const Sums o = {__shfl_xor(me.m, d, 64), __shfl_xor(me.s, d, 64), __shfl_xor(me.t, d, 64)};
      me = lane_id() & d ? join(o, me, a.scale2) : join(me, o, a.scale2);
    }
    if constexpr (TOP) {
      // the top-th largest of the wavefront's 64, 0 if there are not so many
      u32 above = 0;
#pragma unroll
      for (u32 j = 0; j < 64; ++j) {
        const u64 o = ((u64)(u32)__builtin_amdgcn_readlane((int)(u32)(mine >> 32), j) << 32) | (u32)__builtin_amdgcn_readlane((int)(u32)mine, j);
        above += o > mine;
      }
      const u64 at = ballot(above == a.top - 1 && mine != 0);
      const u32 who = at ? (u32)__builtin_ctzll(at) : 0;
      const u64 key = ((u64)(u32)__builtin_amdgcn_readlane((int)(u32)(mine >> 32), who) << 32) | (u32)__builtin_amdgcn_readlane((int)(u32)mine, who);
      if (lane_id() == 0) bounds[wave_id()] = at ? key : 0;
      if (tid == 0) listed = 0;
    }
    if (lane_id() == 0) sums[wave_id()] = me;
    __syncthreads();
    Sums all = sums[0];
#pragma unroll
    for (u32 w = 1; w < W; ++w) all = join(all, sums[w], a.scale2);
    const bool none = all.m == LOGP_NEG_INF && all.s == 0.0f;
    const float ls = __log2f(all.s) * LOGP_LN2, lse = none ? LOGP_NEG_INF : all.m * a.scale + ls;
    if (tid == 0) {
      a.lse[row] = lse;
      if (a.entropy) a.entropy[row] = none ? 0.0f : ls - all.t / all.s * LOGP_LN2;
      if (a.tokens) {
        const int64_t t = ((const int64_t*)a.tokens)[row];
        float lp = __builtin_nanf("");
        if (t == a.ignore) lp = 0.0f;
        else if (t >= 0 && t < (int64_t)a.vocab) lp = none ? LOGP_NEG_INF : (float)r.p[t] * a.scale - lse;
        a.logp[row] = lp;
      }
    }
    if constexpr (TOP) {
      u64 least = bounds[0];
#pragma unroll
      for (u32 w = 1; w < W; ++w) least = bounds[w] > least ? bounds[w] : least;
      if (mine >= least && mine) {
        r.template each<NT>(tid, [&](float x, u32 place) {
          const u64 key = key_of(x, place);
          if (key >= least) {
            const u32 at = atomicAdd(&listed, 1u);
            if (at < LOGP_ROOM) list[at] = key;
          }
        });
      }
      __syncthreads();
      const u32 n = listed;
      auto put = [&](u32 rank, u64 key) {
        a.top_ids[row * a.top + rank] = (int64_t)(u32)~(u32)key;
        a.top_logp[row * a.top + rank] = none ? LOGP_NEG_INF : key >> 32 == LOGP_NAN ? __builtin_nanf("") : out_of_order((u32)(key >> 32)) * a.scale - lse;
      };
      if (n <= LOGP_ROOM && all.s == all.s) {
        for (u32 c = tid; c < n; c += NT) {
          const u64 key = list[c];
          u32 above = 0;
          for (u32 j = 0; j < n; ++j) above += list[j] > key;
          if (above < a.top) put(above, key);
        }
      } else {
        u64 last = ~0ull;                                             // (above every key)
        for (u32 k = 0; k < a.top; ++k) {
          u64 next = 0;
          r.template each<NT>(tid, [&](float x, u32 place) {
            const u64 key = key_of(x, place);
            if (key < last && key > next) next = key;
          });
#pragma unroll
          for (u32 d = 1; d < 64; d *= 2) {
            const u64 o = ((u64)(u32)__shfl_xor((int)(u32)(next >> 32), d, 64) << 32) | (u32)__shfl_xor((int)(u32)next, d, 64);
            next = o > next ? o : next;
          }
          __syncthreads();
          if (lane_id() == 0) bounds[wave_id()] = next;
          __syncthreads();
          last = bounds[0];
#pragma unroll
          for (u32 w = 1; w < W; ++w) last = bounds[w] > last ? bounds[w] : last;
          if (tid == 0) put(k, last);
        }
      }
    }
    __syncthreads();                                                  // (the next row's sums go where these lie)
  }
}

// The gradient of a row: p (c0 + c1 log p), c0 = - (dlogp + dentropy entropy), c1 = - dentropy, and dlogp at the token.
template <class T>
__global__ __launch_bounds__(256) void k_logp_back(const LogpArgs a, u32 vec) {
  constexpr u32 N = Row<T>::N;
  typedef typename Row<T>::V V;
  for (u64 row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const Row<T> r((const T*)a.logits + (int64_t)row * a.ls, a.vocab);
    T* out = (T*)a.dlogits + (int64_t)row * a.ds;
    const float lse = a.lse[row];
    float dl = a.tokens && a.dlogp ? a.dlogp[row] : 0.0f;
    const float de = a.dentropy ? a.dentropy[row] : 0.0f;
    int64_t t = a.tokens ? ((const int64_t*)a.tokens)[row] : -1;
    if (a.tokens) {
      if (t == a.ignore) { dl = 0.0f; t = -1; }
      else if (t < 0 || t >= (int64_t)a.vocab) { dl = __builtin_nanf(""); t = -1; }
    }
    const bool none = lse == LOGP_NEG_INF;
    const float c0 = none ? 0.0f : -(dl + (a.dentropy ? de * a.entropy[row] : 0.0f)) * a.scale, c1 = none ? 0.0f : -de * a.scale, hit = none ? 0.0f : dl * a.scale;
    const bool zero = c0 == 0.0f && c1 == 0.0f && hit == 0.0f;        // (nothing of the row counts: it is not read)
    auto grad = [&](float x, u32 place) {
      const float lp = __builtin_fmaf(x, a.scale, -lse);              // -infinity where there is no probability
      const float p = __builtin_amdgcn_exp2f(lp * LOGP_LOG2E);
      float g = p * c0;
      if (a.dentropy) g += logp_times(p, lp) * c1;
      return (place == (u32)t && t >= 0 ? g + hit : g);
    };
    if (zero) {
      auto nothing = [&](u32 at) { out[at] = (T)0.0f; };
      const u32 head = (u32)((0 - (uintptr_t)out) & 15) / (u32)sizeof(T), h = head < a.vocab ? head : a.vocab, pieces = (a.vocab - h) / N;
      const V z = {};
      if (threadIdx.x < h) nothing(threadIdx.x);
      for (u32 i = threadIdx.x; i < pieces; i += 256) __builtin_nontemporal_store(z, (V*)(out + h + (u64)i * N));
      const u32 at = h + pieces * N + threadIdx.x;
      if (threadIdx.x < N && at < a.vocab) nothing(at);
    } else if (vec) {
      auto one = [&](float x, u32 place) { out[place] = (T)grad(x, place); };
      r.first(threadIdx.x, one);
      r.last(threadIdx.x, one);
      for (u32 i = threadIdx.x; i < r.pieces; i += 256) {
        const V v = r.piece(i);
        V w;
#pragma unroll
        for (u32 k = 0; k < N; ++k) w[k] = (T)grad((float)v[k], r.place(i) + k);
        __builtin_nontemporal_store(w, (V*)(out + r.place(i)));
      }
    } else {
      for (u32 i = threadIdx.x; i < a.vocab; i += 256) out[i] = (T)grad((float)r.p[i], i);
    }
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------------------------------
static int logp_args(const g10_log_probs_args* g, bool back, LogpArgs& a) {
  if (!g) return G10_EINVAL;
  if (g->type > G10_BF16 || !(g->scale > 0.0f) || isinf(g->scale) || !g->vocab || g->vocab >= 0x80000000u || g->rows >= 0x80000000u) return G10_EINVAL;
  const u32 e = g->type == G10_F32 ? 4 : 2;
  if ((uintptr_t)g->logits % e || (uintptr_t)g->dlogits % e || (uintptr_t)g->tokens % 8) return G10_EINVAL;
  if (g->rows && (!g->logits || !g->lse)) return G10_EINVAL;
  if (!back) {
    if (g->top > G10_LOG_PROBS_TOP || g->top > g->vocab) return G10_EINVAL;
    if (g->rows && ((g->tokens && !g->logp) || (g->top && (!g->top_logp || !g->top_ids)))) return G10_EINVAL;
  } else if (g->rows && (!g->dlogits || (g->dlogp && !g->tokens) || (g->dentropy && !g->entropy))) {
    return G10_EINVAL;
  }
  a = LogpArgs{};
  a.logits = g->logits; a.tokens = g->tokens; a.logp = g->logp; a.lse = g->lse; a.entropy = g->entropy;
  a.top_logp = g->top_logp; a.top_ids = g->top_ids; a.dlogp = g->dlogp; a.dentropy = g->dentropy; a.dlogits = g->dlogits;
  a.ls = g->logits_stride; a.ds = g->dlogits_stride; a.ignore = g->ignore;
  a.rows = g->rows; a.vocab = g->vocab; a.top = back ? 0 : g->top;
  a.scale = g->scale; a.scale2 = g->scale * LOGP_LOG2E;
  return G10_OK;
}

template <class T>
static void logp_launch(const LogpArgs& a, hipStream_t s) {
  const u32 grid = a.rows < 1u << 16 ? a.rows : 1u << 16;
  if (a.rows <= 512 && a.vocab > 4096) {
    if (a.top) k_logp<T, 1024, true><<<grid, 1024, 0, s>>>(a); else k_logp<T, 1024, false><<<grid, 1024, 0, s>>>(a);
  } else {
    if (a.top) k_logp<T, 256, true><<<grid, 256, 0, s>>>(a); else k_logp<T, 256, false><<<grid, 256, 0, s>>>(a);
  }
}

extern "C" int g10_log_probs_workspace(const g10_log_probs_args* g, uint64_t* bytes) {
  if (!bytes) return G10_EINVAL;
  LogpArgs a;
  G10_TRY(logp_args(g, false, a));
  *bytes = 0;
  return G10_OK;
}

extern "C" int g10_log_probs(const g10_log_probs_args* g, void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  LogpArgs a;
  G10_TRY(logp_args(g, false, a));
  if (!a.rows) return G10_OK;
  hipStream_t s = (hipStream_t)hip_stream;
  if (g->type == G10_F32) logp_launch<float>(a, s);
  else if (g->type == G10_F16) logp_launch<_Float16>(a, s);
  else logp_launch<__bf16>(a, s);
  G10_HIP(hipGetLastError());
  return G10_OK;
}

extern "C" int g10_log_probs_backward(const g10_log_probs_args* g, void* hip_stream) {
  LogpArgs a;
  G10_TRY(logp_args(g, true, a));
  if (!a.rows) return G10_OK;
  hipStream_t s = (hipStream_t)hip_stream;
  const u32 grid = a.rows < 1u << 16 ? a.rows : 1u << 16, e = g->type == G10_F32 ? 4 : 2;
  // (rows of both tensors lie alike within 16 bytes)
  const u32 vec = !(((uintptr_t)g->logits ^ (uintptr_t)g->dlogits) & 15) && ((g->logits_stride - g->dlogits_stride) * (int64_t)e) % 16 == 0;
  if (g->type == G10_F32) k_logp_back<float><<<grid, 256, 0, s>>>(a, vec);
  else if (g->type == G10_F16) k_logp_back<_Float16><<<grid, 256, 0, s>>>(a, vec);
  else k_logp_back<__bf16><<<grid, 256, 0, s>>>(a, vec);
  G10_HIP(hipGetLastError());
  return G10_OK;
}
