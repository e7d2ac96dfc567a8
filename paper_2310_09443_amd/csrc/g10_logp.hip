// Log probabilities of given tokens, entropy, the likeliest tokens of each row, and the gradient of the logits.
//
// Bound by memory: forward a logit is read once, backward read and written once.  A workgroup takes a row in one pass: each thread keeps
// its own running maximum m, sum s of exp(z - m) and sum t of exp(z - m) (z - m), which are scaled when the maximum moves and brought to
// the row's maximum at the end:  lse = m + log s,  entropy = log s - t / s,  and of a logit  log p = (z - m) - log s.
//
// The `top` likeliest: beside the sums each thread remembers its own largest logit, and 64 groups of threads theirs.  The top-th largest of the
// 64 is no larger than the row's top-th largest, and little is above it: 32000 logits and a top of 20 leave some 24 candidates.  They lie
// with the threads whose own largest passes the bound; these go through theirs again, in registers where the row fits into the
// workgroup's, and a candidate's rank is the number of candidates above it.  Keys are the logit's bits in order with the complement of its place
// below them: no two are equal, and of equal logits the first comes first.  Where there are more candidates than room, or a NaN, the row is read once for
// each of the top.  That is so where one thread's logits are all large; where fewer groups than `top` hold a logit that counts, so that the bound is -infinity or
// there is none: rows of which nearly all is masked (8 rows of 32000 with 10 logits left, a top of 20: 94 us for 9), and tops above 33 of rows of 513 to
// some 1000 pieces, which fill a sixteenth as many groups (8 rows of 5000 in 16 bits: a top of 20 6 us, of 50 108).
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
  // few long rows: `parts` workgroups to a row, `each` logits to one; what they find
  u32 parts, each;
  struct Part* part;               // [row][part]
  u64* part_top;                   // [row][part][top]: keys, 0 where there are no more
};
struct Part { float top, top2, s, t; };   // the largest logit, the same in powers of two as it was taken off; far beyond the range top2 is cut, the sums are not

#define LOGP_LOG2E 1.4426950408889634f
#define LOGP_LN2 0.6931471805599453f
#define LOGP_NEG_INF (-__builtin_inff())
#define LOGP_ROOM 1024u            // candidates of a row
#define LOGP_SCALE 2e38f           // (in powers of two still a number)
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

// z - m is taken as one multiply-add of the logit and m in powers of two, which is rounded: what that leaves over is in every exponential and, with
// the same m, taken out of lse again.  Far from zero it would be more than an exponential holds: m stays within 1e8 (a rounding of 4), and rows
// beyond that are summed again with their differences taken first.
#define LOGP_FAR 1e8f
__device__ __forceinline__ float in_range(float x) { return fminf(fmaxf(x, -LOGP_FAR), LOGP_FAR); }

template <int CTRL>
__device__ __forceinline__ float dpp(float x) { return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(x), __float_as_int(x), CTRL, 0xf, 0xf, false)); }
__device__ __forceinline__ float wave_max(float x) {
  x = fmaxf(x, dpp<0xb1>(x));                                         // lanes 1, 0, 3, 2 of a quad
  x = fmaxf(x, dpp<0x4e>(x));                                         // lanes 2, 3, 0, 1
  x = fmaxf(x, dpp<0x141>(x));                                        // eight lanes mirrored
  x = fmaxf(x, dpp<0x140>(x));                                        // sixteen lanes mirrored
  x = fmaxf(x, __shfl_xor(x, 16, 64));
  return fmaxf(x, __shfl_xor(x, 32, 64));
}
__device__ __forceinline__ float wave_add(float x) {
  x += dpp<0xb1>(x);
  x += dpp<0x4e>(x);
  x += dpp<0x141>(x);
  x += dpp<0x140>(x);
  x += __shfl_xor(x, 16, 64);
  return x + __shfl_xor(x, 32, 64);
}
template <int CTRL>
__device__ __forceinline__ u64 dpp_most(u64 x) {
  const u64 y = ((u64)(u32)__builtin_amdgcn_update_dpp(0, (int)(u32)(x >> 32), CTRL, 0xf, 0xf, false) << 32) |
                (u32)__builtin_amdgcn_update_dpp(0, (int)(u32)x, CTRL, 0xf, 0xf, false);
  return y > x ? y : x;
}
__device__ __forceinline__ u64 lane_key(u64 x, u32 lane) {
  return ((u64)(u32)__builtin_amdgcn_readlane((int)(u32)(x >> 32), (int)lane) << 32) | (u32)__builtin_amdgcn_readlane((int)(u32)x, (int)lane);
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

// What a row's sum was taken from: its largest logit, the same in powers of two as it was taken off, and the sum's logarithm in powers of two.
struct Found { float top, top2, log; };
// The row's lse is a place, which 32 bits round where it lies: a row of 32000 times -1e9 has the lse -1e9.  A logarithm of a probability is a distance,
// and is taken from the row's largest logit: what of top2 is rounding is in the sum as well.
__device__ __forceinline__ bool is_none(const Found& r, float s) { return r.top == LOGP_NEG_INF && s == 0.0f; }
__device__ __forceinline__ bool is_far(const Found& r) { return fabsf(r.top2) >= LOGP_FAR && r.top != LOGP_NEG_INF; }
__device__ __forceinline__ float lse_of(const LogpArgs& a, const Found& r, bool none) {
  return none ? LOGP_NEG_INF : is_far(r) ? __builtin_fmaf(r.top, a.scale, r.log * LOGP_LN2) : (r.top2 + r.log) * LOGP_LN2;
}
__device__ __forceinline__ float log_of(const LogpArgs& a, const Found& r, bool none, float x) {
  if (none) return LOGP_NEG_INF;
  // (halves: logits at both ends of the type lie further apart than it holds; what they lose of a small logit is nothing beside the top)
  if (is_far(r)) return __builtin_fmaf((0.5f * x - 0.5f * r.top) * a.scale, 2.0f, -r.log * LOGP_LN2);
  const float d = __builtin_fmaf(x, a.scale2, -r.top2);
  return d < -LOGP_FAR ? __builtin_fmaf(x, a.scale, -lse_of(a, r, none)) : (d - r.log) * LOGP_LN2;      // (a distance may end 32 bits in powers of two alone)
}

template <class T>
__device__ __forceinline__ void put_logp(const LogpArgs& a, u64 row, const Found& r, bool none) {
  const int64_t token = ((const int64_t*)a.tokens)[row];
  float lp = __builtin_nanf("");
  if (token == a.ignore) lp = 0.0f;
  else if (token >= 0 && token < (int64_t)a.vocab) lp = log_of(a, r, none, (float)((const T*)a.logits)[(int64_t)row * a.ls + token]);
  a.logp[row] = lp;
}
__device__ __forceinline__ void put_top(const LogpArgs& a, u64 row, u32 rank, u64 key, const Found& r, bool none) {
  a.top_ids[row * a.top + rank] = (int64_t)(u32)~(u32)key;
  a.top_logp[row * a.top + rank] = key >> 32 == LOGP_NAN ? __builtin_nanf("") : log_of(a, r, none, out_of_order((u32)(key >> 32)));
}

// NT threads to a row or a part of one.  P > 0: its pieces stay in registers, P to a thread; 0: they are read as they are needed.
enum { LOGP_LSE = 0, LOGP_ENTROPY = 1, LOGP_TOP = 2 };                // each with what the one before gives
template <class T, int NT, int P, int WHAT>
__global__ __launch_bounds__(NT) void k_logp(const LogpArgs a) {
  constexpr u32 W = NT / 64, AHEAD = P ? P : 4, N = Row<T>::N;
  constexpr bool TOP = WHAT == LOGP_TOP, ENTROPY = WHAT >= LOGP_ENTROPY;
  typedef typename Row<T>::V V;
  __shared__ float maxima[W], sums[2][W];
  __shared__ u64 keys[TOP ? 64 : 1], bounds[TOP ? W : 1], list[TOP ? LOGP_ROOM : 1];
  __shared__ u32 rank[TOP ? 64 : 1], listed;
  const u32 tid = threadIdx.x;
  for (u64 b = blockIdx.x; b < (u64)a.rows * a.parts; b += gridDim.x) {
    const u64 row = b / a.parts;
    const u32 first = (u32)(b % a.parts) * a.each, count = a.vocab - first < a.each ? a.vocab - first : a.each;
    const u32 wanted = a.top < count ? a.top : count;                 // of this part
    const Row<T> r((const T*)a.logits + (int64_t)row * a.ls + first, count);
    float m = LOGP_NEG_INF, m2 = 0.0f, s = 0.0f, t = 0.0f;            // m2: the maximum in powers of two, rounded once and then used as it is
    // the thread's largest logit, and where the first piece with it begins
    const bool has = tid < r.head || tid < r.pieces || (tid < N && r.tail() + tid < r.n);
    float best = LOGP_NEG_INF;
    u32 at = tid < r.head ? tid : tid < r.pieces ? r.place(tid) : r.tail() + tid;
    auto take = [&](const float* x, u32 n, u32 place) {
      float top = x[0];
#pragma unroll
      for (u32 k = 1; k < n; ++k) top = fmaxf(top, x[k]);
      if (TOP) {
        at = top > best ? place : at;
        best = fmaxf(best, top);
      }
      if (top > m) {
        const float now = in_range(top * a.scale2), d = m2 - now, f = m == LOGP_NEG_INF ? 1.0f : __builtin_amdgcn_exp2f(d);      // (nothing to scale yet, but a NaN stays)
        if (ENTROPY) t = logp_times(f, t + logp_times(s, d));         // (d may be -infinity: logits apart by more than 32 bits hold)
        s *= f;
        m = top;
        m2 = now;
      }
#pragma unroll
      for (u32 k = 0; k < n; ++k) {
        const float d = __builtin_fmaf(x[k], a.scale2, -m2), e = __builtin_amdgcn_exp2f(d);
        s += e;
        if (ENTROPY) t += logp_times(e, d);
      }
    };
    auto one = [&](float x, u32 place) { take(&x, 1, place); };
    auto piece = [&](const V& v, u32 place) {
      float x[N];
#pragma unroll
      for (u32 k = 0; k < N; ++k) x[k] = (float)v[k];
      take(x, N, place);
    };
    r.first(tid, one);                                                // (places in their order: of equal logits a thread keeps the first)
    V held[AHEAD];
    if constexpr (P > 0) {
      if (r.pieces) {
#pragma unroll
        for (u32 u = 0; u < P; ++u) held[u] = r.piece(tid + u * NT < r.pieces ? tid + u * NT : 0);
      }
#pragma unroll
      for (u32 u = 0; u < P; ++u)
        if (tid + u * NT < r.pieces) piece(held[u], r.place(tid + u * NT));
    } else {
      u32 i = tid;
      for (; i + (AHEAD - 1) * NT < r.pieces; i += AHEAD * NT) {
#pragma unroll
        for (u32 u = 0; u < AHEAD; ++u) held[u] = r.piece(i + u * NT);
#pragma unroll
        for (u32 u = 0; u < AHEAD; ++u) piece(held[u], r.place(i + u * NT));
      }
      for (; i < r.pieces; i += NT) piece(r.piece(i), r.place(i));
    }
    r.last(tid, one);
    // the row's maximum; the largest logits of 64 groups of threads, as keys that are not above those of the logits themselves
    const float wm = wave_max(m);
    if (lane_id() == 0) maxima[wave_id()] = wm;
    if constexpr (TOP) {
      u64 k = has ? key_of(best, first + at + (N - 1)) : 0;
      if (NT >= 128) k = dpp_most<0xb1>(k);
      if (NT >= 256) k = dpp_most<0x4e>(k);
      if (NT >= 512) k = dpp_most<0x141>(k);
      if (NT >= 1024) k = dpp_most<0x140>(k);
      if (tid % (NT / 64) == 0) keys[tid / (NT / 64)] = k;
      if (tid < 64) rank[tid] = 0;
      if (tid == 0) listed = 0;
    }
    __syncthreads();
    float top = maxima[0];
#pragma unroll
    for (u32 w = 1; w < W; ++w) top = fmaxf(top, maxima[w]);
    const float top2 = in_range(top * a.scale2);
    {
      const float d = m == LOGP_NEG_INF ? 0.0f : m2 - top2, f = __builtin_amdgcn_exp2f(d);
      if (ENTROPY) t = logp_times(f, t + logp_times(s, d));
      s *= f;
    }
    s = wave_add(s);
    if (ENTROPY) t = wave_add(t);
    if (lane_id() == 0) {
      sums[0][wave_id()] = s;
      if (ENTROPY) sums[1][wave_id()] = t;
    }
    if constexpr (TOP) {                                              // how many groups' are above each: a share of them to each wavefront
      const u64 k = keys[lane_id()];
      u32 above = 0;
#pragma unroll
      for (u32 j = 0; j < 64 / W; ++j) above += lane_key(k, wave_id() * (64 / W) + j) > k;
      if (above) atomicAdd(&rank[lane_id()], above);
    }
    __syncthreads();
    s = sums[0][0];
    t = ENTROPY ? sums[1][0] : 0.0f;
#pragma unroll
    for (u32 w = 1; w < W; ++w) {
      s += sums[0][w];
      if (ENTROPY) t += sums[1][w];
    }
    Found found = {top, top2, 0.0f};
    const bool none = is_none(found, s);
    if (is_far(found)) {                                              // (a row masked with the type's lowest value, say)
      s = t = 0.0f;
      r.template each<NT>(tid, [&](float x, u32) {
        const float d = (x - top) * a.scale2, e = __builtin_amdgcn_exp2f(d);
        s += e;
        if (ENTROPY) t += logp_times(e, d);
      });
      s = wave_add(s);
      if (ENTROPY) t = wave_add(t);
      __syncthreads();
      if (lane_id() == 0) {
        sums[0][wave_id()] = s;
        if (ENTROPY) sums[1][wave_id()] = t;
      }
      __syncthreads();
      s = t = 0.0f;
      for (u32 w = 0; w < W; ++w) {
        s += sums[0][w];
        if (ENTROPY) t += sums[1][w];
      }
    }
    if (a.parts > 1) {
      if (tid == 0) a.part[b] = {top, top2, s, t};
    }
    found.log = __log2f(s);
    if (tid == 0 && a.parts == 1) {
      a.lse[row] = lse_of(a, found, none);
      if (ENTROPY && a.entropy) a.entropy[row] = none ? 0.0f : (found.log - t / s) * LOGP_LN2;
      if (a.tokens) put_logp<T>(a, row, found, none);
    }
    if constexpr (TOP) {
      // the top-th largest of the groups' keys (0: there are not so many); above it lie at least as many of the row's
      const u64 k = keys[lane_id()], is = ballot(rank[lane_id()] == wanted - 1 && k != 0);
      const u64 least = is ? lane_key(k, (u32)__builtin_ctzll(is)) : 0;
      const float low = least ? out_of_order((u32)(least >> 32)) : LOGP_NEG_INF;
      auto list_it = [&](float x, u32 place) {
        const u64 key = key_of(x, first + place);
        if (key >= least) {
          const u32 to = atomicAdd(&listed, 1u);
          if (to < LOGP_ROOM) list[to] = key;
        }
      };
      if (has && key_of(best, first + at) >= least) {
        r.first(tid, list_it);
        r.last(tid, list_it);
        auto some = [&](const V& v, u32 place) {
          float x[N], most = LOGP_NEG_INF;
#pragma unroll
          for (u32 k = 0; k < N; ++k) { x[k] = (float)v[k]; most = fmaxf(most, x[k]); }
          if (most >= low) {
#pragma unroll
            for (u32 k = 0; k < N; ++k) list_it(x[k], place + k);
          }
        };
        if constexpr (P > 0) {
#pragma unroll
          for (u32 u = 0; u < P; ++u)
            if (tid + u * NT < r.pieces) some(held[u], r.place(tid + u * NT));
        } else {
          u32 i = tid;
          for (; i + (AHEAD - 1) * NT < r.pieces; i += AHEAD * NT) {
#pragma unroll
            for (u32 u = 0; u < AHEAD; ++u) held[u] = r.piece(i + u * NT);
#pragma unroll
            for (u32 u = 0; u < AHEAD; ++u) some(held[u], r.place(i + u * NT));
          }
          for (; i < r.pieces; i += NT) some(r.piece(i), r.place(i));
        }
      }
      __syncthreads();
      const u32 n = listed;
      auto put = [&](u32 rank, u64 key) {
        if (a.parts > 1) a.part_top[b * a.top + rank] = key;
        else put_top(a, row, rank, key, found, none);
      };
      if (a.parts > 1 && tid >= wanted && tid < a.top) a.part_top[b * a.top + tid] = 0;
      if (n <= LOGP_ROOM && s == s) {
        for (u32 c = tid; c < n; c += NT) {
          const u64 key = list[c];
          u32 above = 0;
#pragma unroll 8
          for (u32 j = 0; j < n; ++j) above += list[j] > key;
          if (above < wanted) put(above, key);
        }
      } else {
        u64 last = ~0ull;                                             // (above every key)
        for (u32 k = 0; k < wanted; ++k) {
          u64 next = 0;
          r.template each<NT>(tid, [&](float x, u32 place) {
            const u64 key = key_of(x, first + place);
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

// Rows in parts: their sums brought to the row's maximum, and the top of the parts' tops.
#define LOGP_PARTS 16u
template <class T>
__global__ __launch_bounds__(256) void k_logp_join(const LogpArgs a) {
  __shared__ u64 list[LOGP_PARTS * G10_LOG_PROBS_TOP];
  for (u64 row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const Part* p = a.part + row * a.parts;
    float top = LOGP_NEG_INF, top2 = -LOGP_FAR;
    for (u32 i = 0; i < a.parts; ++i) { top = fmaxf(top, p[i].top); top2 = fmaxf(top2, p[i].top2); }
    Found found = {top, top2, 0.0f};
    const bool far = is_far(found);
    float s = 0.0f, t = 0.0f;
    for (u32 i = 0; i < a.parts; ++i) {
      const Part q = p[i];
      const float d = q.top == LOGP_NEG_INF ? LOGP_NEG_INF : far ? (q.top - top) * a.scale2 : q.top2 - top2, f = __builtin_amdgcn_exp2f(d);
      s += q.s * f;
      t += logp_times(f, q.t + logp_times(q.s, d));
    }
    const bool none = is_none(found, s);
    found.log = __log2f(s);
    if (threadIdx.x == 0) {
      a.lse[row] = lse_of(a, found, none);
      if (a.entropy) a.entropy[row] = none ? 0.0f : (found.log - t / s) * LOGP_LN2;
      if (a.tokens) put_logp<T>(a, row, found, none);
    }
    const u32 n = a.parts * a.top;
    for (u32 i = threadIdx.x; i < n; i += 256) list[i] = a.part_top[row * n + i];
    __syncthreads();
    for (u32 i = threadIdx.x; i < n; i += 256) {
      const u64 key = list[i];
      u32 above = 0;
#pragma unroll 8
      for (u32 j = 0; j < n; ++j) above += list[j] > key;
      if (above < a.top && key) put_top(a, row, above, key, found, none);
    }
    __syncthreads();
  }
}

// How far from zero lse may lie for p to be taken from it.  Its roundings are in every p: at 64 up to 6e-6 of p, a hundred half steps of 32 bits (the
// roundings of a product with `scale` are as large); at 256 3e-5, an eighth of half a step of 16 bits of 5 exponent bits.
template <class T> struct Near { static constexpr float LSE = sizeof(T) == 4 ? 64.0f : 256.0f; };

// A whole row's largest logit and the logarithm of its sum once more, in all threads (rows without NaN and +infinity).
template <class T>
__device__ __forceinline__ Found again(const LogpArgs& a, u64 row) {
  constexpr u32 NT = 256, W = NT / 64, N = Row<T>::N;
  __shared__ float room[2][W];
  const Row<T> r((const T*)a.logits + (int64_t)row * a.ls, a.vocab);
  float m = LOGP_NEG_INF, s = 0.0f;
  auto take = [&](const float* x, u32 n) {
    float top = x[0];
#pragma unroll
    for (u32 k = 1; k < n; ++k) top = fmaxf(top, x[k]);
    if (top > m) {
      s *= m == LOGP_NEG_INF ? 0.0f : __builtin_amdgcn_exp2f((m - top) * a.scale2);
      m = top;
    }
    const float from = m == LOGP_NEG_INF ? 0.0f : m;
#pragma unroll
    for (u32 k = 0; k < n; ++k) s += __builtin_amdgcn_exp2f((x[k] - from) * a.scale2);
  };
  auto one = [&](float x, u32) { take(&x, 1); };
  r.first(threadIdx.x, one);
  r.last(threadIdx.x, one);
#pragma unroll 4
  for (u32 i = threadIdx.x; i < r.pieces; i += NT) {
    const typename Row<T>::V v = r.piece(i);
    float x[N];
#pragma unroll
    for (u32 k = 0; k < N; ++k) x[k] = (float)v[k];
    take(x, N);
  }
  const float wm = wave_max(m);
  if (lane_id() == 0) room[0][wave_id()] = wm;
  __syncthreads();
  float top = room[0][0];
#pragma unroll
  for (u32 w = 1; w < W; ++w) top = fmaxf(top, room[0][w]);
  s = wave_add(m == LOGP_NEG_INF ? 0.0f : s * __builtin_amdgcn_exp2f((m - top) * a.scale2));
  if (lane_id() == 0) room[1][wave_id()] = s;
  __syncthreads();
  s = room[1][0];
#pragma unroll
  for (u32 w = 1; w < W; ++w) s += room[1][w];
  __syncthreads();                                                    // (a next row's go where these lie)
  return {top, 0.0f, __log2f(s)};
}

// The gradient of a row: p (c0 + c1 log p), c0 = - (dlogp + dentropy entropy), c1 = - dentropy, and dlogp at the token.  Few rows are cut into parts.
// log p = scale (x - from) - off: from lse, or where that lies too far from zero from the row's largest logit and its sum, for which the row is read once more
// (32768 x 32000 in bf16: 0.80 ms, 0.87 where all rows are such).  Each of a row's parts reads it, or with `whole` the first part does the row's work alone.
template <class T>
__global__ __launch_bounds__(256) void k_logp_back(const LogpArgs a, u32 vec, u32 whole) {
  constexpr u32 NT = 256, N = Row<T>::N;
  typedef typename Row<T>::V V;
  for (u64 b = blockIdx.x; b < (u64)a.rows * a.parts; b += gridDim.x) {
    const u64 row = b % a.rows;                                       // (all rows' first parts go ahead, and are on all XCDs)
    const u32 first = (u32)(b / a.rows) * a.each;
    u32 count = a.vocab - first < a.each ? a.vocab - first : a.each;
    const float lse = a.lse[row];
    float dl = a.tokens && a.dlogp ? a.dlogp[row] : 0.0f;
    const float de = a.dentropy ? a.dentropy[row] : 0.0f;
    int64_t t = a.tokens ? ((const int64_t*)a.tokens)[row] : -1;
    if (a.tokens) {
      if (t == a.ignore) { dl = 0.0f; t = -1; }
      else if (t < 0 || t >= (int64_t)a.vocab) { dl = dl != 0.0f ? __builtin_nanf("") : 0.0f; t = -1; }
    }
    const float c0 = -(dl + (de != 0.0f ? de * a.entropy[row] : 0.0f)) * a.scale, c1 = -de * a.scale, hit = dl * a.scale;
    bool zero = c0 == 0.0f && c1 == 0.0f && hit == 0.0f;              // (nothing of the row counts: it is not read)
    float from = 0.0f, off = lse;
    if (!zero && fabsf(lse) >= Near<T>::LSE) {
      if (whole) {
        if (first) continue;
        count = a.vocab;
      }
      const Found found = again<T>(a, row);
      zero = found.top == LOGP_NEG_INF;                               // (a row without any probability)
      from = found.top;
      off = found.log * LOGP_LN2;
    }
    t -= first;                                                       // (its place in this part, or outside it)
    const Row<T> r((const T*)a.logits + (int64_t)row * a.ls + first, count);
    T* out = (T*)a.dlogits + (int64_t)row * a.ds + first;
    auto grad = [&](float x, u32 place) {
      const float lp = __builtin_fmaf(x - from, a.scale, -off);       // -infinity where there is no probability
      const float p = __builtin_amdgcn_exp2f(lp * LOGP_LOG2E);
      float g = p * c0;
      if (a.dentropy) g += logp_times(p, lp) * c1;
      return (int64_t)place == t ? g + hit : g;
    };
    if (zero) {
      auto nothing = [&](u32 at) { out[at] = (T)0.0f; };
      const u32 head = (u32)((0 - (uintptr_t)out) & 15) / (u32)sizeof(T), h = head < count ? head : count, pieces = (count - h) / N;
      const V z = {};
      if (threadIdx.x < h) nothing(threadIdx.x);
      for (u32 i = threadIdx.x; i < pieces; i += NT) __builtin_nontemporal_store(z, (V*)(out + h + (u64)i * N));
      const u32 at = h + pieces * N + threadIdx.x;
      if (threadIdx.x < N && at < count) nothing(at);
    } else if (vec) {
      auto one = [&](float x, u32 place) { out[place] = (T)grad(x, place); };
      r.first(threadIdx.x, one);
      r.last(threadIdx.x, one);
      for (u32 i = threadIdx.x; i < r.pieces; i += NT) {
        const V v = r.piece(i);
        V w;
#pragma unroll
        for (u32 k = 0; k < N; ++k) w[k] = (T)grad((float)v[k], r.place(i) + k);
        __builtin_nontemporal_store(w, (V*)(out + r.place(i)));
      }
    } else {
      for (u32 i = threadIdx.x; i < count; i += NT) out[i] = (T)grad((float)r.p[i], i);
    }
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------------------------------
static int logp_args(const g10_log_probs_args* g, bool back, LogpArgs& a) {
  if (!g) return G10_EINVAL;
  if (g->type > G10_BF16 || !(g->scale > 0.0f) || !(g->scale <= LOGP_SCALE) || !g->vocab || g->vocab >= 0x80000000u || g->rows >= 0x80000000u) return G10_EINVAL;
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
  a.parts = 1; a.each = a.vocab;
  // Few long rows are cut into parts of 16384 logits or more, and joined: a unit's issue is what a row waits for (200000 in 16 bits, entropy 15 us, so 9; a top
  // of 20 24, so 15).
  if (!back && a.rows && a.rows <= 64 && a.vocab >= 65536) {
    const u32 most = a.vocab / 16384, room = 512 / a.rows;
    a.parts = most < LOGP_PARTS ? most : LOGP_PARTS;
    a.parts = a.parts < room ? a.parts : room;
    a.each = ((a.vocab + a.parts - 1) / a.parts + 63) / 64 * 64;
    a.parts = (a.vocab + a.each - 1) / a.each;
  }
  if (back && a.rows && a.rows < 2048 && a.vocab > 8192) {             // (2 rows of 194004: 32 us on a unit each, so 4)
    a.each = 8192;
    a.parts = (a.vocab + a.each - 1) / a.each;
  }
  return G10_OK;
}

// Few rows take 1024 threads each, which for a row's top keep it in registers (8 rows of 32000 with a top of 20: 8.6 us; read a second time where
// needed, 21).  Many rows take 256 and read again the eighth or so of a row in which candidates lie: more workgroups to a unit are worth
// more than the registers (1500 rows of 30522 in 32 bits, a top of 5: 43 us, in registers of 512 threads 56).  Rows of up to 512 pieces take a
// wavefront.
template <class T, int WHAT>
static void logp_rows(const LogpArgs& a, hipStream_t s) {
  const u64 rows = (u64)a.rows * a.parts;
  const u32 grid = (u32)(rows < 1u << 16 ? rows : 1u << 16), pieces = a.each / (16 / (u32)sizeof(T));
  if (rows <= 512 && pieces > 512) {
    if (WHAT == LOGP_TOP && pieces <= 4096) k_logp<T, 1024, WHAT == LOGP_TOP ? 4 : 0, WHAT><<<grid, 1024, 0, s>>>(a);
    else if (WHAT == LOGP_TOP && pieces <= 16384) k_logp<T, 1024, WHAT == LOGP_TOP ? 16 : 0, WHAT><<<grid, 1024, 0, s>>>(a);
    else k_logp<T, 1024, 0, WHAT><<<grid, 1024, 0, s>>>(a);
  } else if (pieces > 512) {
    k_logp<T, 256, 0, WHAT><<<grid, 256, 0, s>>>(a);
  } else {
    k_logp<T, 64, 0, WHAT><<<grid, 64, 0, s>>>(a);
  }
}
template <class T>
static void logp_launch(const LogpArgs& a, hipStream_t s) {
  if (a.top) logp_rows<T, LOGP_TOP>(a, s);
  else if (a.entropy) logp_rows<T, LOGP_ENTROPY>(a, s);
  else logp_rows<T, LOGP_LSE>(a, s);
  if (a.parts > 1) k_logp_join<T><<<a.rows, 256, 0, s>>>(a);
}

static u64 logp_room(const LogpArgs& a) { return a.parts > 1 ? (u64)a.rows * a.parts * (sizeof(Part) + a.top * 8) : 0; }

extern "C" int g10_log_probs_workspace(const g10_log_probs_args* g, uint64_t* bytes) {
  if (!bytes) return G10_EINVAL;
  LogpArgs a;
  G10_TRY(logp_args(g, false, a));
  *bytes = logp_room(a);
  return G10_OK;
}

extern "C" int g10_log_probs(const g10_log_probs_args* g, void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  LogpArgs a;
  G10_TRY(logp_args(g, false, a));
  if (!a.rows) return G10_OK;
  if (const u64 n = logp_room(a)) {
    if (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < n) return G10_EINVAL;
    a.part = (Part*)workspace;
    a.part_top = (u64*)(a.part + (u64)a.rows * a.parts);
  }
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
  const u64 groups = (u64)a.rows * a.parts;
  const u32 grid = (u32)(groups < 1u << 16 ? groups : 1u << 16), e = g->type == G10_F32 ? 4 : 2;
  // (rows of both tensors lie alike within 16 bytes)
  const u32 vec = !(((uintptr_t)g->logits ^ (uintptr_t)g->dlogits) & 15) && ((g->logits_stride - g->dlogits_stride) * (int64_t)e) % 16 == 0;
  // Written over the logits a row that is summed again stays with one workgroup: a part would read what another has written.  So it does where there are
  // workgroups enough (all rows such, read by each part and by one: 2 x 194004 18 us and 49, 32 x 100000 19 and 28, 64 x 200000 85 and 55, 2047 x 32000 113 and 63).
  const u32 whole = a.parts > 1 && (g->logits == g->dlogits || groups > 1024);
  if (g->type == G10_F32) k_logp_back<float><<<grid, 256, 0, s>>>(a, vec, whole);
  else if (g->type == G10_F16) k_logp_back<_Float16><<<grid, 256, 0, s>>>(a, vec, whole);
  else k_logp_back<__bf16><<<grid, 256, 0, s>>>(a, vec, whole);
  G10_HIP(hipGetLastError());
  return G10_OK;
}
