// What the attention kernels share: which keys a query sees, tiles of keys or queries in LDS, fragments
// of the matrix instructions.
#pragma once

#include <math.h>

#include "g10_internal.h"
#include "g10_ops.h"

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef u32 u32x2 __attribute__((ext_vector_type(2)));
typedef u32 u32x4 __attribute__((ext_vector_type(4)));

template <class T> struct Vec;
template <> struct Vec<__bf16> {
  typedef __bf16 x8 __attribute__((ext_vector_type(8)));
  typedef __bf16 x4 __attribute__((ext_vector_type(4)));
  typedef __bf16 x2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ x4 read_tr(u32 at) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) x4*)(uintptr_t)at);
  }
};
template <> struct Vec<_Float16> {
  typedef _Float16 x8 __attribute__((ext_vector_type(8)));
  typedef _Float16 x4 __attribute__((ext_vector_type(4)));
  typedef _Float16 x2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ x4 read_tr(u32 at) {
    typedef __fp16 h4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(x4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) h4*)(uintptr_t)at));
  }
};

// f(0), f(1), ... f(N - 1) with constant arguments, whatever the size of what f does (the compiler stops unrolling long loops).
template <int N> struct Const { static constexpr int value = N; };
template <int I, int N, class F>
__device__ __forceinline__ void each_of(F&& f) {
  if constexpr (I < N) {
    f(Const<I>{});
    each_of<I + 1, N>(f);
  }
}

struct Cut { u32 b, hk, kt, more; };   // backward: a tile of keys that begins in a share and goes on in `more` others

struct AttnArgs {
  const void *q, *k, *v;
  void *o, *dq, *dk, *dv;
  const void* d_o;
  float* lse;
  const float* delta;              // backward: - sum of do * o per query
  const float* lse2;               // backward: lse in powers of two, less the lift of P
  const u32* amax;                 // backward: bits of the largest |do| of each wavefront of k_attn_dq
  float *part, *part_ml;           // split over the keys: unfinished outputs and their maxima and sums; how many to a row.  Backward: unfinished dv and dk
  u32* part_n;
  Cut* cuts;                       // backward: a share's
  int64_t qs[3], ks[3], vs[3], os[3], dos[3], dqs[3], dks[3], dvs[3];   // batch, token, head
  const int *q_start, *k_start, *k_len;
  u32 batch, heads, kv_heads, group, dim;
  u32 seq_q, seq_k, max_q, max_k;
  u32 causal, window, sinks;
  u32 tiles;                       // of queries (or of keys) per sequence and head in the grid
  u32 splits;                      // forward: pieces of a block that there is room for
  u32 shares;                      // that the work is cut into; backward: 0: it is not
  u32 q_tiles;                     // backward: of queries per sequence and head in k_attn_dq's grid
  u32 work;                        // workgroups of the grid with work on sequences; the ones behind them clear rows of none
  float scale, scale2;             // scale2 = scale * log2(e)
};

// One sequence's place.  Numbers of a packed batch that point outside the tensors are moved to their border.
struct Seq {
  int64_t q0, k0;                  // first row in the tensors, in rows behind the batch's own
  int nq, nk;
};

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

__device__ __forceinline__ Seq seq_of(const AttnArgs& a, u32 b) {
  Seq s;
  if (a.q_start) {
    const int q0 = clampi(a.q_start[b], 0, (int)a.seq_q), q1 = clampi(a.q_start[b + 1], q0, (int)a.seq_q);
    const int k0 = clampi(a.k_start[b], 0, (int)a.seq_k), k1 = clampi(a.k_start[b + 1], k0, (int)a.seq_k);
    s.q0 = q0; s.k0 = k0; s.nq = q1 - q0; s.nk = k1 - k0;
  } else {
    s.q0 = s.k0 = 0; s.nq = (int)a.seq_q;
    s.nk = a.k_len ? clampi(a.k_len[b], 0, (int)a.seq_k) : (int)a.seq_k;
  }
  return s;
}
__device__ __forceinline__ int64_t batch_off(const AttnArgs& a, u32 b, int64_t stride) { return a.q_start ? 0 : (int64_t)b * stride; }
// the place of (sequence, head, first query) in lse and delta
__device__ __forceinline__ int64_t row_off(const AttnArgs& a, u32 b, u32 h, const Seq& s) {
  return a.q_start ? (int64_t)h * a.seq_q + s.q0 : ((int64_t)b * a.heads + h) * a.seq_q;
}

// The keys that the query at position p sees: lo .. lo + span - 1, and those below `first`.
struct Seen {
  int lo, first;
  u32 span;
  __device__ __forceinline__ bool key(int j) const { return (u32)(j - lo) < span || j < first; }
};
__device__ __forceinline__ Seen keys_of(const AttnArgs& a, int p, int nk) {
  const int w = (int)a.window, last = nk - 1;
  int hi = last;
  if (a.causal) hi = p < last ? p : last;
  else if (w && p < last - w + 1) hi = p + w - 1;
  Seen s;
  s.lo = w && p - w + 1 > 0 ? p - w + 1 : 0;
  s.span = hi >= s.lo ? (u32)(hi - s.lo + 1) : 0u;
  s.first = 0;
  if (w) {
    const int end = a.causal ? (p < last ? p : last) + 1 : nk;
    s.first = (int)a.sinks < end ? (int)a.sinks : end;
  }
  return s;
}
// Whether all positions p0..p1 see all keys j0..j1.
__device__ __forceinline__ bool all_see(const AttnArgs& a, int p0, int p1, int j0, int j1, int nk) {
  const int w = (int)a.window;
  if (j1 >= nk || (a.causal && j1 > p0)) return false;
  return w == 0 || j1 < (int)a.sinks || (p1 - j0 < w && (a.causal || j1 - p0 < w));
}

// The keys that any of the positions p0..p1 sees, as tiles of TILE keys: first `head` tiles from 0 on (the sinks), then
// the tiles lo.. of the window, `count` in all.
struct Tiles {
  int head, lo, count;
  __device__ __forceinline__ int at(int i) const { return i < head ? i : lo + i - head; }
};
template <int TILE>
__device__ __forceinline__ Tiles key_tiles(const AttnArgs& a, int p0, int p1, int nk) {
  const int w = (int)a.window;
  int64_t hi = (int64_t)nk - 1;
  if (a.causal) hi = p1 < hi ? p1 : hi;
  else if (w && (int64_t)p1 + w - 1 < hi) hi = (int64_t)p1 + w - 1;
  const int lo = w && p0 - w + 1 > 0 ? p0 - w + 1 : 0;
  int first = (int)a.sinks < nk ? (int)a.sinks : nk;                 // sinks that any of them sees
  if (a.causal && first > p1 + 1) first = p1 + 1 > 0 ? p1 + 1 : 0;
  if (!w) first = 0;
  Tiles t;
  t.head = (first + TILE - 1) / TILE;
  if (hi < lo) { t.lo = 0; t.count = t.head; return t; }
  t.lo = lo / TILE;
  if (t.head > t.lo) t.head = t.lo;
  t.count = t.head + (int)(hi / TILE) - t.lo + 1;
  return t;
}

// Those of a workgroup's tiles in which the positions p0..p1 (none: p1 < p0) among its own see any key: 0..head-1 and from..end-1.
struct Runs { int head, from, end; };
template <int TILE>
__device__ __forceinline__ Runs runs_of(const AttnArgs& a, const Tiles& t, int p0, int p1, int nk) {
  Runs r = {0, t.count, t.count};
  if (p1 < p0) return r;
  const Tiles mine = key_tiles<TILE>(a, p0, p1, nk);
  const int rest = mine.count - mine.head;
  r.head = mine.head;                                                // (more than t.head only where t's tiles are all in a row)
  if (rest > 0) { r.from = mine.lo - t.lo + t.head; r.end = r.from + rest; }
  if (r.from == r.head) r.head = r.from = 0;
  return r;
}

// The queries (indices 0..nq-1) that see any key of j0..j1: lo..hi (empty: hi < lo).
__device__ __forceinline__ void query_range(const AttnArgs& a, int j0, int j1, const Seq& s, int& lo, int& hi) {
  const int off = s.nk - s.nq, w = (int)a.window;                    // p = i + off
  lo = 0; hi = s.nq - 1;
  if (a.causal && j0 - off > lo) lo = j0 - off;
  if (w && !(j0 < (int)a.sinks)) {
    if (!a.causal && j0 - w + 1 - off > lo) lo = j0 - w + 1 - off;
    if ((int64_t)j1 + w - 1 - off < hi) hi = j1 + w - 1 - off;
  }
}
// The queries that see all of them.
__device__ __forceinline__ void full_range(const AttnArgs& a, int j0, int j1, const Seq& s, int& lo, int& hi) {
  const int off = s.nk - s.nq, w = (int)a.window;
  lo = 0; hi = j1 < s.nk ? s.nq - 1 : -1;
  if (a.causal && j1 - off > lo) lo = j1 - off;
  if (w && j1 >= (int)a.sinks) {
    if (!a.causal && j1 - w + 1 - off > lo) lo = j1 - w + 1 - off;
    if ((int64_t)j0 + w - 1 - off < hi) hi = j0 + w - 1 - off;
  }
}

// Rows of a sequence that nobody sees: lo..hi-1.  Whatever they hold, nothing comes of it: a probability of 0 times NaN would be NaN, so a tile
// holds one of its other rows in their place.
struct Unseen { int lo, hi; };
// Keys between the sinks and the first query's window.
__device__ __forceinline__ Unseen unseen_keys(const AttnArgs& a, const Seq& s) {
  const int64_t first = (int64_t)s.nk - s.nq - a.window + 1;
  Unseen u;
  u.hi = a.window && first > 0 ? (int)first : 0;
  u.lo = (int)a.sinks < u.hi ? (int)a.sinks : u.hi;
  return u;
}
// Queries before the first key (s.nk > 0).
__device__ __forceinline__ Unseen unseen_queries(const AttnArgs& a, const Seq& s) {
  int64_t before = (int64_t)s.nq - s.nk;
  if (!a.causal) before = a.window && !a.sinks ? before - a.window + 1 : 0;
  return Unseen{0, before > 0 ? (int)before : 0};
}

// ---------------------------------------------------------------------------------------------------------------------
// Tiles in LDS.  A row holds DP values (DP * 2 bytes), in pieces of 16 bytes; piece c of row r lies at place c ^ swz(r), so that
// the reads below take each of the 64 banks once a cycle: a fragment read takes one piece of 16 rows running (their places
// in a line of 256 bytes all differ), a transposing read takes four neighbouring pieces of 4 rows running, 64 bytes of each.
// ---------------------------------------------------------------------------------------------------------------------
template <int DP>
__device__ __forceinline__ int swz(int r) {
  return DP == 64 ? ((r & 2) << 1) | ((r >> 2) & 3) : ((r & 3) << 2) | ((r >> 2) & 3);
}

// 64 pieces straight from memory to LDS, lane i's to the place i behind lds (which is the same in every lane).
// The address is that of the lane's piece: base (the same in every lane) + off bytes.
// The instruction has no output register and its address is read when it is issued; who reads the tile waits for it first
// (loads_done) and then meets the others at a barrier.  m0 is not named as written: the compiler reserves it (and warns where a list names it), keeps no
// value there and sets it right before an instruction of its own that reads it, of which these kernels have none.
__device__ __forceinline__ void load_piece(const void* base, u32 off, u32 lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void loads_done() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0f70);                              // vmcnt 0 (as a builtin: the compiler then knows its own loads done too)
  asm volatile("" ::: "memory");
}
// All but the wavefront's last N of them.
template <int N>
__device__ __forceinline__ void loads_done_but() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | ((N >> 4) << 14));
  asm volatile("" ::: "memory");
}
// 64 words, lane i's from its own address to the place i behind lds.
__device__ __forceinline__ void load_words(const void* p, u32 lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(p) : "memory");
}
__device__ __forceinline__ u32 lds_addr(const void* p) { return (u32)(uintptr_t)(__attribute__((address_space(3))) const void*)p; }

// What row r of a tile is taken from, of n rows in the sequence and those unseen, all counted from the tile's first row; some row of the tile is seen.
__device__ __forceinline__ int row_for(int r, int n, int lo, int hi) {
  r = r < n ? r : n - 1;
  return r < lo || r >= hi ? r : lo > 0 ? lo - 1 : hi;
}

// ROWS rows by NT threads (t = 0..NT-1) from row `row0` of a sequence of n > 0 rows; rows past its end repeat the last one
// (no query sees them), pieces past the head's values repeat the first (they meet zeros, or go nowhere).
template <int DP, int ROWS, int NT>
struct Stage {
  static constexpr int CPR = DP / 8, IT = ROWS * CPR / NT, STEP = NT / CPR;       // rows of a round
  static constexpr bool EVEN = STEP % 16 == 0;                                    // every round's pieces lie alike
  static_assert(ROWS * CPR % NT == 0 && NT % CPR == 0, "whole rounds of whole rows");
  u32 off[EVEN ? 1 : IT];
  int row;
  __device__ __forceinline__ void init(u32 t, u32 dim, int64_t stride) {
    row = (int)t / CPR;
#pragma unroll
    for (int i = 0; i < (EVEN ? 1 : IT); ++i) {
      const int r = i * STEP + row;
      int c = ((int)t % CPR) ^ swz<DP>(r);
      if (c >= (int)(dim / 8)) c = 0;
      off[i] = (u32)(r * (int)stride + c * 8) * 2;
    }
  }
  // lds: LDS address of the tile + this wavefront's first piece (wave * 1024)
  __device__ __forceinline__ void load(const void* seq_base, int64_t stride, int row0, int n, const Unseen& u, u32 lds) const {
    const char* base = (const char*)seq_base + (int64_t)row0 * stride * 2;
    if (row0 + ROWS <= n && row0 >= u.hi) {
#pragma unroll
      for (int i = 0; i < IT; ++i) {
        if constexpr (EVEN) load_piece(base + (int64_t)(i * STEP) * stride * 2, off[0], lds + (u32)(i * NT * 16));
        else load_piece(base, off[i], lds + (u32)(i * NT * 16));
      }
    } else {
#pragma unroll
      for (int i = 0; i < IT; ++i) {
        const int r = i * STEP + row, over = r - row_for(r, n - row0, u.lo - row0, u.hi - row0);
        const u32 at = EVEN ? off[0] + (u32)(i * STEP * (int)stride) * 2 : off[EVEN ? 0 : i];
        load_piece(base, at - (u32)(over * (int)stride) * 2, lds + (u32)(i * NT * 16));
      }
    }
  }
};

// The same for a walk over tiles one behind the other, with nothing to multiply on the way: `at` is the next tile's place.
template <int DP, int ROWS, int NT>
struct Walk {
  Stage<DP, ROWS, NT> st;
  const char* at;
  int64_t step;                    // bytes of a round's rows
  static_assert(Stage<DP, ROWS, NT>::EVEN, "rounds of 16 rows");
  __device__ __forceinline__ void init(u32 t, u32 dim, int64_t stride) { st.init(t, dim, stride); step = (int64_t)st.STEP * stride * 2; }
  __device__ __forceinline__ void from(const void* seq_base, int64_t stride, int row0) { at = (const char*)seq_base + (int64_t)row0 * stride * 2; }
  __device__ __forceinline__ void load(int row0, int n, const Unseen& u, int64_t stride, u32 lds) {
    if (row0 + ROWS <= n && row0 >= u.hi) {
#pragma unroll
      for (int i = 0; i < st.IT; ++i) { load_piece(at, st.off[0], lds + (u32)(i * NT * 16)); at += step; }
    } else {
#pragma unroll
      for (int i = 0; i < st.IT; ++i) {
        const int r = i * st.STEP + st.row, over = r - row_for(r, n - row0, u.lo - row0, u.hi - row0);
        load_piece(at, st.off[0] + (u32)((i * st.STEP - over) * (int)stride) * 2, lds + (u32)(i * NT * 16));
      }
      at += st.IT * step;
    }
  }
};

// LDS addresses (of tiles that begin at a multiple of 256 bytes) as the places' exclusive or makes them: a base for all
// fragments of a tile, and one operation for each.
//   fragment of rows r0..r0+31, values 16 ks..: lane l holds row l % 32, values 16 ks + 8 (l / 32) + 0..7
template <int DP>
__device__ __forceinline__ u32 rows_base(u32 tile) {
  const u32 l = lane_id();
  return tile + (l & 31) * (DP * 2) + (((l >> 5) ^ (u32)swz<DP>((int)(l & 15))) << 4);
}
template <class T, int DP>
__device__ __forceinline__ typename Vec<T>::x8 frag_rows(u32 base, int r0, int ks) {
  typedef typename Vec<T>::x8 x8;
  return *(__attribute__((address_space(3))) const x8*)(uintptr_t)((base ^ (u32)(ks << 5)) + (u32)(r0 * DP * 2));
}
//   fragment of the transposed tile: lane l holds value 32 db + l % 32 of the rows k0 + 4 (l / 32) + 0..3 and the same + 8: the
//   order of rows in which the results of a product lie (one register group each), so that these feed the next product as they are
template <int DP>
__device__ __forceinline__ u32 cols_base(u32 tile) {
  const u32 l = lane_id(), row = 4 * (l >> 5) + ((l & 15) >> 2), c = 2 * ((l >> 4) & 1) + ((l & 3) >> 1);
  return tile + row * (DP * 2) + ((c ^ (u32)swz<DP>((int)row)) << 4) + (l & 1) * 8;
}
template <class T, int DP>
__device__ __forceinline__ typename Vec<T>::x8 frag_tr(u32 base, int k0, int db) {
  const u32 at = base ^ (u32)(db << 6);
  const typename Vec<T>::x4 a = Vec<T>::read_tr(at + (u32)(k0 * DP * 2)), b = Vec<T>::read_tr((at ^ 32) + (u32)((k0 + 8) * DP * 2));
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
// The row of a result's register r (0..15) in lane l.
__device__ __forceinline__ int res_row(int r) { return 8 * (r >> 2) + 4 * (int)(lane_id() >> 5) + (r & 3); }

// Fragments of 32 rows straight from memory (rows past `last` repeat it, values past dim are zeros).
template <class T, int DP>
__device__ __forceinline__ void frags_global(typename Vec<T>::x8 (&f)[DP / 16], const T* base, int64_t stride, int row, int last, u32 dim) {
  const int l = (int)lane_id();
  const T* p = base + (int64_t)(row < last ? row : last) * stride;
#pragma unroll
  for (int ks = 0; ks < DP / 16; ++ks) {
    const u32 d = 16 * ks + 8 * (l >> 5);
    typename Vec<T>::x8 z = {};
    f[ks] = d < dim ? *(const typename Vec<T>::x8*)(p + d) : z;
  }
}

// What the two halves of a wavefront hold of one row, joined.
__device__ __forceinline__ float both_max(float x) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float both_sum(float x) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// A product that is 0 where p is, whatever x is (v_mul_legacy_f32, which the compiler knows by this name only).
extern "C" __device__ float times(float p, float x) __asm("llvm.amdgcn.fmul.legacy");
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

template <class T>
__device__ __forceinline__ typename Vec<T>::x8 pack8(const f32x16& x, int s) {
  typename Vec<T>::x8 r;
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    const f32x2 two = {x[8 * s + j], x[8 * s + j + 1]};
    const typename Vec<T>::x2 p = __builtin_convertvector(two, typename Vec<T>::x2);
    r[j] = p[0]; r[j + 1] = p[1];
  }
  return r;
}

// Products in groups of four with the fragments of the next group on their way from LDS.  The compiler left to itself puts each read right
// before its product and has the wavefront wait for LDS every time; nothing moves over a line drawn by hold().
__device__ __forceinline__ void hold() { __builtin_amdgcn_sched_barrier(0); }

#define G10_NEG_INF (-__builtin_inff())
#define G10_LOG2E 1.4426950408889634f
#define G10_LN2 0.6931471805599453f

// A workgroup's place among units (a sequence's key head) of `per` workgroups each.  Workgroups go round the 8 XCDs by
// their number: a unit's keys and values stay in one L2 where there are enough units for all of them.
__device__ __forceinline__ bool unit_of(u32 units, u32 per, u32& unit, u32& at) {
  const u32 id = blockIdx.x;
  if (units % 8 == 0 || units >= 64) {
    const u32 slot = id / 8;
    unit = id % 8 + 8 * (slot / per);
    at = slot % per;
    return unit < units;
  }
  unit = id / per; at = id % per;
  return unit < units;
}
// The same for blocks of queries: unit, head of its group, block.  Four heads side by side, their last blocks first, which are the longest of
// a causal sequence: the kernel ends with short ones (16 x 2048 tokens of 32 heads, head after head: 719 us, four side by side 686, eight 688).
__device__ __forceinline__ bool block_of(u32 units, u32 group, u32 tiles, u32& unit, u32& head, u32& qt) {
  const bool round = units % 8 == 0 || units >= 64;
  const u32 x = round ? blockIdx.x % 8 : 0u, slot = round ? blockIdx.x / 8 : blockIdx.x;
  const u32 heads = (round ? (units + 7) / 8 : units) * group, four = slot / (4 * tiles), in = slot % (4 * tiles);
  const u32 side = heads - 4 * four < 4 ? heads - 4 * four : 4u, line = 4 * four + in % side;
  unit = round ? x + 8 * (line / group) : line / group;
  head = line % group;
  qt = tiles - 1 - in / side;
  return unit < units;
}
static inline u32 unit_grid(u32 units, u32 per) {
  return units % 8 == 0 || units >= 64 ? 8 * ((units + 7) / 8) * per : units * per;
}

// Rows of a packed tensor that belong to no sequence, as padding behind the last one: below lo and from hi on. Their outputs and gradients are
// zeros: the allocator's memory holds whatever it held. REST workgroups behind the grid's others clear them, so that it takes no
// launch of its own. (Where the starts fall, which they must not, rows between may belong to none as well.)
#define REST 64u
struct Rest { int lo, hi, rows; u32 part; };                         // rows: how many; part: this workgroup's number
__device__ __forceinline__ Rest rest_of(const int* start, u32 batch, u32 n, u32 part) {
  __shared__ u32 tmp[G10_WAVES];
  u32 lo = n, hi = 0;
  for (u32 b = threadIdx.x; b <= batch; b += G10_BLOCK) {
    const u32 x = (u32)clampi(start[b], 0, (int)n);
    lo = min(lo, x);
    hi = max(hi, x);
  }
  lo = n - block_max(n - lo, tmp);
  hi = block_max(hi, tmp);
  return Rest{(int)lo, (int)hi, (int)(lo + n - hi), part};
}
template <class F>
__device__ __forceinline__ void each_rest(const Rest& r, u32 per, F&& f) {   // f(row, 0..per-1)
  const u64 all = (u64)r.rows * per;
  for (u64 e = (u64)r.part * G10_BLOCK + threadIdx.x; e < all; e += (u64)REST * G10_BLOCK) {
    const int row = (int)(e / per);
    f(row < r.lo ? row : r.hi + row - r.lo, (u32)(e % per));
  }
}
template <class T>
__device__ __forceinline__ void clear_rest(const Rest& r, void* p, const int64_t (&st)[3], u32 heads, u32 dim) {
  const u32 pieces = dim / 8;
  each_rest(r, heads * pieces, [&](int row, u32 e) { *(u32x4*)((T*)p + row * st[1] + (int64_t)(e / pieces) * st[2] + e % pieces * 8) = u32x4{}; });
}
// The forward kernels' outputs.
template <class T>
__device__ __forceinline__ void clear_outputs(const AttnArgs& a) {
  const Rest r = rest_of(a.q_start, a.batch, a.seq_q, blockIdx.x - a.work);
  clear_rest<T>(r, a.o, a.os, a.heads, a.dim);
  each_rest(r, a.heads, [&](int row, u32 h) { a.lse[(int64_t)h * a.seq_q + row] = -__builtin_inff(); });
}
// Tiles (of `per` workgroups each) that a grid holds for every unit, of those wanted. The kernels go on by a.tiles, so any number is right; where only the sum
// of packed sequences' lengths is told, most workgroups of a grid for the longest possible one find nothing to do (forward, 4096 sequences of one token, 32 heads
// on 8: 290 us with the lengths told, else 570 with up to 2^16 workgroups, 3280 with 2^20; 300 of 1000 tokens: 2350, 2430 and 3230). 256 x
// 2048 tokens of 32 heads, whose 2^17 blocks all have work, take 5910 us with 2^16 workgroups and 5980 with one to a block.
#define GRID_MOST (1u << 16)
static inline u32 tiles_in(u32 units, u32 per, u64 tiles) {
  const u32 one = unit_grid(units, per), most = one < GRID_MOST ? GRID_MOST / one : 1;
  return tiles < most ? (u32)tiles : most;
}
static inline u32 with_rest(AttnArgs& a, u32 grid) {
  a.work = grid;
  return a.q_start ? grid + REST : grid;
}

int attn_args(const g10_attention_args* g, bool back, AttnArgs& a);
u32 attn_splits(const AttnArgs& a);
u64 attn_split_bytes(const AttnArgs& a, u32 splits);
int attn_forward_split(AttnArgs a, u32 splits, void* workspace, u32 type, hipStream_t s);
