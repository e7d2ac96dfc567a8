// Rows of a table by token, and the table's gradient.
//
// Both are bound by memory: the lookup reads a row and writes it; the gradient reads every token's row once and writes every row of the
// table once.  For the sums the tokens are sorted by id (a stable radix sort of ids and places, so that a row's tokens come in their
// own order), and the sorted list is cut into pieces of one length: a wavefront takes a piece and 16 bytes a lane of its rows,
// whatever ids the piece holds.  A run of one id inside a piece is a finished row of the table; where a run goes over the ends of
// pieces its parts go to memory in 32 bits and are added in order by a second kernel.  So a frequent token is no one's long row,
// and no sum depends on who comes first.
#include "g10_internal.h"
#include "g10_ops.h"

#include <math.h>

struct EmbedArgs {
  const void *ids, *table, *dout;
  void *out, *dtable;
  int64_t ts, os, ds, gs;
  u32 tokens, vocab, dim, slabs, ids64;
  float scale;
  // backward
  u32 *keys[2], *places[2];        // ids and places of tokens, before and after a pass of the sort
  u32* counts;                     // [tile][digit]
  u32 tiles, tile, bits, passes;   // tiles of `tile` tokens; bits to a pass
  float* parts;                    // [piece][2][part_row]: a run that comes from the piece before, one that goes on
  u32 part_row;
  u32 pieces, per;                 // pieces of `per` tokens
  u32 sum_groups;                  // workgroups that sum; the others clear rows without tokens
};

// N values side by side, at any address of a value: accesses to memory need not be aligned.  A row's last lane takes the row's last N values, whatever
// it shares with the lane before it: both work out and write the same.  (Value by value, a token's loads wait for the one's before: 32768
// tokens of 4095 values 71 and 198 us, so 63 and 159.)  SHORT: rows of fewer than N values, value by value.
template <class T, int N> struct Pack { typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T)))); };
typedef float f4u __attribute__((ext_vector_type(4), aligned(4)));
template <int N, bool SHORT>
__device__ __forceinline__ u32 lane_column(u32 d, u32 dim) { return SHORT || d + N <= dim ? d : dim - N; }
template <class T, int N, bool SHORT>
__device__ __forceinline__ typename Pack<T, N>::type get(const T* p, u32 d, u32 dim) {
  typedef typename Pack<T, N>::type V;
  if constexpr (!SHORT) return *(const V*)(p + d);
  V v = {};
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (d + k < dim) v[k] = p[d + k];
  return v;
}
template <class T, int N, bool SHORT>
__device__ __forceinline__ void put(T* p, u32 d, u32 dim, const typename Pack<T, N>::type& v) {
  typedef typename Pack<T, N>::type V;
  if constexpr (!SHORT) {
    __builtin_nontemporal_store(v, (V*)(p + d));                       // (past the L2)
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (d + k < dim) p[d + k] = v[k];
  }
}

__device__ __forceinline__ int64_t id_at(const EmbedArgs& a, u32 t) {
  return a.ids64 ? ((const int64_t*)a.ids)[t] : (int64_t)((const int*)a.ids)[t];
}

// ---------------------------------------------------------------------------------------------------------------------
// lookup: a wavefront to a token's slab of 64 N values, four tokens at a time
// ---------------------------------------------------------------------------------------------------------------------
template <class T, int N, bool SHORT>
__global__ __launch_bounds__(256) void k_embed(const EmbedArgs a) {
  typedef typename Pack<T, N>::type V;
  const u64 tasks = (u64)((a.tokens + 3) / 4) * a.slabs, step = (u64)gridDim.x * 4;
  for (u64 task = (u64)blockIdx.x * 4 + wave_id(); task < tasks; task += step) {
    const u32 t0 = (u32)(task / a.slabs) * 4, d0 = ((u32)(task % a.slabs) * 64 + lane_id()) * N;
    if (d0 >= a.dim) continue;
    const u32 d = lane_column<N, SHORT>(d0, a.dim);
    V v[4];
    bool fine[4];
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {
      const u32 t = t0 + i < a.tokens ? t0 + i : a.tokens - 1;
      const int64_t id = id_at(a, t);
      fine[i] = id >= 0 && id < (int64_t)a.vocab;
      v[i] = get<T, N, SHORT>((const T*)a.table + (fine[i] ? id : 0) * a.ts, d, a.dim);
    }
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {
      if (t0 + i >= a.tokens) break;
      V w;
#pragma unroll
      for (int k = 0; k < N; ++k) w[k] = (T)(fine[i] ? (float)v[i][k] * a.scale : __builtin_nanf(""));
      put<T, N, SHORT>((T*)a.out + (int64_t)(t0 + i) * a.os, d, a.dim, w);
    }
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// the sort: passes of up to 9 bits, stable, each a count by tile and the move.  Where a tile's digits begin each workgroup works out itself from
// all tiles' counts, of which there are 128 at most: launches that do little wait for one another (32768 tokens, two passes: with running
// sums in launches of their own 31 us, so 21.  Counted for the next pass by the move before it, with atomics in memory: 27, they meet at the
// frequent ids.  All in one workgroup: 85, its unit's accesses to scattered places take as long).
// ---------------------------------------------------------------------------------------------------------------------
#define EMBED_ROUND 1024u          // tokens of a tile that a workgroup takes at a time
#define EMBED_TILES 128u
#define EMBED_DIGITS 512u

// (ids outside the table sort behind all others)
__device__ __forceinline__ u32 key_at(const EmbedArgs& a, u32 t, bool first, const u32* keys) {
  if (!first) return keys[t];
  const int64_t id = id_at(a, t);
  return id >= 0 && id < (int64_t)a.vocab ? (u32)id : a.vocab;
}

template <bool FIRST>
__global__ __launch_bounds__(256) void k_embed_count(const EmbedArgs a, u32 pass, const u32* keys) {
  __shared__ u32 n[EMBED_DIGITS];
  const u32 digits = 1u << a.bits;
  for (u32 d = threadIdx.x; d < digits; d += 256) n[d] = 0;
  __syncthreads();
  const u64 t0 = (u64)blockIdx.x * a.tile, t1 = t0 + a.tile < a.tokens ? t0 + a.tile : a.tokens;
#pragma unroll 4
  for (u64 t = t0 + threadIdx.x; t < t1; t += 256) atomicAdd(&n[(key_at(a, (u32)t, FIRST, keys) >> (pass * a.bits)) & (digits - 1)], 1u);
  __syncthreads();
  for (u32 d = threadIdx.x; d < digits; d += 256) a.counts[(u64)blockIdx.x * digits + d] = n[d];
}

// The lanes that are on and whose lower `bits` bits are this lane's.
__device__ __forceinline__ u64 same_digit(bool on, u32 key, u32 bits) {
  const u64 all = ballot(on);
  u32 lo = (u32)all, hi = (u32)(all >> 32);
  for (u32 b = 0; b < bits; ++b) {
    const u32 mine = (u32)((int)(key << (31 - b)) >> 31);              // all ones where the bit is set
    const u64 m = ballot((int)mine < 0);
    lo &= ~((u32)m ^ mine);
    hi &= ~((u32)(m >> 32) ^ mine);
  }
  return ((u64)hi << 32) | lo;
}

// A wavefront takes 64 tokens running, four times a round; the rank of a token among its digit's is that of the rounds and wavefronts before it and
// of the lanes below it with the same digit.
template <bool FIRST>
__global__ __launch_bounds__(256) void k_embed_move(const EmbedArgs a, u32 pass, const u32* keys, const u32* places, u32* to_keys, u32* to_places) {
  __shared__ u32 seen[4][EMBED_DIGITS], begin[EMBED_DIGITS], sums[4];
  const u32 digits = 1u << a.bits, shift = pass * a.bits, w = wave_id(), l = lane_id();
  const u32* counts = a.counts;
  // where the tile's tokens of each digit begin: behind all of lower digits, and those of earlier tiles.  Two digits to a thread, side by side
  u32 before[2] = {}, all[2] = {};
  const u32 d0 = threadIdx.x * 2;
  if (d0 < digits) {
#pragma unroll 8
    for (u32 t = 0; t < a.tiles; ++t) {
      const uint2 c = *(const uint2*)(counts + (u64)t * digits + d0);
      all[0] += c.x; all[1] += c.y;
      before[0] += t < blockIdx.x ? c.x : 0u; before[1] += t < blockIdx.x ? c.y : 0u;
    }
  }
  const u32 upto = wave_scan_dpp<OpAdd>(all[0] + all[1], 0u);
  if (l == 63) sums[w] = upto;
  __syncthreads();
  if (d0 < digits) {
    u32 at = upto - all[0] - all[1];
#pragma unroll
    for (u32 v = 0; v < 4; ++v) at += v < w ? sums[v] : 0u;
    begin[d0] = at + before[0];
    begin[d0 + 1] = at + all[0] + before[1];
  }
  const u64 end = (u64)blockIdx.x * a.tile + a.tile < a.tokens ? (u64)blockIdx.x * a.tile + a.tile : a.tokens;
  for (u64 round = (u64)blockIdx.x * a.tile; round < end; round += EMBED_ROUND) {
    u32 key[4], rank[4], from[4];
    const u64 t0 = round + w * 256 + l;                                // a wavefront's 256 tokens lie side by side
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {
      const u64 t = t0 + i * 64;
      const u32 r = (u32)(t < end ? t : end - 1);
      key[i] = key_at(a, r, FIRST, keys);
      from[i] = FIRST ? r : places[r];
    }
    for (u32 d = threadIdx.x; d < 4 * EMBED_DIGITS; d += 256) (&seen[0][0])[d] = 0;
    __syncthreads();
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {
      const bool on = t0 + i * 64 < end;
      const u32 d = (key[i] >> shift) & (digits - 1);
      const u64 same = same_digit(on, key[i] >> shift, a.bits);
      const u32 below = (u32)__popcll(same & ((1ull << l) - 1)), before = seen[w][d];
      rank[i] = before + below;
      __builtin_amdgcn_wave_barrier();                                 // (a wavefront's LDS accesses stay in order: all read before one writes)
      if (on && !below) seen[w][d] = before + (u32)__popcll(same);
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    for (u32 d = threadIdx.x; d < digits; d += 256) {                  // where each wavefront's tokens of a digit begin
      u32 at = begin[d];
#pragma unroll
      for (u32 v = 0; v < 4; ++v) { const u32 n = seen[v][d]; seen[v][d] = at; at += n; }
      begin[d] = at;
    }
    __syncthreads();
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {
      if (t0 + i * 64 >= end) continue;
      const u32 at = seen[w][(key[i] >> shift) & (digits - 1)] + rank[i];
      if (at >= a.tokens) continue;                                    // (ids that change while they are sorted)
      to_keys[at] = key[i];
      to_places[at] = from[i];
    }
    __syncthreads();
  }
}

// Up to 4096 tokens: all passes in one workgroup's LDS, 256 tokens running to a wavefront (4 launches less of 4 us each).
#define EMBED_FEW 4096u
__global__ __launch_bounds__(1024) void k_embed_sort(const EmbedArgs a, u32* to_keys, u32* to_places) {
  __shared__ u32 seen[16][EMBED_DIGITS], sums[8], order[2][EMBED_FEW];
  const u32 digits = 1u << a.bits, w = wave_id(), l = lane_id(), t0 = w * 256 + l;
  u32 key[4], place[4], rank[4];
#pragma unroll
  for (u32 i = 0; i < 4; ++i) {
    place[i] = t0 + i * 64;
    key[i] = key_at(a, place[i] < a.tokens ? place[i] : 0, true, nullptr);
  }
  for (u32 pass = 0; pass < a.passes; ++pass) {
    const u32 shift = pass * a.bits;
    for (u32 d = threadIdx.x; d < 16 * EMBED_DIGITS; d += 1024) (&seen[0][0])[d] = 0;
    __syncthreads();
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {
      const bool on = t0 + i * 64 < a.tokens;
      const u32 d = (key[i] >> shift) & (digits - 1);
      const u64 same = same_digit(on, key[i] >> shift, a.bits);
      const u32 below = (u32)__popcll(same & ((1ull << l) - 1)), before = seen[w][d];
      rank[i] = before + below;
      __builtin_amdgcn_wave_barrier();                                 // (a wavefront's LDS accesses stay in order: all read before one writes)
      if (on && !below) seen[w][d] = before + (u32)__popcll(same);
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    const u32 d = threadIdx.x;                                         // where each wavefront's tokens of a digit begin: a thread to a digit
    u32 n[16], all = 0, upto = 0;
    if (d < EMBED_DIGITS) {
#pragma unroll
      for (u32 v = 0; v < 16; ++v) { n[v] = seen[v][d]; all += n[v]; }
      upto = wave_scan_dpp<OpAdd>(all, 0u);
      if (l == 63) sums[w] = upto;
    }
    __syncthreads();
    if (d < EMBED_DIGITS) {
      u32 at = upto - all;
#pragma unroll
      for (u32 v = 0; v < 8; ++v) at += v < w ? sums[v] : 0u;
#pragma unroll
      for (u32 v = 0; v < 16; ++v) { seen[v][d] = at; at += n[v]; }
    }
    __syncthreads();
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {
      if (t0 + i * 64 >= a.tokens) continue;
      const u32 at = seen[w][(key[i] >> shift) & (digits - 1)] + rank[i];
      order[0][at] = key[i];                                           // (below `tokens`: the keys are this workgroup's own)
      order[1][at] = place[i];
    }
    __syncthreads();
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {
      const u32 t = t0 + i * 64 < a.tokens ? t0 + i * 64 : 0;
      key[i] = order[0][t];
      place[i] = order[1][t];
    }
  }
#pragma unroll
  for (u32 i = 0; i < 4; ++i) {
    if (t0 + i * 64 >= a.tokens) continue;
    to_keys[t0 + i * 64] = key[i];
    to_places[t0 + i * 64] = place[i];
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// the sums
// ---------------------------------------------------------------------------------------------------------------------
template <class T, int N, bool SHORT>
__device__ __forceinline__ void write_row(const EmbedArgs& a, u32 v, u32 d, const float (&s)[N]) {
  typedef typename Pack<T, N>::type V;
  V w;
#pragma unroll
  for (int k = 0; k < N; ++k) w[k] = (T)(s[k] * a.scale);
  put<T, N, SHORT>((T*)a.dtable + (int64_t)v * a.gs, d, a.dim, w);
}

// Zeros, by way of the L2.
template <class T, int N, bool SHORT>
__device__ __forceinline__ void put_near(T* p, u32 d, u32 dim) {
  typedef typename Pack<T, N>::type V;
  if constexpr (!SHORT) {
    *(V*)(p + d) = V{};
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (d + k < dim) p[d + k] = (T)0.0f;
  }
}

// The first place in the sorted keys whose key is not below v.
__device__ __forceinline__ u32 first_of(const u32* keys, u32 n, u32 v) {
  u32 lo = 0, hi = n;
  while (lo < hi) {
    const u32 mid = lo + (hi - lo) / 2;
    if (keys[mid] < v) lo = mid + 1; else hi = mid;
  }
  return lo;
}

#define EMBED_CLEAR 8u              // rows of the table that a wavefront looks after (32: 5 tokens, 191 rows of 2141, 16 us for 6)

// NEAR: rows that begin inside a line, so that two of them write it: the ones without tokens, side by side, go by way of the L2 (100000 of 1001 values past
// it 94 us, so 53; rows of whole lines are faster past it).
template <class T, int N, bool SHORT, bool NEAR>
__global__ __launch_bounds__(256) void k_embed_sum(const EmbedArgs a, const u32* keys, const u32* places) {
  typedef typename Pack<T, N>::type V;
  const u32 l = lane_id();
  if (blockIdx.x < a.sum_groups) {
    const u64 tasks = (u64)a.pieces * a.slabs, step = (u64)a.sum_groups * 4;
    for (u64 task = (u64)blockIdx.x * 4 + uniform(wave_id()); task < tasks; task += step) {
      const u32 piece = (u32)(task / a.slabs), d0 = ((u32)(task % a.slabs) * 64 + l) * N;
      const bool on = d0 < a.dim;
      const u32 d = on ? lane_column<N, SHORT>(d0, a.dim) : 0;
      const u32 t0 = piece * a.per, n = a.tokens - t0 < a.per ? a.tokens - t0 : a.per;
      const T* src = (const T*)a.dout;
      // ids and places of the piece, a lane each (a piece has 64 tokens at most)
      const u32 mykey = l < n ? keys[t0 + l] : ~0u, myplace = l < n ? places[t0 + l] : 0;
      const u32 before = t0 ? keys[t0 - 1] : ~0u, behind = t0 + n < a.tokens ? keys[t0 + n] : ~0u;
      float s[N] = {};
      u32 key = (u32)__builtin_amdgcn_readlane((int)mykey, 0);
      bool from = key == before;                                       // the run comes from the piece before
      auto flush = [&](bool on_from, bool goes_on) {
        if (on && key < a.vocab) {
          if (on_from || goes_on) {
            f4u* p = (f4u*)(a.parts + ((u64)piece * 2 + (on_from ? 0 : 1)) * a.part_row + d);
#pragma unroll
            for (int k = 0; k < N; k += 4) p[k / 4] = f4u{s[k], s[k + 1], s[k + 2], s[k + 3]};
          } else {
            write_row<T, N, SHORT>(a, key, d, s);
          }
        }
      };
      for (u32 i = 0; i < n; i += 8) {
        V v[8];
#pragma unroll
        for (u32 j = 0; j < 8; ++j) {
          const u32 place = (u32)__builtin_amdgcn_readlane((int)myplace, (int)(i + j < n ? i + j : n - 1));
          v[j] = get<T, N, SHORT>(src + (int64_t)(place < a.tokens ? place : 0) * a.ds, d, a.dim);
        }
#pragma unroll
        for (u32 j = 0; j < 8; ++j) {
          if (i + j >= n) break;
          const u32 k2 = (u32)__builtin_amdgcn_readlane((int)mykey, (int)(i + j));
          if (k2 != key) {
            flush(from, false);
            key = k2;
            from = false;
#pragma unroll
            for (int k = 0; k < N; ++k) s[k] = 0.0f;
          }
#pragma unroll
          for (int k = 0; k < N; ++k) s[k] += (float)v[j][k];
        }
      }
      flush(from, key == behind);
    }
    return;
  }
  // rows without a token
  const float zero[N] = {};
  const u32 waves = (gridDim.x - a.sum_groups) * 4;
  const u64 rows = ((u64)a.vocab + EMBED_CLEAR - 1) / EMBED_CLEAR;
  for (u64 r = (u64)(blockIdx.x - a.sum_groups) * 4 + uniform(wave_id()); r < rows; r += waves) {
    const u32 v0 = (u32)(r * EMBED_CLEAR), v = v0 + l < a.vocab ? v0 + l : a.vocab;
    const u32 begin = l <= EMBED_CLEAR ? first_of(keys, a.tokens, v) : 0;
    const u32 end = (u32)__shfl_down((int)begin, 1, 64);
    u64 empty = ballot(l < EMBED_CLEAR && v0 + l < a.vocab && begin == end);
    while (empty) {
      const u32 i = (u32)__builtin_ctzll(empty);
      empty &= empty - 1;
      T* row = (T*)a.dtable + (int64_t)(v0 + i) * a.gs;
      for (u32 d = l * N; d < a.dim; d += 64 * N) {
        if constexpr (NEAR) put_near<T, N, SHORT>(row, lane_column<N, SHORT>(d, a.dim), a.dim);
        else write_row<T, N, SHORT>(a, v0 + i, lane_column<N, SHORT>(d, a.dim), zero);
      }
    }
  }
}

// Runs over the ends of pieces: the piece in which such a run begins adds its parts.
template <class T, int N, bool SHORT>
__global__ __launch_bounds__(256) void k_embed_join(const EmbedArgs a, const u32* keys) {
  const u64 tasks = (u64)a.pieces * a.slabs, step = (u64)gridDim.x * 4;
  for (u64 task = (u64)blockIdx.x * 4 + uniform(wave_id()); task < tasks; task += step) {
    const u32 piece = (u32)(task / a.slabs), d0 = ((u32)(task % a.slabs) * 64 + lane_id()) * N;
    const u32 t0 = piece * a.per, t1 = t0 + a.per;
    if (t1 >= a.tokens) continue;
    // lane j looks at the first token of the j-th piece behind this one
    const u64 next = (u64)t1 + (u64)lane_id() * a.per;
    const u32 key = uniform(keys[t1 - 1]), before = t0 ? uniform(keys[t0 - 1]) : ~0u, theirs = next < a.tokens ? keys[next] : ~0u;
    u64 on = ballot(theirs == key);
    if (key >= a.vocab || before == key || !(on & 1)) continue;        // nothing begins here that goes on
    u32 more = on == ~0ull ? 64u : (u32)__builtin_ctzll(~on);          // pieces that the run goes into
    while (more % 64 == 0 && on == ~0ull) {
      const u64 far = (u64)t1 + ((u64)more + lane_id()) * a.per;
      on = ballot(far < a.tokens && keys[far < a.tokens ? far : 0] == key);
      more += on == ~0ull ? 64u : (u32)__builtin_ctzll(~on);
    }
    if (d0 >= a.dim) continue;
    const u32 d = lane_column<N, SHORT>(d0, a.dim);
    const float* p = a.parts + ((u64)piece * 2 + 1) * a.part_row + d;
    float s[N];
#pragma unroll
    for (int k = 0; k < N; ++k) s[k] = p[k];
    p += a.part_row;                                                   // (the next piece's first part)
    for (u32 q = 0; q < more; q += 8) {                                // (past the last one it is read again, and not added)
      float v[8][N];
#pragma unroll
      for (u32 u = 0; u < 8; ++u) {
        const f4u* o = (const f4u*)(p + (u64)(q + u < more ? q + u : more - 1) * 2 * a.part_row);
#pragma unroll
        for (int k = 0; k < N; ++k) v[u][k] = o[k / 4][k % 4];
      }
#pragma unroll
      for (u32 u = 0; u < 8; ++u)
#pragma unroll
        for (int k = 0; k < N; ++k) s[k] += q + u < more ? v[u][k] : 0.0f;
    }
    write_row<T, N, SHORT>(a, key, d, s);
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------------------------------
struct EmbedPlan { bool few, near; u32 grid, clear_groups, join_groups; u64 at_keys[2], at_places[2], at_counts, at_parts, bytes; };

static u64 up256(u64 x) { return (x + 255) & ~(u64)255; }

static int embed_args(const g10_embed_args* g, bool back, EmbedArgs& a, EmbedPlan& p) {
  if (!g) return G10_EINVAL;
  if (g->type > G10_BF16 || g->ids_64 > 1 || !(g->scale == g->scale) || isinf(g->scale)) return G10_EINVAL;
  if (!g->dim || g->dim > 65536 || !g->vocab || g->vocab >= 0x80000000u || g->tokens >= 0x80000000u) return G10_EINVAL;
  const u32 e = g->type == G10_F32 ? 4 : 2;
  const void *src = back ? g->dout : g->table, *dst = back ? g->dtable : g->out;
  const int64_t sd = back ? g->dtable_stride : g->out_stride;
  if (!dst && (back || g->tokens)) return G10_EINVAL;
  if (g->tokens && (!src || !g->ids)) return G10_EINVAL;
  if ((uintptr_t)src % e || (uintptr_t)dst % e || (uintptr_t)g->ids % (g->ids_64 ? 8 : 4)) return G10_EINVAL;
  a = EmbedArgs{};
  a.ids = g->ids; a.table = g->table; a.out = g->out; a.dout = g->dout; a.dtable = g->dtable;
  a.ts = g->table_stride; a.os = g->out_stride; a.ds = g->dout_stride; a.gs = g->dtable_stride;
  a.tokens = g->tokens; a.vocab = g->vocab; a.dim = g->dim; a.scale = g->scale; a.ids64 = g->ids_64;
  const u32 n = 16 / e;
  p = EmbedPlan{};
  p.few = g->dim < n;
  p.near = g->dim % n || ((uintptr_t)dst & 15) || sd % (int64_t)n;
  a.slabs = (g->dim + 64 * n - 1) / (64 * n);
  a.part_row = (g->dim + 7) & ~7u;
  auto groups = [](u64 waves, u32 most) { const u64 n = (waves + 3) / 4; return (u32)(n < most ? n : most); };
  p.grid = groups((u64)((a.tokens + 3) / 4) * a.slabs, 1u << 16);
  if (!back) return G10_OK;
  u32 bits = 1;
  while (bits < 32 && (g->vocab >> bits)) ++bits;                      // ids and one more, for those outside
  a.passes = (bits + 8) / 9;
  a.bits = (bits + a.passes - 1) / a.passes;
  const u32 rounds = (a.tokens + EMBED_ROUND - 1) / EMBED_ROUND;
  a.tile = (rounds + EMBED_TILES - 1) / EMBED_TILES * EMBED_ROUND;
  a.tiles = a.tokens ? (a.tokens + a.tile - 1) / a.tile : 0;
  // pieces of 64 tokens; of 16 where that leaves few wavefronts, each of which waits eight times for its tokens (326 tokens: 15 us for the kernel, so 6; 16384 of
  // 768 values in pieces of 16 63 us altogether for 57, more runs are joined)
  a.per = a.tokens > 64 && (u64)a.tokens / 64 * a.slabs < 512 ? 16 : 64;
  a.pieces = (a.tokens + a.per - 1) / a.per;
  a.sum_groups = groups((u64)a.pieces * a.slabs, 1u << 16);
  p.join_groups = a.sum_groups;
  p.clear_groups = groups(((u64)a.vocab + EMBED_CLEAR - 1) / EMBED_CLEAR, 1u << 14);
  u64 at = 0;
  auto take = [&](u64 bytes) { const u64 here = at; at += up256(bytes); return here; };
  for (int i = 0; i < 2; ++i) { p.at_keys[i] = take((u64)a.tokens * 4); p.at_places[i] = take((u64)a.tokens * 4); }
  p.at_counts = take(((u64)a.tiles << a.bits) * 4);
  p.at_parts = take((u64)a.pieces * 2 * a.part_row * 4);
  p.bytes = at;
  return G10_OK;
}

template <class T, bool SHORT>
static void embed_sums(const EmbedArgs& a, const EmbedPlan& p, int last, hipStream_t s) {
  constexpr int N = 16 / sizeof(T);
  if (SHORT || p.near) k_embed_sum<T, N, SHORT, true><<<a.sum_groups + p.clear_groups, 256, 0, s>>>(a, a.keys[last], a.places[last]);
  else k_embed_sum<T, N, SHORT, SHORT><<<a.sum_groups + p.clear_groups, 256, 0, s>>>(a, a.keys[last], a.places[last]);
  if (a.pieces > 1) k_embed_join<T, N, SHORT><<<p.join_groups, 256, 0, s>>>(a, a.keys[last]);
}

extern "C" int g10_embed(const g10_embed_args* g, void* hip_stream) {
  EmbedArgs a; EmbedPlan p;
  G10_TRY(embed_args(g, false, a, p));
  if (!a.tokens) return G10_OK;
  hipStream_t s = (hipStream_t)hip_stream;
  if (g->type == G10_F32) { if (p.few) k_embed<float, 4, true><<<p.grid, 256, 0, s>>>(a); else k_embed<float, 4, false><<<p.grid, 256, 0, s>>>(a); }
  else if (g->type == G10_F16) { if (p.few) k_embed<_Float16, 8, true><<<p.grid, 256, 0, s>>>(a); else k_embed<_Float16, 8, false><<<p.grid, 256, 0, s>>>(a); }
  else { if (p.few) k_embed<__bf16, 8, true><<<p.grid, 256, 0, s>>>(a); else k_embed<__bf16, 8, false><<<p.grid, 256, 0, s>>>(a); }
  G10_HIP(hipGetLastError());
  return G10_OK;
}

extern "C" int g10_embed_backward_workspace(const g10_embed_args* g, uint64_t* bytes) {
  if (!bytes) return G10_EINVAL;
  EmbedArgs a; EmbedPlan p;
  G10_TRY(embed_args(g, true, a, p));
  *bytes = p.bytes;
  return G10_OK;
}

extern "C" int g10_embed_backward(const g10_embed_args* g, void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  EmbedArgs a; EmbedPlan p;
  G10_TRY(embed_args(g, true, a, p));
  if (p.bytes && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < p.bytes)) return G10_EINVAL;
  hipStream_t s = (hipStream_t)hip_stream;
  char* ws = (char*)workspace;
  for (int i = 0; i < 2; ++i) { a.keys[i] = (u32*)(ws + p.at_keys[i]); a.places[i] = (u32*)(ws + p.at_places[i]); }
  a.counts = (u32*)(ws + p.at_counts);
  a.parts = (float*)(ws + p.at_parts);
  int at = 0;
  if (a.tokens && a.tokens <= EMBED_FEW) k_embed_sort<<<1, 1024, 0, s>>>(a, a.keys[0], a.places[0]);
  for (u32 pass = 0; a.tokens > EMBED_FEW && pass < a.passes; ++pass) {
    const int to = (int)(pass & 1), from = to ^ 1;
    if (!pass) {
      k_embed_count<true><<<a.tiles, 256, 0, s>>>(a, pass, nullptr);
      k_embed_move<true><<<a.tiles, 256, 0, s>>>(a, pass, nullptr, nullptr, a.keys[to], a.places[to]);
    } else {
      k_embed_count<false><<<a.tiles, 256, 0, s>>>(a, pass, a.keys[from]);
      k_embed_move<false><<<a.tiles, 256, 0, s>>>(a, pass, a.keys[from], a.places[from], a.keys[to], a.places[to]);
    }
    at = to;
  }
  if (g->type == G10_F32) { if (p.few) embed_sums<float, true>(a, p, at, s); else embed_sums<float, false>(a, p, at, s); }
  else if (g->type == G10_F16) { if (p.few) embed_sums<_Float16, true>(a, p, at, s); else embed_sums<_Float16, false>(a, p, at, s); }
  else { if (p.few) embed_sums<__bf16, true>(a, p, at, s); else embed_sums<__bf16, false>(a, p, at, s); }
  G10_HIP(hipGetLastError());
  return G10_OK;
}
