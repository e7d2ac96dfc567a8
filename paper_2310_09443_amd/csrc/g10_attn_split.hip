// Attention, forward, for few queries: the keys are split over the wavefronts and over workgroups, and joined.
//
// With one new token there is nothing to use a key twice for but the heads of its group: the pass is bound by the memory that holds the
// cache.  The 32 columns of a product are the group's heads of the queries (query i, head g of the group at column
// i * group + g), the wavefronts of a workgroup take every fourth tile of 32 keys, each with two tiles of its own in LDS and
// no barrier between them: one is on its way from memory while the other is worked on.
#include "g10_attn.h"

#define ST 32                      // keys of a tile
#define SW 4                       // wavefronts of a workgroup
#define JOIN 8                     // parts of a row on their way at once
#define BATCH (64 * SW)            // sequences whose work is cut into equal shares
#define LEAST 8                    // tiles of a share: two for each wavefront

// P is held times 2^LIFT where 16-bit floats have a short exponent: it is at most 1 here, so a key keeps all its bits down to 2^-29 of the largest
// of its part. The parts' sums are lifted alike; the lift leaves with 1 / l, and from lse.
template <class T> constexpr float LIFT = 0.0f;
template <class T> constexpr float DROP = 1.0f;
template <> constexpr float LIFT<_Float16> = 15.0f;
template <> constexpr float DROP<_Float16> = 0x1p-15f;

// The work of all sequences' key heads and blocks of 32 columns in one row, in tiles of keys, cut into equal shares: sequences of unlike
// lengths keep all compute units busy to the end.  A cut goes through a block wherever it falls; the pieces of a
// block meet in k_attn_join.  At most BATCH sequences; a sequence to a thread.
struct Shares {
  u32 each, total;                 // tiles of a share, of all
  const u32* end;                  // in LDS: tiles up to and with sequence b
};
struct Row { u32 blocks, tiles; };                                   // of a sequence: blocks of columns, tiles of keys to each
__device__ __forceinline__ Row row_of(const AttnArgs& a, const Seq& s) {
  const Tiles t = key_tiles<ST>(a, s.nk - s.nq, s.nk - 1, s.nk);
  return Row{((u32)s.nq * a.group + 31) / 32, s.nq ? (u32)t.count : 0u};
}
__device__ __forceinline__ Shares shares_of(const AttnArgs& a, u32* end, u32* tmp) {
  u32 n = 0, most = 0;
  if (threadIdx.x < a.batch) {
    const Row w = row_of(a, seq_of(a, threadIdx.x));
    n = w.blocks * w.tiles * a.kv_heads;
    most = w.tiles;
  }
  const u32 sum = wave_scan_incl(n), top = wave_max(most);
  if (lane_id() == 63) { tmp[wave_id()] = sum; tmp[SW + wave_id()] = top; }
  __syncthreads();
  u32 before = 0, longest = 0;
  Shares x = {0, 0, end};
  for (u32 w = 0; w < SW; ++w) {
    if (w < wave_id()) before += tmp[w];
    x.total += tmp[w];
    longest = max(longest, tmp[SW + w]);
  }
  end[threadIdx.x] = before + sum;
  __syncthreads();
  // no more pieces to a block than there is room for, and a piece is worth its joining
  x.each = max(max((x.total + a.shares - 1) / a.shares, (longest + a.splits - 2) / (a.splits - 1)), (u32)LEAST);
  return x;
}

struct Piece { float *o, *ml; u32* n; };                             // unfinished output of a row and a piece: [dim] and {maximum, sum}; the row's pieces

__device__ __forceinline__ Piece piece_of(const AttnArgs& a, u32 b, const Seq& s, int i, u32 h, u32 split) {
  const u64 row = ((a.q_start ? (u64)s.q0 : (u64)b * a.seq_q) + (u64)i) * a.heads + h;
  Piece p;
  p.o = a.part + (row * a.splits + split) * a.dim;
  p.ml = a.part_ml + (row * a.splits + split) * 2;
  p.n = a.part_n + row;
  return p;
}

// SHARED: a workgroup to a share, pieces of blocks to the workspace.  Otherwise a workgroup to a block.
template <class T, int DP, bool SHARED>
__global__ __launch_bounds__(64 * SW) void k_attn_split(const AttnArgs a) {
  // [wavefront][buffer][keys, values]; afterwards the wavefronts' outputs
  __shared__ __attribute__((aligned(256))) T lds[SW][2][2][ST * DP];
  __shared__ float ms[SW][32], ls[SW][32];
  __shared__ u32 ends[BATCH], tmp[2 * SW];
  typedef typename Vec<T>::x8 x8;
  if (blockIdx.x >= a.work) { clear_outputs<T>(a); return; }
  const u32 wave = uniform(wave_id()), lane = lane_id();
  u32 lk[2], lv[2];
  for (int i = 0; i < 2; ++i) { lk[i] = lds_addr(lds[wave][i][0]); lv[i] = lds_addr(lds[wave][i][1]); }
  Stage<DP, ST, 64> sk, sv;
  sk.init(lane, a.dim, a.ks[1]);
  sv.init(lane, a.dim, a.vs[1]);
  u32 unit = 0, at = 0, mine = 0, place = 0, stop = 0;
  Shares sh = {};
  if constexpr (SHARED) {
    sh = shares_of(a, ends, tmp);
    mine = blockIdx.x % a.tiles * (a.shares / a.tiles) + blockIdx.x / a.tiles;
    if ((u64)mine * sh.each >= sh.total) return;
    place = mine * sh.each;
    stop = min(place + sh.each, sh.total);
  } else {
    if (!unit_of(a.batch * a.kv_heads, a.tiles, unit, at)) return;
  }
  while (true) {
    u32 b, hk, piece = 0, pieces = 1, from = 0, take = 1, whole = 1;             // tiles from / whole .. (from + take) / whole of the block's
    int rb;
    Seq s;
    if constexpr (SHARED) {
      u32 lo = 0, hi = a.batch - 1;
      while (lo < hi) {
        const u32 mid = (lo + hi) / 2;
        if (uniform(sh.end[mid]) > place) hi = mid;
        else lo = mid + 1;
      }
      b = lo;
      s = seq_of(a, b);
      const Row w = row_of(a, s);
      const u32 in = place - (b ? uniform(sh.end[b - 1]) : 0);
      hk = in / w.tiles / w.blocks;
      rb = (int)(in / w.tiles % w.blocks);
      whole = w.tiles;
      from = in % w.tiles;
      take = min(whole - from, stop - place);
      const u32 first = place - from;                                // of the block
      piece = mine - first / sh.each;
      pieces = (first + whole - 1) / sh.each - first / sh.each + 1;
      place += take;
    } else {
      b = unit / a.kv_heads;
      hk = unit % a.kv_heads;
      s = seq_of(a, b);
      rb = (int)at;
    }
    const int off = s.nk - s.nq, rows = s.nq * (int)a.group;
    const Unseen unseen = unseen_keys(a, s);
    const T* K = (const T*)a.k + batch_off(a, b, a.ks[0]) + s.k0 * a.ks[1] + (int64_t)hk * a.ks[2];
    const T* V = (const T*)a.v + batch_off(a, b, a.vs[0]) + s.k0 * a.vs[1] + (int64_t)hk * a.vs[2];
    if (!SHARED && rb * 32 >= rows) break;
    const int r0 = rb * 32, r1 = r0 + 31 < rows ? r0 + 31 : rows - 1;
    const int row = r0 + (int)(lane & 31), c = row < rows ? row : rows - 1;
    const int i = c / (int)a.group;
    const u32 h = hk * a.group + (u32)(c % (int)a.group);
    const Seen seen = keys_of(a, i + off, s.nk);
    const int p0 = r0 / (int)a.group + off, p1 = r1 / (int)a.group + off;
    const Tiles tiles = key_tiles<ST>(a, p0, p1, s.nk);
    const int t0 = (int)((int64_t)tiles.count * from / whole), t1 = (int)((int64_t)tiles.count * (from + take) / whole);
    x8 q[DP / 16];
    const T* Q = (const T*)a.q + batch_off(a, b, a.qs[0]) + (s.q0 + i) * a.qs[1] + (int64_t)h * a.qs[2];
    frags_global<T, DP>(q, Q, 0, 0, 0, a.dim);
    f32x16 o[DP / 32] = {};
    float m = G10_NEG_INF, l = 0.0f;
    int t = t0 + (int)wave;
    if (t < t1) {
      sk.load(K, a.ks[1], tiles.at(t) * ST, s.nk, unseen, lk[0]);
      sv.load(V, a.vs[1], tiles.at(t) * ST, s.nk, unseen, lv[0]);
    }
    for (int buf = 0; t < t1; t += SW, buf ^= 1) {
      const int j0 = tiles.at(t) * ST;
      loads_done();
      if (t + SW < t1) {
        sk.load(K, a.ks[1], tiles.at(t + SW) * ST, s.nk, unseen, lk[buf ^ 1]);
        sv.load(V, a.vs[1], tiles.at(t + SW) * ST, s.nk, unseen, lv[buf ^ 1]);
      }
      const u32 tk = rows_base<DP>(lk[buf]), tv = cols_base<DP>(lv[buf]);
      f32x16 sc = {};
#pragma unroll
      for (int ks = 0; ks < DP / 16; ++ks) sc = Vec<T>::mfma(frag_rows<T, DP>(tk, 0, ks), q[ks], sc);
      if (!all_see(a, p0, p1, j0, j0 + ST - 1, s.nk)) {
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] = seen.key(j0 + res_row(r)) ? sc[r] : G10_NEG_INF;
      }
      float top = sc[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) top = fmaxf(top, sc[r]);
      top = fmaxf(m, both_max(top));
      const float base = top == G10_NEG_INF ? 0.0f : top * a.scale2;
      const float fade = exp2_fast(m * a.scale2 - base);
      m = top;
      float sum = 0.0f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        sc[r] = exp2_fast(sc[r] * a.scale2 - (base - LIFT<T>));
        sum += sc[r];
      }
      l = l * fade + both_sum(sum);
#pragma unroll
      for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[db][r] *= fade;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const x8 pf = pack8<T>(sc, k);
#pragma unroll
        for (int db = 0; db < DP / 32; ++db) o[db] = Vec<T>::mfma(frag_tr<T, DP>(tv, 16 * k, db), pf, o[db]);
      }
    }
    // the wavefronts' parts, joined
    if (lane < 32) { ms[wave][lane] = m * a.scale2; ls[wave][lane] = l; }
    __syncthreads();
    float big = ms[0][lane & 31];
    for (int w = 1; w < SW; ++w) big = fmaxf(big, ms[w][lane & 31]);
    const float mine = m == G10_NEG_INF ? 0.0f : exp2_fast(m * a.scale2 - big);
    float total = 0.0f;
    for (int w = 0; w < SW; ++w) {
      const float x = ms[w][lane & 31];
      total += x == G10_NEG_INF ? ls[w][lane & 31] : ls[w][lane & 31] * exp2_fast(x - big);
    }
    float* const part = (float*)&lds[0][0][0][0] + wave * 32 * DP;  // [column][value], 4 neighbouring values swapped round by the column
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int d = 8 * db + 2 * g + (int)(lane >> 5);            // in fours
        f32x4 x;
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = times(mine, o[db][4 * g + r]);
        *(f32x4*)(part + (lane & 31) * DP + ((d ^ (int)(lane & 7)) << 2)) = x;
      }
    __syncthreads();
    // eight threads to a column
    const int col = (int)threadIdx.x / 8, orow = r0 + col;
    const float cl = __shfl(total, col & 31, 64), cm = __shfl(big, col & 31, 64);
    if (orow < rows) {
      const int oi = orow / (int)a.group;
      const u32 oh = hk * a.group + (u32)(orow % (int)a.group);
      const float inv = cl > 0.0f ? 1.0f / cl : cl == 0.0f ? 0.0f : cl;
      const Piece to = piece_of(a, b, s, oi, oh, piece);
      T* out = (T*)a.o + batch_off(a, b, a.os[0]) + (s.q0 + oi) * a.os[1] + (int64_t)oh * a.os[2];
      for (int d = (int)threadIdx.x % 8; d < (int)a.dim / 4; d += 8) {
        const float* src = (const float*)&lds[0][0][0][0] + col * DP + ((d ^ (col & 7)) << 2);
        f32x4 x = *(const f32x4*)src;
        for (int w = 1; w < SW; ++w) x += *(const f32x4*)(src + w * 32 * DP);
        if (SHARED) *(f32x4*)(to.o + 4 * d) = x;
        else {
          typename Vec<T>::x4 y;
          for (int r = 0; r < 4; ++r) y[r] = (T)times(inv, x[r]);
          *(typename Vec<T>::x4*)(out + 4 * d) = y;
        }
      }
      if (threadIdx.x % 8 == 0) {
        if (SHARED) {
          to.ml[0] = cm;
          to.ml[1] = cl;
          if (!piece) *to.n = pieces;
        }
        if (!SHARED) (a.lse + row_off(a, b, oh, s))[oi] = cl > 0.0f ? (cm + __log2f(cl * DROP<T>)) * G10_LN2 : cl == 0.0f ? G10_NEG_INF : cl;
      }
    }
    __syncthreads();                                                // (the next block's tiles go where the parts lie)
    if constexpr (SHARED) {
      if (place >= stop) break;
    } else {
      at += a.tiles;
    }
  }
}

// A row's pieces joined, a wavefront to a row, eight pieces on their way at once.  Bound by the memory's latency: 5 us for 8 sequences of
// up to 32768 keys, one piece after the other 17.
template <class T>
__global__ __launch_bounds__(64 * SW) void k_attn_join(const AttnArgs a) {
  const u32 unit = blockIdx.x / a.tiles, b = unit / a.kv_heads, hk = unit % a.kv_heads, lane = lane_id();
  const Seq s = seq_of(a, b);
  const Row w = row_of(a, s);
  const int rows = s.nq * (int)a.group;
  for (int r = (int)((blockIdx.x % a.tiles) * SW + wave_id()); r < rows; r += (int)a.tiles * SW) {
    const int i = r / (int)a.group;
    const u32 h = hk * a.group + (u32)(r % (int)a.group);
    const Piece p = piece_of(a, b, s, i, h, 0);
    const u32 splits = w.tiles ? uniform(*p.n) : 0u;                 // (no key, no piece)
    float big = G10_NEG_INF;
    for (u32 k = lane; k < splits; k += 64) big = fmaxf(big, p.ml[2 * k]);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) big = fmaxf(big, __shfl_xor(big, d, 64));
    float x0 = 0.0f, x1 = 0.0f, l = 0.0f;
    const bool has = 2 * lane < a.dim;
    for (u32 k0 = 0; k0 < splits; k0 += 64) {                      // a lane to a split for the weights, then a lane to two values
      const u32 n = splits - k0 < 64 ? splits - k0 : 64;
      const float m = lane < n ? p.ml[2 * (k0 + lane)] : G10_NEG_INF, w = m == G10_NEG_INF ? 0.0f : exp2_fast(m - big);
      if (lane < n) l += m == G10_NEG_INF ? p.ml[2 * (k0 + lane) + 1] : p.ml[2 * (k0 + lane) + 1] * w;
      const float* from = p.o + (u64)k0 * a.dim + (has ? 2 * lane : 0);
      for (u32 k = 0; k < n; k += JOIN) {
        f32x2 y[JOIN];
#pragma unroll
        for (u32 j = 0; j < JOIN; ++j) y[j] = *(const f32x2*)(from + (u64)(k + j < n ? k + j : n - 1) * a.dim);
#pragma unroll
        for (u32 j = 0; j < JOIN; ++j) {
          const float wk = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), k + j < 64 ? k + j : 63));
          if (k + j < n) {
            x0 += times(wk, y[j][0]);
            x1 += times(wk, y[j][1]);
          }
        }
      }
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) l += __shfl_xor(l, d, 64);
    const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
    if (has) {
      typename Vec<T>::x2 y;
      y[0] = (T)times(inv, x0); y[1] = (T)times(inv, x1);
      *(typename Vec<T>::x2*)((T*)a.o + batch_off(a, b, a.os[0]) + (s.q0 + i) * a.os[1] + (int64_t)h * a.os[2] + 2 * lane) = y;
    }
    if (!lane) (a.lse + row_off(a, b, h, s))[i] = l > 0.0f ? (big + __log2f(l * DROP<T>)) * G10_LN2 : l == 0.0f ? G10_NEG_INF : l;
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------------------------------
#define CUS 256                    // compute units

static u32 attn_shares(const AttnArgs& a) { return a.dim <= 64 ? 2 * CUS : CUS; }

// Whether few queries meet so many keys that these kernels are faster than k_attn_fwd, whose workgroups take 128 queries of a head each.  Times
// in nanoseconds, measured: k_attn_fwd takes 16 for a workgroup's key (20 where two share a compute unit), these kernels 12 for a
// block's key on a compute unit, and 9000 for the joining.  32 queries of 32 heads (8 of keys) on 32768 keys: 516 us there,
// 54 here; 256 queries: 519 and 340; 512 queries: 520 and 688.  (Packed sequences go by their mean lengths, which are known here; max_q and max_k only cut the grid.)
static bool few_queries(const AttnArgs& a, u64& blocks, u64& keys) {
  const u64 nq = a.q_start ? ((u64)a.seq_q + a.batch - 1) / a.batch : a.seq_q, nk = a.q_start ? ((u64)a.seq_k + a.batch - 1) / a.batch : a.seq_k;
  blocks = (u64)a.batch * a.kv_heads * ((nq * a.group + 31) / 32);
  keys = nk;
  if (a.window) {
    const u64 near = (u64)a.window * (a.causal ? 1 : 2) + nq + a.sinks;
    if (near < keys) keys = near;
  }
  if (nq * a.group <= 32) return true;                               // (three of four wavefronts there would have no query)
  const u64 there = (u64)a.batch * a.heads * ((nq + 127) / 128), rounds = there <= CUS ? CUS : there * 5 / 4;
  return 12 * keys * blocks / CUS + 9000 < 16 * keys * rounds / CUS;
}
// The pieces of a block that there is room for; 0: the work is not for these kernels; 1: nothing is cut.  A compute unit holds one workgroup
// (heads of up to 64 values: two), each gets a share: with four times as many shares one sequence of 32768 keys takes 52 us in
// place of 32, with twice as many 40.  Cutting costs a second launch and a workgroup's search for its share: 512 keys of
// one sequence take 13.0 us cut and 10.8 whole, 1024 keys 13.3 and 16.2; where there is a block for every compute unit, 1024 keys
// of 32 sequences 30 us and 25, 2048 of 64 109 and 105 - more keys are cut all the same, for sequences of unlike lengths.
u32 attn_splits(const AttnArgs& a) {
  u64 blocks, keys;
  if (!few_queries(a, blocks, keys)) return 0;
  if (a.batch > BATCH || keys <= 768 || blocks >= 4 * CUS || (blocks >= CUS && keys <= 2048)) return 1;
  // Tiles are counted in 32 bits. Starts of packed sequences must not fall, but they are numbers on the device: where they do, every second sequence may
  // be as long as all rows, and a count that wraps would point outside the tensors.
  const u64 most = ((u64)a.seq_q * a.group / 32 + 1) * (a.q_start ? (a.batch + 1) / 2 : a.batch) + 2 * a.batch;
  if (most * a.kv_heads * (a.seq_k / ST + 2) >= 1ull << 31) return 1;
  const u64 n = (u64)a.batch * a.kv_heads;                           // (blocks of one key head lie in a row: the more, the fewer pieces)
  return (u32)(2 * ((attn_shares(a) + n - 1) / n) + 2);
}
u64 attn_split_bytes(const AttnArgs& a, u32 splits) {
  if (splits <= 1) return 0;
  const u64 rows = (u64)(a.q_start ? 1 : a.batch) * a.seq_q * a.heads;
  return rows * (splits * (a.dim + 2) + 1) * 4;
}

template <class T>
static void launch(AttnArgs a, hipStream_t s) {
  const u32 units = a.batch * a.kv_heads;
  if (a.splits > 1) {
    // with several blocks to a key head an XCD's shares lie in a row, so that blocks of the same keys meet in its L2 (64 queries of 4 x 8192
    // keys: 168 -> 101 us); with one they do not (8 x 32768 keys: 188 us, in a row 204)
    a.tiles = a.max_q * a.group > 32 ? 8 : 1;
    const u32 grid = with_rest(a, a.shares);
    if (a.dim <= 64) k_attn_split<T, 64, true><<<grid, 64 * SW, 0, s>>>(a);
    else k_attn_split<T, 128, true><<<grid, 64 * SW, 0, s>>>(a);
    a.tiles = tiles_in(units, 1, ((u64)a.max_q * a.group + SW - 1) / SW);
    k_attn_join<T><<<units * a.tiles, 64 * SW, 0, s>>>(a);
  } else {
    a.tiles = tiles_in(units, 1, ((u64)a.max_q * a.group + 31) / 32);
    const dim3 grid(with_rest(a, unit_grid(units, a.tiles)));
    if (a.dim <= 64) k_attn_split<T, 64, false><<<grid, 64 * SW, 0, s>>>(a);
    else k_attn_split<T, 128, false><<<grid, 64 * SW, 0, s>>>(a);
  }
}

int attn_forward_split(AttnArgs a, u32 splits, void* workspace, u32 type, hipStream_t s) {
  a.splits = splits;
  a.shares = attn_shares(a);
  const u64 rows = (u64)(a.q_start ? 1 : a.batch) * a.seq_q * a.heads;
  a.part = (float*)workspace;
  a.part_ml = splits > 1 ? a.part + rows * splits * a.dim : nullptr;
  a.part_n = splits > 1 ? (u32*)(a.part_ml + rows * splits * 2) : nullptr;
  if (type == G10_BF16) launch<__bf16>(a, s);
  else launch<_Float16>(a, s);
  G10_HIP(hipGetLastError());
  return G10_OK;
}
