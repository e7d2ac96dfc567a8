// Attention, backward: a kernel for the gradients of the queries and one for those of keys and values.  Both work P = 2^(S - lse) and dS = P (do V^T - delta) out again from q, k, v and the forward pass's lse.  Two
// kernels make seven products of the five that are needed; in return every gradient is summed by one wavefront in one order:
// no atomics, and nothing of the size of the scores in memory.
#include "g10_attn.h"

#define BT 64                      // rows of a tile in LDS
#define BW 128                     // rows of a workgroup, 32 to a wavefront
#define FEW 12                     // tiles of 32 keys up to which delta comes from P and dP
#define SOME 768                   // keys that a query sees up to which dS keeps its lower half for dq
#define FEWEST 128                 // and up to which P and dS keep theirs for dk and dv

// Whether lower halves are kept: in no sequence, in all, or where a sequence's own lengths say so. The third kernels hold both walks, one behind
// the other: both forms of a step in one loop would take 100 to 450 registers that there are not.
enum { PLAIN, FINE, OWN };

// In 16-bit floats with a short exponent, P and dS of long rows would fall below the smallest number.  P is held times
// 2^12 (it is at most 1), dS times 8 over the power of two at the largest |do| of what it is summed over: of the query for dQ, of the
// group's heads for dK.  Both leave by exact powers of two at the end.  (dS passes the type's largest number only where sum |v - o| of a key and a
// query is above 4000.)
template <class T> struct Lift;
template <> struct Lift<__bf16> {
  static constexpr float p2 = 0.0f, p = 1.0f;
  static constexpr bool ds = false;
};
template <> struct Lift<_Float16> {
  static constexpr float p2 = 12.0f, p = 4096.0f;
  static constexpr bool ds = true;
};
__device__ __forceinline__ float lift_of(u32 top) { return __uint_as_float((u32)(127 + 3 - clampi((int)(top >> 23) - 127, -60, 60)) << 23); }

// The work of k_attn_dkdv, all sequences' key heads and tiles of 128 keys in one row, in steps of 64 queries and ENTRY more a tile, cut
// into equal shares: a tile with sinks is seen by all later queries and one at the end of a causal sequence by few, and
// few tiles, or a few more than there are compute units, leave units idle.  A cut goes through a tile wherever it falls; its pieces
// meet in k_attn_cuts.
#define ENTRY 2u                   // steps that a tile's begin and end take
#define JOIN 4                     // pieces of a tile on their way at once where they are joined
#define SHARE 8                    // steps of a share at least: its pieces are worth their joining
struct Steps { int first, hi, each; u32 all; };                      // first and last query, tiles of 64 queries to a head, steps
__device__ __forceinline__ Steps steps_of(const AttnArgs& a, const Seq& s, int kt) {
  int lo = 0;                                                        // queries that see any key of the tile
  const int e1 = (kt + 1) * BW < s.nk ? (kt + 1) * BW - 1 : s.nk - 1;
  Steps x;
  x.hi = -1;
  if (kt * BW < s.nk) query_range(a, kt * BW, e1, s, lo, x.hi);
  x.first = lo / 32 * 32;
  x.each = x.hi >= lo ? (x.hi - x.first) / BT + 1 : 0;
  x.all = ENTRY + (u32)x.each * a.group;
  return x;
}
__device__ __forceinline__ int key_rows(const AttnArgs& a, const Seq& s) { return a.q_start ? s.nk : (int)a.seq_k; }   // of dk and dv to be written
__device__ __forceinline__ u64 head_steps(const AttnArgs& a, u32 b) {
  const Seq s = seq_of(a, b);
  u64 n = 0;
  for (int kt = 0; kt * BW < key_rows(a, s); ++kt) n += steps_of(a, s, kt).all;
  return n;
}
struct Place {
  u32 b, hk;
  int kt;
  u32 in;                          // steps of the tile before it
};
struct Row {
  u64 each, total;                 // steps of a share, of all
  const u64* end;                  // in LDS: steps up to and with a thread's sequences
  u32 seqs;                        // sequences to a thread
  __device__ __forceinline__ Place at(const AttnArgs& a, u64 place) const {
    u32 lo = 0, hi = 255;
    while (lo < hi) {
      const u32 mid = (lo + hi) / 2;
      if (uniform(end[mid]) > place) hi = mid;
      else lo = mid + 1;
    }
    const u64 before = lo ? uniform(end[lo - 1]) : 0;
    u64 in = place - before, head;
    Place p = {lo * seqs, 0, 0, 0};
    while (true) {
      head = seqs == 1 ? (uniform(end[lo]) - before) / a.kv_heads : head_steps(a, p.b);
      if (in < head * a.kv_heads) break;
      in -= head * a.kv_heads;
      ++p.b;
    }
    p.hk = (u32)(in / head);
    in %= head;
    const Seq s = seq_of(a, p.b);
    for (u32 n; in >= (n = steps_of(a, s, p.kt).all); ++p.kt) in -= n;
    p.in = (u32)in;
    return p;
  }
};
__device__ __forceinline__ Row row_of(const AttnArgs& a, u64* end) {
  Row r = {0, 0, end, (a.batch + 255) / 256};
  u64 n = 0;
  for (u32 b = threadIdx.x * r.seqs; b < (threadIdx.x + 1) * r.seqs && b < a.batch; ++b) n += head_steps(a, b) * a.kv_heads;
  end[threadIdx.x] = n;
  __syncthreads();
  for (u32 d = 1; d < 256; d *= 2) {
    const u64 x = threadIdx.x >= d ? end[threadIdx.x - d] : 0;
    __syncthreads();
    end[threadIdx.x] += x;
    __syncthreads();
  }
  r.total = uniform(end[255]);
  r.each = (r.total + a.shares - 1) / a.shares;
  if (r.each < SHARE) r.each = SHARE;
  return r;
}

// Gradients of 128 keys and values, 32 to a wavefront, which holds their rows and sums in registers and walks over the
// queries that see them, of all heads of the group, 32 at a time:
//   S = Q K^T,  P = 2^(S - lse),  dP = dO V^T,  dS = P (dP - delta),  dV^T += dO^T P,  dK^T += Q^T dS
// The first products come out with a key to a lane and feed the second ones as they lie.  A wavefront has a SIMD's registers to
// itself (in heads of 64 values: half of them), so nobody else's work fills its waits: it works on the next 32 queries' first
// products and these ones' second ones, product by product, with these ones' exponentials strewn between and the fragments four
// ahead on their way from LDS.  Tiles of 64 queries: this one, the next, and the one on its way from memory.
// SHARED: a workgroup to a share.  Otherwise one to a tile.
struct Half { u32 rows, cols, stats; };                              // LDS addresses of 32 queries of a tile: rows_base and cols_base of Q, with dO a tile behind it; lse2 and delta

// The sums of dP begin with what is taken from them.
__device__ __forceinline__ f32x16 minus_delta(const Half& x) {
  f32x16 d;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const f32x4 four = *(__attribute__((address_space(3))) const f32x4*)(uintptr_t)(x.stats + (u32)(BT * 4 + k * 32));
#pragma unroll
    for (int r = 0; r < 4; ++r) d[4 * k + r] = four[r];
  }
  return d;
}

// Keys that the query at position p sees.
__device__ __forceinline__ int keys_at(const AttnArgs& a, int p, int nk) {
  const Seen s = keys_of(a, p, nk);
  const int first = s.first > 0 ? s.first : 0;
  return !s.span || s.lo < first ? max(first, s.span ? s.lo + (int)s.span : 0) : first + (int)s.span;
}
// Whether any of the queries at p0..p1 sees some keys, and SOME at most. (It sees more the further it stands, or is nearer to the middle: one at an end sees fewest.)
__device__ __forceinline__ bool some_see_few(const AttnArgs& a, int p0, int p1, int nk) {
  if (a.causal && p0 < 0) p0 = 0;
  return p0 <= p1 && min(keys_at(a, p0, nk), keys_at(a, p1, nk)) <= SOME;
}
// Whether none of a sequence's queries sees more than FEWEST.
__device__ __forceinline__ bool all_see_few(const AttnArgs& a, int nk) {
  const u64 near = a.window ? (u64)a.window * (a.causal ? 1 : 2) + a.sinks : (u64)nk;
  return (u64)nk <= FEWEST || near <= FEWEST;
}

// What rounding eight values of x left of them.
template <class T>
__device__ __forceinline__ typename Vec<T>::x8 left8(f32x16& x, const typename Vec<T>::x8& got, int s) {
#pragma unroll
  for (int k = 0; k < 8; ++k) x[8 * s + k] -= (float)got[k];
  return pack8<T>(x, s);
}

// In: the tile's scores and dP - delta in sc and dp.  Out: the next tile's.  BOTH: P and dS meet dO and Q as their rounding and what that left.
template <class T, int DP, bool BOTH>
__device__ __forceinline__ void back_step(const Half& cu, const Half& nx, const typename Vec<T>::x8 (&kf)[DP / 16], const typename Vec<T>::x8 (&vf)[DP / 16],
                                          f32x16& sc, f32x16& dp, f32x16 (&dk)[DP / 32], f32x16 (&dv)[DP / 32], float scale2, float lift_ds) {
  typedef typename Vec<T>::x8 x8;
  constexpr int KS = DP / 16, DB = DP / 32, N = 2 * KS + 4 * DB, AHEAD = 4, RING = 5;
  x8 f[RING], pf[2], df[2], pl[2], dl[2];
  auto read = [&](int e) -> x8 {
    if (e < 2 * KS) return frag_rows<T, DP>(nx.rows, e % 2 * BT, e / 2);
    e -= 2 * KS;
    return frag_tr<T, DP>(cu.cols, (e < 2 * DB ? BT : -32) + e / DB * 16, e % DB);
  };
  // four queries' lse2, read one group ahead
  f32x4 row[2];
  auto row_read = [&](int k) { row[k & 1] = *(__attribute__((address_space(3))) const f32x4*)(uintptr_t)(cu.stats + (u32)(k * 32)); };
  auto exps = [&](int from, int to) {
#pragma unroll
    for (int r = from; r < to; ++r) {
      if (r % 4 == 0 && r < 12) row_read(r / 4 + 1);
      sc[r] = exp2_fast(sc[r] * scale2 - row[r / 4 & 1][r % 4]);
      if (r % 8 == 7) pf[r / 8] = pack8<T>(sc, r / 8);
    }
  };
  auto grads = [&](int from, int to) {
#pragma unroll
    for (int r = from; r < to; ++r) {
      dp[r] = times(sc[r], Lift<T>::ds ? dp[r] * lift_ds : dp[r]);
      if (r % 8 == 7) df[r / 8] = pack8<T>(dp, r / 8);
    }
  };
  row_read(0);
#pragma unroll
  for (int e = 0; e < AHEAD; ++e) f[e % RING] = read(e);
  f32x16 sn = {}, dn = minus_delta(nx);
  hold();
  each_of<0, N>([&](auto step) __attribute__((always_inline)) {
    constexpr int e = decltype(step)::value;
    if constexpr (e + AHEAD < N) f[(e + AHEAD) % RING] = read(e + AHEAD);
    if constexpr (e < 2 * KS) {                                      // (in turn: a product on the sums of the one before would wait for it)
      if constexpr (e % 2 == 0) sn = Vec<T>::mfma(f[e % RING], kf[e / 2], sn);
      else dn = Vec<T>::mfma(f[e % RING], vf[e / 2], dn);
      if constexpr (e < KS) exps(16 * e / KS, 16 * (e + 1) / KS);
      else grads(16 * (e - KS) / KS, 16 * (e - KS + 1) / KS);
      if constexpr (BOTH && e == 2 * KS - 1) {
#pragma unroll
        for (int k = 0; k < 2; ++k) { pl[k] = left8<T>(sc, pf[k], k); dl[k] = left8<T>(dp, df[k], k); }
      }
    } else {
      constexpr int v = e - 2 * KS;
      if constexpr (v < 2 * DB) dv[v % DB] = Vec<T>::mfma(f[e % RING], pf[v / DB], dv[v % DB]);
      else dk[v % DB] = Vec<T>::mfma(f[e % RING], df[v / DB - 2], dk[v % DB]);
      if constexpr (BOTH && v < 2 * DB) dv[v % DB] = Vec<T>::mfma(f[e % RING], pl[v / DB], dv[v % DB]);
      if constexpr (BOTH && v >= 2 * DB) dk[v % DB] = Vec<T>::mfma(f[e % RING], dl[v / DB - 2], dk[v % DB]);
#pragma unroll
      for (int r = 16 * v / (4 * DB); r < 16 * (v + 1) / (4 * DB); ++r) { sc[r] = sn[r]; dp[r] = dn[r]; }
    }
    hold();
  });
}

template <class T, int DP, int FORM, bool SHARED>
__global__ __launch_bounds__(256, DP == 64 ? 2 : 1) void k_attn_dkdv(const AttnArgs a) {
  __shared__ __attribute__((aligned(256))) T lds[3][2][BT * DP];
  __shared__ __attribute__((aligned(16))) float rows[3][2][BT];      // lse2, delta of a tile's queries
  __shared__ u64 ends[SHARED ? 256 : 1];
  typedef typename Vec<T>::x8 x8;
  if (blockIdx.x >= a.work) {
    const Rest r = rest_of(a.k_start, a.batch, a.seq_k, blockIdx.x - a.work);
    clear_rest<T>(r, a.dk, a.dks, a.kv_heads, a.dim);
    clear_rest<T>(r, a.dv, a.dvs, a.kv_heads, a.dim);
    return;
  }
  Place at = {};
  u64 place = 0, stop = 0;
  Row row = {};
  u32 mine = 0;
  if constexpr (SHARED) {
    row = row_of(a, ends);
    mine = blockIdx.x % 8 * (a.shares / 8) + blockIdx.x / 8;         // (an XCD's shares lie in a row)
    if (!threadIdx.x) a.cuts[mine] = Cut{};
    place = mine * row.each;
    if (place >= row.total) return;
    stop = place + row.each < row.total ? place + row.each : row.total;
    at = row.at(a, place);
  } else {
    u32 unit, kt;
    if (!unit_of(a.batch * a.kv_heads, a.tiles, unit, kt)) return;
    at.b = unit / a.kv_heads;
    at.hk = unit % a.kv_heads;
    at.kt = (int)kt;
  }
  const u32 wave = uniform(wave_id()), lane = lane_id();
  Walk<DP, BT, 256> sq, sd;
  sq.init(threadIdx.x, a.dim, a.qs[1]);
  sd.init(threadIdx.x, a.dim, a.dos[1]);
  const u32 tile0 = lds_addr(lds[0][0]) + wave * 1024, rows0 = lds_addr(rows[0]);
  bool again = false;
  while (true) {
    const u32 b = at.b, hk = at.hk;
    const int kt = at.kt;
    const Seq s = seq_of(a, b);
    const int nk_all = key_rows(a, s);
    if (!SHARED && kt * BW >= nk_all) break;
    const T* Q0 = (const T*)a.q + batch_off(a, b, a.qs[0]) + s.q0 * a.qs[1] + (int64_t)hk * a.group * a.qs[2];
    const T* D0 = (const T*)a.d_o + batch_off(a, b, a.dos[0]) + s.q0 * a.dos[1] + (int64_t)hk * a.group * a.dos[2];
    float lift = 1.0f;
    if (Lift<T>::ds) {
      const u32 n = a.group * a.q_tiles * 4;
      const u32* all = a.amax + ((u64)b * a.kv_heads + hk) * n;
      u32 top = 0;
      for (u32 x = lane; x < n; x += 64) top = max(top, all[x]);
      top = wave_max(top);
      lift = lift_of(top);
    }
    const float lift_ds = lift / Lift<T>::p;
    const Unseen unseen = unseen_queries(a, s);
    const int j0 = kt * BW + (int)wave * 32, j = j0 + (int)(lane & 31);
    f32x16 dk[DP / 32] = {}, dv[DP / 32] = {};
    const Steps steps = steps_of(a, s, kt);
    const int first = steps.first, each = steps.each, hi = steps.hi;
    int from = 0, all = each * (int)a.group;                         // tiles of queries of all heads one after the other
    u32 take = steps.all;
    if constexpr (SHARED) {
      if ((u64)(take - at.in) > stop - place) take = at.in + (u32)(stop - place);
      from = at.in > ENTRY ? (int)(at.in - ENTRY) : 0;
      all = (take > ENTRY ? (int)(take - ENTRY) : 0) - from;
    }
    const bool whole = !SHARED || (!at.in && take == steps.all);
    if (all > 0) {
      int ilo = 0, ihi = -1, flo, fhi;                               // ... of the lane; that see all of the wavefront's keys
      if (j < s.nk) query_range(a, j, j, s, ilo, ihi);
      full_range(a, j0, j0 + 31, s, flo, fhi);
      const u32 span = ihi >= ilo ? (u32)(ihi - ilo + 1) : 0u;
      const int head = from / each;
      int fi = first + from % each * BT, cur = fi;                   // first query of the tile to be fetched, of this tile
      const T *Q = Q0 + head * a.qs[2], *D = D0 + head * a.dos[2];   // of the head to be fetched
      const float* L = (wave == 0 ? a.lse2 : a.delta) + row_off(a, b, hk * a.group + (u32)head, s) + lane;
      sq.from(Q, a.qs[1], fi);
      sd.from(D, a.dos[1], fi);
      u32 to = 0;                                                    // buffer of the next tile to be fetched
      auto fetch = [&]() {
        const u32 at = tile0 + to * (2 * BT * DP * 2);
        sq.load(fi, s.nq, unseen, a.qs[1], at);
        sd.load(fi, s.nq, unseen, a.dos[1], at + BT * DP * 2);
        if (wave < 2) load_words(L + (fi + (int)lane < s.nq ? fi : s.nq - 1 - (int)lane), rows0 + (2 * to + wave) * (BT * 4));
        to = to == 2 ? 0 : to + 1;
        fi += BT;
        if (fi > hi) {                                               // the next head of the group
          fi = first;
          Q += a.qs[2];
          D += a.dos[2];
          L += a.seq_q;
          sq.from(Q, a.qs[1], first);
          sd.from(D, a.dos[1], first);
        }
      };
      if (again) __syncthreads();                                    // (the tiles of the keys before are read)
      again = true;
      fetch();
      if (all > 1) fetch();
      x8 kf[DP / 16], vf[DP / 16];
      frags_global<T, DP>(kf, (const T*)a.k + batch_off(a, b, a.ks[0]) + s.k0 * a.ks[1] + (int64_t)hk * a.ks[2], a.ks[1], j, s.nk - 1, a.dim);
      frags_global<T, DP>(vf, (const T*)a.v + batch_off(a, b, a.vs[0]) + s.k0 * a.vs[1] + (int64_t)hk * a.vs[2], a.vs[1], j, s.nk - 1, a.dim);
      const u32 rb = rows_base<DP>(lds_addr(lds[0][0])), cb = cols_base<DP>(lds_addr(lds[0][0])), lb = rows0 + 16 * (lane >> 5);
      auto half = [&](u32 buf, u32 n) {
        return Half{rb + buf * (2 * BT * DP * 2) + n * (32 * DP * 2), cb + buf * (2 * BT * DP * 2) + n * (32 * DP * 2), lb + buf * (2 * BT * 4) + n * 128};
      };
      loads_done();
      __syncthreads();
      f32x16 sc = {}, dp = minus_delta(half(0, 0));
#pragma unroll
      for (int ks = 0; ks < DP / 16; ++ks) sc = Vec<T>::mfma(frag_rows<T, DP>(rb, 0, ks), kf[ks], sc);
#pragma unroll
      for (int ks = 0; ks < DP / 16; ++ks) dp = Vec<T>::mfma(frag_rows<T, DP>(rb, BT, ks), vf[ks], dp);
      u32 buf = 0, n = 0;                                            // this tile's buffer; its half
      int t = 0;
      auto walk = [&](auto both) __attribute__((always_inline)) {
#pragma nounroll
        while (t < all) {
          if (!n) {                                                    // this tile and the next are there; the one behind them goes where the one before lay
            loads_done();
            __syncthreads();
            if (t + 2 < all) fetch();
          }
          if (!(cur >= flo && cur + 31 <= fhi)) {                      // not all queries see all keys
            const int at = cur + 4 * (int)(lane >> 5) - ilo;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const bool seen = (u32)(at + 8 * (r / 4) + r % 4) < span;
              sc[r] = seen ? sc[r] : G10_NEG_INF;
            }
          }
          const Half here = half(buf, n);
          cur += 32;
          if (n || cur > hi) {                                         // the tile's last
            n = 0;
            ++t;
            buf = buf == 2 ? 0 : buf + 1;
            if (cur > hi) cur = first;
          } else n = 1;
          back_step<T, DP, decltype(both)::value != 0>(here, half(buf, n), kf, vf, sc, dp, dk, dv, a.scale2, lift_ds);
        }
      };
      if constexpr (FORM != OWN) walk(Const<FORM == FINE>{});
      else if (all_see_few(a, s.nk)) walk(Const<1>{});
      else walk(Const<0>{});
    }
    const float fk = a.scale / lift, fv = 1.0f / Lift<T>::p;
    if (!whole) {
      if (!at.in && !threadIdx.x) {                                  // the first piece
        const u64 last = place + steps.all - 1;
        a.cuts[mine] = Cut{b, hk, (u32)kt, (u32)(last / row.each) - mine};
      }
      float* to = a.part + ((u64)mine * 2 + !at.in) * (2 * BW * DP) + ((int)wave * 32 + (int)(lane & 31)) * DP;
#pragma unroll
      for (int x = 0; x < DP / 32; ++x)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int d = 32 * x + 8 * g + 4 * (int)(lane >> 5);
          *(f32x4*)(to + d) = f32x4{dv[x][4 * g], dv[x][4 * g + 1], dv[x][4 * g + 2], dv[x][4 * g + 3]} * fv;
          *(f32x4*)(to + BW * DP + d) = f32x4{dk[x][4 * g], dk[x][4 * g + 1], dk[x][4 * g + 2], dk[x][4 * g + 3]} * fk;
        }
    } else if (j < nk_all) {
      T* dK = (T*)a.dk + batch_off(a, b, a.dks[0]) + (s.k0 + j) * a.dks[1] + (int64_t)hk * a.dks[2];
      T* dV = (T*)a.dv + batch_off(a, b, a.dvs[0]) + (s.k0 + j) * a.dvs[1] + (int64_t)hk * a.dvs[2];
#pragma unroll
      for (int x = 0; x < DP / 32; ++x)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int d = 32 * x + 8 * g + 4 * (int)(lane >> 5);
          if (d < (int)a.dim) {
            typename Vec<T>::x4 y, z;
#pragma unroll
            for (int r = 0; r < 4; ++r) { y[r] = (T)(dk[x][4 * g + r] * fk); z[r] = (T)(dv[x][4 * g + r] * fv); }
            *(typename Vec<T>::x4*)(dK + d) = y;
            *(typename Vec<T>::x4*)(dV + d) = z;
          }
        }
    }
    if constexpr (SHARED) {
      place += take - at.in;
      if (place >= stop) break;
      at.in = 0;
      if (++at.kt * BW >= nk_all) {                                  // the next key head; the next sequence with keys
        at.kt = 0;
        if (++at.hk == a.kv_heads) {
          at.hk = 0;
          while (!key_rows(a, seq_of(a, ++at.b))) {}
        }
      }
    } else {
      at.kt += (int)a.tiles;
    }
  }
}

// The pieces of a tile that is cut, joined in their order: the first lies in its share's second place, the others in the first ones
// of the shares behind.  Bound by the memory that holds them: 256 shares of heads of 128 values 64 MB, 17 us.
template <class T, int DP>
__global__ __launch_bounds__(256) void k_attn_cuts(const AttnArgs a) {
  const Cut c = a.cuts[blockIdx.x];
  if (!c.more) return;
  const u32 b = c.b, hk = c.hk, kt = c.kt;
  const bool key = blockIdx.y & 1;
  const Seq s = seq_of(a, b);
  const int nk_all = key_rows(a, s);
  const float* from = a.part + ((u64)blockIdx.x * 4 + 2 + key) * (BW * DP);
  T* out = key ? (T*)a.dk + batch_off(a, b, a.dks[0]) + s.k0 * a.dks[1] + (int64_t)hk * a.dks[2]
               : (T*)a.dv + batch_off(a, b, a.dvs[0]) + s.k0 * a.dvs[1] + (int64_t)hk * a.dvs[2];
  for (u32 e = blockIdx.y / 2 * 256 + threadIdx.x; e < BW * DP / 4; e += 4 * 256) {
    const int j = (int)(kt * BW + e / (DP / 4)), d = (int)(e % (DP / 4)) * 4;
    if (j >= nk_all || d >= (int)a.dim) continue;
    f32x4 x = *(const f32x4*)(from + 4 * e);
    auto piece = [&](u32 k) { return *(const f32x4*)(from + ((u64)k * 4 - 2) * (BW * DP) + 4 * e); };
    u32 k = 1;
    for (; k + JOIN - 1 <= c.more; k += JOIN) {
      f32x4 y[JOIN];
#pragma unroll
      for (u32 n = 0; n < JOIN; ++n) y[n] = piece(k + n);
#pragma unroll
      for (u32 n = 0; n < JOIN; ++n) x += y[n];
    }
    for (; k <= c.more; ++k) x += piece(k);
    typename Vec<T>::x4 y;
#pragma unroll
    for (int r = 0; r < 4; ++r) y[r] = (T)x[r];
    *(typename Vec<T>::x4*)(out + (int64_t)j * (key ? a.dks[1] : a.dvs[1]) + d) = y;
  }
}

// Gradients of 128 queries, 32 to a wavefront, which walks over the keys they see, 32 at a time:
//   S^T = K Q^T,  dP^T = V dO^T  come out with a query to a lane,  dQ^T += K^T dS^T;   first, delta = sum(do o) of each query, which
// the keys' kernel takes from here.  The same pipeline as there, two wavefronts to a SIMD.
// These keys' scores and dP are in sc and dp, the next ones' go to sn and dn.  LDS: rows_base of the next keys, with their values behind them,
// cols_base of these keys.  BOTH: dS meets the keys as its rounding and what that left, in two products.
template <class T, int DP, bool BOTH>
__device__ __forceinline__ void query_step(u32 rows, u32 cols, const typename Vec<T>::x8 (&q)[DP / 16], const typename Vec<T>::x8 (&dout)[DP / 16],
                                           f32x16& sc, f32x16& dp, f32x16& sn, f32x16& dn, f32x16 (&dq)[DP / 32], float scale2, float le, const f32x16& less, float lift) {
  typedef typename Vec<T>::x8 x8;
  constexpr int KS = DP / 16, DB = DP / 32, N = 2 * KS + 2 * DB, AHEAD = 4, RING = 5;
  x8 f[RING], df[2], left[2];
  auto read = [&](int e) -> x8 {
    if (e < 2 * KS) return frag_rows<T, DP>(rows, e % 2 * 32, e / 2);
    return frag_tr<T, DP>(cols, (e - 2 * KS) / DB * 16, (e - 2 * KS) % DB);
  };
#pragma unroll
  for (int e = 0; e < AHEAD; ++e) f[e % RING] = read(e);
  sn = f32x16{};
  dn = less;
  hold();
  each_of<0, N>([&](auto step) __attribute__((always_inline)) {
    constexpr int e = decltype(step)::value;
    if constexpr (e + AHEAD < N) f[(e + AHEAD) % RING] = read(e + AHEAD);
    if constexpr (e < 2 * KS) {
      if constexpr (e % 2 == 0) sn = Vec<T>::mfma(f[e % RING], q[e / 2], sn);
      else dn = Vec<T>::mfma(f[e % RING], dout[e / 2], dn);
      // (a value's product one behind its exponential, which takes its time)
#pragma unroll
      for (int r = 16 * e / (2 * KS); r < 16 * (e + 1) / (2 * KS) + (e == 2 * KS - 1); ++r) {
        if (r < 16) sc[r] = exp2_fast(sc[r] * scale2 - le);
        if (r) dp[r - 1] = times(sc[r - 1], Lift<T>::ds ? dp[r - 1] * lift : dp[r - 1]);
        if (r == 8 || r == 16) df[r / 8 - 1] = pack8<T>(dp, r / 8 - 1);
      }
    } else {
      constexpr int v = e - 2 * KS;
      dq[v % DB] = Vec<T>::mfma(f[e % RING], df[v / DB], dq[v % DB]);
      if constexpr (BOTH) {
        if constexpr (v % DB == 0) left[v / DB] = left8<T>(dp, df[v / DB], v / DB);
        dq[v % DB] = Vec<T>::mfma(f[e % RING], left[v / DB], dq[v % DB]);
      }
    }
    hold();
  });
}

template <class T, int DP, int FORM>
__global__ __launch_bounds__(256, 2) void k_attn_dq(const AttnArgs a) {
  constexpr int KT = 32, NB = 4;                                     // keys of a tile; these, the next, two on their way
  __shared__ __attribute__((aligned(256))) T lds[NB][2][KT * DP];
  typedef typename Vec<T>::x8 x8;
  if (blockIdx.x >= a.work) {
    clear_rest<T>(rest_of(a.q_start, a.batch, a.seq_q, blockIdx.x - a.work), a.dq, a.dqs, a.heads, a.dim);
    return;
  }
  u32 unit, head, first;
  if (!block_of(a.batch * a.kv_heads, a.group, a.tiles, unit, head, first)) return;
  const u32 b = unit / a.kv_heads, hk = unit % a.kv_heads, h = hk * a.group + head;
  const Seq s = seq_of(a, b);
  const int off = s.nk - s.nq;
  const u32 wave = uniform(wave_id()), lane = lane_id();
  const T* K = (const T*)a.k + batch_off(a, b, a.ks[0]) + s.k0 * a.ks[1] + (int64_t)hk * a.ks[2];
  const T* V = (const T*)a.v + batch_off(a, b, a.vs[0]) + s.k0 * a.vs[1] + (int64_t)hk * a.vs[2];
  Walk<DP, KT, 256> sk, sv;
  sk.init(threadIdx.x, a.dim, a.ks[1]);
  sv.init(threadIdx.x, a.dim, a.vs[1]);
  const u32 tile0 = lds_addr(lds[0][0]) + wave * 1024;
  const u32 rb = rows_base<DP>(lds_addr(lds[0][0])), cb = cols_base<DP>(lds_addr(lds[0][0]));
  const Unseen unseen = unseen_keys(a, s);
  bool again = false;
  u32 most = 0;
  for (int qt = (int)first; qt * BW < s.nq; qt += (int)a.tiles) {
    const int i0 = qt * BW + (int)wave * 32, i = i0 + (int)(lane & 31), c = i < s.nq ? i : s.nq - 1;
    const Seen seen = keys_of(a, i + off, s.nk);
    const int wp0 = i0 + off, wp1 = (i0 + 31 < s.nq ? i0 + 31 : s.nq - 1) + off;
    const int e1 = (qt + 1) * BW - 1 < s.nq ? (qt + 1) * BW - 1 : s.nq - 1;
    const Tiles tiles = key_tiles<KT>(a, qt * BW + off, e1 + off, s.nk);
    // keys that all of the wavefront's queries see: flo..fhi, and the sinks up to fhi
    const int w = (int)a.window;
    int flo = w ? wp1 - w + 1 : 0, fhi = s.nk - 1;
    if (a.causal && wp0 < fhi) fhi = wp0;
    if (!a.causal && w && wp0 + w - 1 < fhi) fhi = wp0 + w - 1;
    const int ftop = a.causal ? fhi : s.nk - 1;

    // delta is sum(P dP) as well as sum(do o).  The second costs a reading of o, but o is rounded, and where few keys are seen that
    // error is large beside dq and dk: against a result that is only rounded once, theirs is 1.4 times as large with the first and with
    // the second 2.3 times for 4 keys, 1.6 for 128, 1.5 for 400.  So the first up to 384 keys of the workgroup's, for one more walk over them
    // (two of a step's three products).  (See form_dq for more of them.)
    const bool few = tiles.count <= FEW;
    u32 to = 0;
    int ft = 0, rest = few ? 2 * tiles.count : tiles.count;          // next tile to be fetched; how many there are to be
    auto fetch = [&]() {
      if (ft == 0 || ft == tiles.head) { sk.from(K, a.ks[1], tiles.at(ft) * KT); sv.from(V, a.vs[1], tiles.at(ft) * KT); }
      const u32 to_at = tile0 + to * (2 * KT * DP * 2);
      const int row0 = tiles.at(ft) * KT;
      sk.load(row0, s.nk, unseen, a.ks[1], to_at);
      sv.load(row0, s.nk, unseen, a.vs[1], to_at + KT * DP * 2);
      to = (to + 1) % NB;
      if (++ft == tiles.count) ft = 0;
      --rest;
    };
    if (again) __syncthreads();                                      // (the tiles of the queries before are read)
    again = true;
    for (int t = 0; t < 3 && rest; ++t) fetch();
    x8 q[DP / 16], dout[DP / 16];
    frags_global<T, DP>(q, (const T*)a.q + batch_off(a, b, a.qs[0]) + s.q0 * a.qs[1] + (int64_t)h * a.qs[2], a.qs[1], i, s.nq - 1, a.dim);
    frags_global<T, DP>(dout, (const T*)a.d_o + batch_off(a, b, a.dos[0]) + s.q0 * a.dos[1] + (int64_t)h * a.dos[2], a.dos[1], i, s.nq - 1, a.dim);
    float de = 0.0f, big = 0.0f, le;
    const int64_t r0 = row_off(a, b, h, s) + c;
    le = a.lse[r0];
    le = le == G10_NEG_INF ? -le : le * G10_LOG2E;                   // (a query that sees no key: its probabilities are to be 0)
    if (!few) {
      x8 o[DP / 16];
      frags_global<T, DP>(o, (const T*)a.o + batch_off(a, b, a.os[0]) + s.q0 * a.os[1] + (int64_t)h * a.os[2], a.os[1], i, s.nq - 1, a.dim);
#pragma unroll
      for (int ks = 0; ks < DP / 16; ++ks)
#pragma unroll
        for (int x = 0; x < 8; ++x) de += (float)dout[ks][x] * (float)o[ks][x];
    }
    float lift = 1.0f;
    if (Lift<T>::ds) {
#pragma unroll
      for (int ks = 0; ks < DP / 16; ++ks)
#pragma unroll
        for (int x = 0; x < 8; ++x) big = fmaxf(big, fabsf((float)dout[ks][x]));
      big = le == -G10_NEG_INF ? 0.0f : both_max(big);               // (a query that sees no key has no part in the gradients)
      lift = lift_of(__float_as_uint(big));
      most = max(most, wave_max(__float_as_uint(big)));
    }
    f32x16 dq[DP / 32] = {};
    loads_done();
    __syncthreads();
    u32 buf = 0;
    auto arrive = [&]() __attribute__((always_inline)) {
      if (rest) loads_done_but<Stage<DP, KT, 256>::IT * 2>();        // the next tile is there, the one behind it may be on its way
      else loads_done();
      __syncthreads();
      if (rest) fetch();
    };
    f32x16 sa, da;
    auto scores = [&](u32 rows, const f32x16& from) __attribute__((always_inline)) {
      sa = f32x16{};
      da = from;
#pragma unroll
      for (int ks = 0; ks < DP / 16; ++ks) {
        sa = Vec<T>::mfma(frag_rows<T, DP>(rows, 0, ks), q[ks], sa);
        da = Vec<T>::mfma(frag_rows<T, DP>(rows, KT, ks), dout[ks], da);
      }
    };
    if (few) {                                                       // (without a pipeline: it is short)
#pragma nounroll
      for (int t = 0; t < tiles.count; ++t) {
        arrive();
        scores(rb + buf * (2 * KT * DP * 2), f32x16{});
        const int j0 = tiles.at(t) * KT;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float p = exp2_fast((seen.key(j0 + res_row(r)) ? sa[r] : G10_NEG_INF) * a.scale2 - le);
          de += times(p, da[r]);
        }
        buf = (buf + 1) % NB;
      }
    }
    de = both_sum(de);
    if (lane < 32 && i < s.nq) {
      ((float*)a.delta)[r0] = -de;
      ((float*)a.lse2)[r0] = le - Lift<T>::p2;
    }
    if (tiles.count) {
      f32x16 sb, db, less;                                           // (the sums of dP begin with minus delta)
#pragma unroll
      for (int r = 0; r < 16; ++r) less[r] = -de;
      auto walk = [&](auto both) __attribute__((always_inline)) {
        int t = 0;
        auto turn = [&](f32x16& sc, f32x16& dp, f32x16& sn, f32x16& dn) __attribute__((always_inline)) {
          arrive();
          const int j0 = tiles.at(t) * KT, j1 = j0 + KT - 1;
          if (!((j0 >= flo && j1 <= fhi) || (j1 < (int)a.sinks && j1 <= ftop))) {
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[r] = seen.key(j0 + res_row(r)) ? sc[r] : G10_NEG_INF;
          }
          const u32 next = (buf + 1) % NB;
          query_step<T, DP, decltype(both)::value != 0>(rb + next * (2 * KT * DP * 2), cb + buf * (2 * KT * DP * 2), q, dout, sc, dp, sn, dn, dq, a.scale2, le, less, lift);
          buf = next;
          ++t;
        };
        const Runs runs = runs_of<KT>(a, tiles, wp0, wp1, s.nk);
        // two runs of tiles with something to do; between them only what the other wavefronts' tiles need
#pragma nounroll
        for (int run = 0; run < 3; ++run) {
          const int from = run == 0 ? 0 : run == 1 ? runs.from : tiles.count, end = run == 0 ? runs.head : run == 1 ? runs.end : 0;
#pragma nounroll
          for (; t < from; ++t) {
            arrive();
            buf = (buf + 1) % NB;
          }
          if (t >= end) continue;
          scores(rb + buf * (2 * KT * DP * 2), less);
#pragma nounroll
          while (t + 1 < end) {
            turn(sa, da, sb, db);
            turn(sb, db, sa, da);
          }
          if (t < end) turn(sa, da, sb, db);
        }
      };
      if constexpr (FORM != OWN) walk(Const<FORM == FINE>{});
      else if (some_see_few(a, qt * BW + off, e1 + off, s.nk)) walk(Const<1>{});
      else walk(Const<0>{});
    }
    if (i < s.nq) {
      T* dQ = (T*)a.dq + batch_off(a, b, a.dqs[0]) + (s.q0 + i) * a.dqs[1] + (int64_t)h * a.dqs[2];
      const float f = le == -G10_NEG_INF ? 0.0f : a.scale / lift;
#pragma unroll
      for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int d = 32 * db + 8 * g + 4 * (int)(lane >> 5);
          if (d < (int)a.dim) {
            typename Vec<T>::x4 x;
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = (T)times(f, dq[db][4 * g + r]);
            *(typename Vec<T>::x4*)(dQ + d) = x;
          }
        }
    }
  }
  if (Lift<T>::ds && !lane) ((u32*)a.amax)[(((u64)unit * a.group + head) * a.tiles + first) * 4 + wave] = most;
}

// ---------------------------------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------------------------------
static uint64_t rows_of(const AttnArgs& a) { return (uint64_t)(a.q_start ? 1 : a.batch) * a.heads * a.seq_q; }

static uint64_t pad256(uint64_t x) { return (x + 255) / 256 * 256; }

// The workspace: the largest |do| of each wavefront of the queries' kernel; delta and lse2; a share's two pieces at most, what is cut.
static u32 query_tiles(const AttnArgs& a) { return tiles_in(a.batch * a.kv_heads, a.group, (a.max_q + BW - 1) / BW); }
static uint64_t top_bytes(const AttnArgs& a) { return pad256((uint64_t)a.batch * a.heads * query_tiles(a) * 16); }

// Shares for the keys' kernel, one to a place on a compute unit; 0: a workgroup to a tile. Cutting and joining cost 20 us, some 12 steps (of narrow heads
// 20); what they save is the longest tile's steps beyond a share's where every tile has a place of its own, and else about half of the longest
// tile's. Measured, forward and backward, a workgroup to a tile and shares: one sequence of 1000 tokens of 32 heads on 8 194 us and 119; 16 of 2048 of 32
// heads 3311 and 3148; 14 of 1490 with a window of 1 and 4 sinks 479 and 405; but 3 of 700 of 12 heads of 64 62 and 76, 8 of 600 of 8 heads 119 and
// 127. (Packed sequences go by their mean lengths, which are known here; max_q and max_k only cut the grid.)
static u32 key_shares(const AttnArgs& a) {
  const uint64_t nq = a.q_start ? ((uint64_t)a.seq_q + a.batch - 1) / a.batch : a.seq_q, nk = a.q_start ? ((uint64_t)a.seq_k + a.batch - 1) / a.batch : a.seq_k;
  const uint64_t near = a.window ? (uint64_t)a.window * (a.causal ? 1 : 2) + BW : nq;
  const uint64_t all = (nq + BT - 1) / BT * a.group, some = ((near < nq ? near : nq) + BT - 1) / BT * a.group;
  const uint64_t longest = a.window && !a.sinks ? some : all, mean = a.causal && !a.window ? (all + 1) / 2 : some;
  const uint64_t units = (uint64_t)a.batch * a.kv_heads, tiles = (nk + BW - 1) / BW, shares = a.dim <= 64 ? 512 : 256;
  if (!longest || !nk) return 0;
  const uint64_t each = units * (tiles * (mean + ENTRY) + longest - mean) / shares, share = each > SHARE ? each : SHARE;
  const uint64_t saved = units * tiles > shares ? longest / 2 : longest > share ? longest - share : 0;
  if (saved <= (a.dim <= 64 ? 20 : 12)) return 0;
  return (u32)shares;
}
static uint64_t share_bytes(const AttnArgs& a) { return (uint64_t)a.shares * (sizeof(Cut) + 4 * BW * (a.dim <= 64 ? 64 : 128) * 4); }

// As 16-bit numbers P and dS add about as much error to the gradients as those' own rounding, 1.41 times that in all; o's rounding in delta brings dq to 1.5
// times where few keys are seen, and with very few of them a single factor's rounding may rule a row.  So dq has both halves of dS in blocks of queries any of which sees up to 768
// keys (1.05 to 1.08 times its rounding, for one product of three more: 32 x 512 tokens of 12 heads of 64, 198 -> 204 us forward and backward; delta from
// P and dP up to there: 245), and dk and dv have those of dS and P in sequences of which no query sees more than 128.  What is decided goes by a sequence's own lengths alone;
// where these are known here, a kernel for them is taken.
static uint64_t keys_near(const AttnArgs& a) { return a.window ? (uint64_t)a.window * (a.causal ? 1 : 2) + a.sinks : ~0ull; }
static int form_dq(const AttnArgs& a) {
  if (keys_near(a) <= SOME || a.seq_k <= SOME) return FINE;
  if (a.q_start || a.k_len || (a.window && a.window <= SOME)) return OWN;
  if (!a.causal) return !a.window || a.seq_q <= a.seq_k ? PLAIN : OWN;
  return (int64_t)a.seq_k - a.seq_q + 1 > SOME ? PLAIN : OWN;
}
static int form_dkdv(const AttnArgs& a) {
  if (keys_near(a) <= FEWEST || a.seq_k <= FEWEST) return FINE;
  return a.q_start || a.k_len ? OWN : PLAIN;
}

template <class T, int DP>
static void launch_dq(const AttnArgs& a, int form, dim3 grid, hipStream_t s) {
  if (form == FINE) k_attn_dq<T, DP, FINE><<<grid, 256, 0, s>>>(a);
  else if (form == PLAIN) k_attn_dq<T, DP, PLAIN><<<grid, 256, 0, s>>>(a);
  else k_attn_dq<T, DP, OWN><<<grid, 256, 0, s>>>(a);
}

template <class T, int DP, int FORM>
static void launch_dkdv(const AttnArgs& a, dim3 grid, hipStream_t s) {
  if (a.shares) k_attn_dkdv<T, DP, FORM, true><<<grid, 256, 0, s>>>(a);
  else k_attn_dkdv<T, DP, FORM, false><<<grid, 256, 0, s>>>(a);
}
template <class T, int DP>
static void launch_dkdv(const AttnArgs& a, int form, dim3 grid, hipStream_t s) {
  if (form == FINE) launch_dkdv<T, DP, FINE>(a, grid, s);
  else if (form == PLAIN) launch_dkdv<T, DP, PLAIN>(a, grid, s);
  else launch_dkdv<T, DP, OWN>(a, grid, s);
}

extern "C" int g10_attention_backward_workspace(const g10_attention_args* g, uint64_t* bytes) {
  if (!bytes) return G10_EINVAL;
  AttnArgs a;
  G10_TRY(attn_args(g, true, a));
  if (!a.batch) { *bytes = 0; return G10_OK; }
  a.shares = key_shares(a);
  *bytes = top_bytes(a) + pad256(rows_of(a) * 8) + share_bytes(a);
  return G10_OK;
}

extern "C" int g10_attention_backward(const g10_attention_args* g, void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  AttnArgs a;
  G10_TRY(attn_args(g, true, a));
  if (!a.batch) return G10_OK;
  const uint64_t rows = rows_of(a);
  const u32 units = a.batch * a.kv_heads;
  a.shares = key_shares(a);
  if (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < top_bytes(a) + pad256(rows * 8) + share_bytes(a)) return G10_EINVAL;
  const u32 qt = a.q_tiles = query_tiles(a), kt = tiles_in(units, 1, (a.max_k + BW - 1) / BW);
  hipStream_t s = (hipStream_t)hip_stream;
  a.amax = (const u32*)workspace;
  a.delta = (const float*)((char*)workspace + top_bytes(a));
  a.lse2 = a.delta + rows;
  a.part = (float*)((char*)a.delta + pad256(rows * 8));
  a.cuts = (Cut*)(a.part + (uint64_t)a.shares * 4 * BW * (a.dim <= 64 ? 64 : 128));
  const bool narrow = a.dim <= 64, bf = g->type == G10_BF16;
  if (qt) {
    const int form = form_dq(a);
    a.tiles = qt;
    const dim3 grid(with_rest(a, unit_grid(units, a.group * a.tiles)));
    if (bf && narrow) launch_dq<__bf16, 64>(a, form, grid, s);
    else if (bf) launch_dq<__bf16, 128>(a, form, grid, s);
    else if (narrow) launch_dq<_Float16, 64>(a, form, grid, s);
    else launch_dq<_Float16, 128>(a, form, grid, s);
  }
  if (kt) {
    const int form = form_dkdv(a);
    a.tiles = kt;
    const dim3 grid(with_rest(a, a.shares ? a.shares : unit_grid(units, a.tiles)));
    if (bf && narrow) launch_dkdv<__bf16, 64>(a, form, grid, s);
    else if (bf) launch_dkdv<__bf16, 128>(a, form, grid, s);
    else if (narrow) launch_dkdv<_Float16, 64>(a, form, grid, s);
    else launch_dkdv<_Float16, 128>(a, form, grid, s);
  }
  if (kt && a.shares) {
    const dim3 grid(a.shares, 8);
    if (bf && narrow) k_attn_cuts<__bf16, 64><<<grid, 256, 0, s>>>(a);
    else if (bf) k_attn_cuts<__bf16, 128><<<grid, 256, 0, s>>>(a);
    else if (narrow) k_attn_cuts<_Float16, 64><<<grid, 256, 0, s>>>(a);
    else k_attn_cuts<_Float16, 128><<<grid, 256, 0, s>>>(a);
  }
  G10_HIP(hipGetLastError());
  return G10_OK;
}
