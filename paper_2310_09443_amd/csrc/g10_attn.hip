// Attention, forward.
#include "g10_attn.h"

#define BN 64                      // keys of a tile

// Forward pass.  A wavefront holds 32 queries in registers and walks over the keys they see, 64 at a time, with a running
// maximum m and sum l of the softmax:  S = K Q^T,  P = 2^(S - m),  O^T = O^T 2^(m' - m) + V^T P.  S comes out transposed
// (a lane holds one query's scores), so the row's maximum and sum are sums over registers and one exchange of the two halves,
// and P feeds the second product as it lies in the registers.
// A tile's exponentials take the vector unit as long as its products take the matrix unit, so each wavefront works on both at
// once: the scores of the next tile and the outputs of this one, product by product, with the exponentials of this tile
// strewn between and the fragments of the products four ahead on their way from LDS.  hold() keeps the compiler from putting
// these apart again.

// P is rounded to 16 bits for the second product. A 16-bit float with a short exponent has its smallest normal number at 2^-14, so P is held times
// 2^LIFT there, and the maximum that it is relative to may lag by LAG less: 2^(LAG + LIFT) is below the largest number, and a key keeps
// all its bits down to 2^-26 of the row's largest (18 nats: a first token that takes nearly all of a row, and thousands of keys that share the
// rest). l sums P as it is held; the lift leaves with 1 / l, and from lse.  Lagging by 2^3 in place of 2^8 costs 1 to 3 % in heads of 64 (3 x 700 tokens of 12 heads,
// forward and backward, 60.6 -> 62.8 us; 32 x 512 202.8 -> 204.0).
template <class T> struct Hold;
template <> struct Hold<__bf16> { static constexpr float lift = 0.0f, drop = 1.0f, lag = 8.0f; };
template <> struct Hold<_Float16> { static constexpr float lift = 12.0f, drop = 0x1p-12f, lag = 3.0f; };

// The products of a tile, in order: NS of the next tile's scores (none if !NEXT), NV of this tile's outputs.
template <class T, int DP, bool NEXT>
__device__ __forceinline__ void tile_step(u32 tk, u32 tv, const typename Vec<T>::x8 (&q)[DP / 16], f32x16 (&sc)[2], f32x16 (&sn)[2],
                                          f32x16 (&o)[DP / 32], float scale2, float base, float& l) {
  typedef typename Vec<T>::x8 x8;
  constexpr int NS = NEXT ? 2 * DP / 16 : 0, NV = 4 * DP / 32, N = NS + NV, DB = DP / 32, AHEAD = 4, RING = 5;
  // exponentials of the first 32 keys before the first output's product, of the others before the second half's
  constexpr int EARLY = NEXT ? 20 : 16;
  x8 f[RING], pf[4];
  float sum[4] = {};
  auto read = [&](int e) -> x8 {
    return e < NS ? frag_rows<T, DP>(tk, e % 2 * 32, e / 2) : frag_tr<T, DP>(tv, (e - NS) / DB * 16, (e - NS) % DB);
  };
  auto exps = [&](int from, int to) {
#pragma unroll
    for (int x = from; x < to; ++x) {
      const int n = x / 16, r = x % 16;
      sc[n][r] = exp2_fast(sc[n][r] * scale2 - base);
      sum[r & 3] += sc[n][r];
      if (r % 8 == 7) pf[x / 8] = pack8<T>(sc[n], r / 8);
    }
  };
#pragma unroll
  for (int e = 0; e < AHEAD; ++e) f[e % RING] = read(e);
  hold();
  if (!NEXT) { exps(0, EARLY); hold(); }
#pragma unroll
  for (int e = 0; e < N; ++e) {
    if (e + AHEAD < N) f[(e + AHEAD) % RING] = read(e + AHEAD);
    if (e < NS) {
      if (e < 2) sn[e] = f32x16{};
      sn[e % 2] = Vec<T>::mfma(f[e % RING], q[e / 2], sn[e % 2]);
      exps(EARLY * e / (NS ? NS : 1), EARLY * (e + 1) / (NS ? NS : 1));
    } else {
      const int v = e - NS;
      o[v % DB] = Vec<T>::mfma(f[e % RING], pf[v / DB], o[v % DB]);
      if (v < NV / 2) exps(EARLY + (32 - EARLY) * v / (NV / 2), EARLY + (32 - EARLY) * (v + 1) / (NV / 2));
    }
    hold();
  }
  l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

// NW wavefronts to a workgroup, 32 queries each.
template <class T, int DP, int NW>
__global__ __launch_bounds__(64 * NW, DP == 64 ? 3 : 2) void k_attn_fwd(const AttnArgs a) {
  constexpr int BM = 32 * NW;
  __shared__ __attribute__((aligned(256))) T lds[2][2][BN * DP];      // keys, values; even and odd tiles
  typedef typename Vec<T>::x8 x8;
  if (blockIdx.x >= a.work) { clear_outputs<T>(a); return; }
  u32 unit, head, last;
  if (!block_of(a.batch * a.kv_heads, a.group, a.tiles, unit, head, last)) return;
  const u32 b = unit / a.kv_heads, hk = unit % a.kv_heads, h = hk * a.group + head;
  const Seq s = seq_of(a, b);
  const int off = s.nk - s.nq;
  const Unseen unseen = unseen_keys(a, s);
  const u32 wave = uniform(wave_id()), lane = lane_id();
  const T* Q = (const T*)a.q + batch_off(a, b, a.qs[0]) + s.q0 * a.qs[1] + (int64_t)h * a.qs[2];
  const T* K = (const T*)a.k + batch_off(a, b, a.ks[0]) + s.k0 * a.ks[1] + (int64_t)hk * a.ks[2];
  const T* V = (const T*)a.v + batch_off(a, b, a.vs[0]) + s.k0 * a.vs[1] + (int64_t)hk * a.vs[2];
  Stage<DP, BN, 64 * NW> sk, sv;
  sk.init(threadIdx.x, a.dim, a.ks[1]);
  sv.init(threadIdx.x, a.dim, a.vs[1]);
  const u32 lk = lds_addr(lds[0][0]) + wave * 1024, lv = lds_addr(lds[1][0]) + wave * 1024;
  constexpr u32 odd = BN * DP * 2;
  const u32 tk = rows_base<DP>(lds_addr(lds[0][0])), tv = cols_base<DP>(lds_addr(lds[1][0]));
  bool again = false;
  for (int qt = (int)last; qt * BM < s.nq; qt += (int)a.tiles) {
    const int i0 = qt * BM + (int)wave * 32, i = i0 + (int)(lane & 31);
    const Seen seen = keys_of(a, i + off, s.nk);
    const int wp0 = i0 + off, wp1 = (i0 + 31 < s.nq ? i0 + 31 : s.nq - 1) + off;       // the wavefront's positions
    const int e1 = (qt + 1) * BM - 1 < s.nq ? (qt + 1) * BM - 1 : s.nq - 1;
    const Tiles tiles = key_tiles<BN>(a, qt * BM + off, e1 + off, s.nk);
    f32x16 o[DP / 32] = {};
    float m = G10_NEG_INF, l = 0.0f;                                 // m in powers of two
    if (tiles.count) {
      if (again) __syncthreads();                                    // (the tiles of the queries before are read)
      again = true;
      sk.load(K, a.ks[1], tiles.at(0) * BN, s.nk, unseen, lk);
      sv.load(V, a.vs[1], tiles.at(0) * BN, s.nk, unseen, lv);
      x8 q[DP / 16];
      frags_global<T, DP>(q, Q, a.qs[1], i, s.nq - 1, a.dim);
      f32x16 sa[2], sb[2];
      // scores of a tile that are not seen leave; the maximum
      auto settle = [&](f32x16(&sc)[2], int t) {
        const int j0 = tiles.at(t) * BN;
        if (!all_see(a, wp0, wp1, j0, j0 + BN - 1, s.nk)) {
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[n][r] = seen.key(j0 + 32 * n + res_row(r)) ? sc[n][r] : G10_NEG_INF;
        }
        float top = sc[0][0];
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int r = 0; r < 16; ++r) top = fmaxf(top, sc[n][r]);
        top = both_max(top) * a.scale2;
        // The sums stay relative to an older maximum until it is passed by more than 2^LAG: what is added then is below 2^(LAG + LIFT), far from
        // the type's end, and most tiles leave the outputs as they are.
        if (ballot(top > m + Hold<T>::lag)) {
          const float now = fmaxf(m, top), fade = exp2_fast(m - (now == G10_NEG_INF ? 0.0f : now));
          m = now;
          l *= fade;
#pragma unroll
          for (int db = 0; db < DP / 32; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[db][r] *= fade;
        }
      };
      loads_done();
      __syncthreads();
      if (tiles.count > 1) sk.load(K, a.ks[1], tiles.at(1) * BN, s.nk, unseen, lk + odd);
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        sa[n] = f32x16{};
#pragma unroll
        for (int ks = 0; ks < DP / 16; ++ks) sa[n] = Vec<T>::mfma(frag_rows<T, DP>(tk, 32 * n, ks), q[ks], sa[n]);
      }
      settle(sa, 0);
      // tile t: its scores lie in sc; the next tile's keys and this one's values are in LDS, the ones behind them on their way
      auto turn = [&](f32x16(&sc)[2], f32x16(&sn)[2], int t, u32 even, u32 other) {
        loads_done();
        __syncthreads();
        if (t + 2 < tiles.count) sk.load(K, a.ks[1], tiles.at(t + 2) * BN, s.nk, unseen, lk + even);
        sv.load(V, a.vs[1], tiles.at(t + 1) * BN, s.nk, unseen, lv + other);
        tile_step<T, DP, true>(tk + other, tv + even, q, sc, sn, o, a.scale2, (m == G10_NEG_INF ? 0.0f : m) - Hold<T>::lift, l);
        settle(sn, t + 1);
      };
      int t = 0;
      for (; t + 2 < tiles.count; t += 2) {
        turn(sa, sb, t, 0, odd);
        turn(sb, sa, t + 1, odd, 0);
      }
      if (t + 1 < tiles.count) {
        turn(sa, sb, t, 0, odd);
        sa[0] = sb[0];
        sa[1] = sb[1];
        ++t;
      }
      loads_done();
      __syncthreads();
      tile_step<T, DP, false>(0, tv + (t & 1 ? odd : 0), q, sa, sb, o, a.scale2, (m == G10_NEG_INF ? 0.0f : m) - Hold<T>::lift, l);
    }
    l = both_sum(l);
    if (i < s.nq) {
      T* out = (T*)a.o + batch_off(a, b, a.os[0]) + (s.q0 + i) * a.os[1] + (int64_t)h * a.os[2];
      const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;  // (l is NaN where a score is)
#pragma unroll
      for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int d = 32 * db + 8 * g + 4 * (int)(lane >> 5);
          if (d < (int)a.dim) {
            typename Vec<T>::x4 w;
#pragma unroll
            for (int r = 0; r < 4; ++r) w[r] = (T)times(inv, o[db][4 * g + r]);
            *(typename Vec<T>::x4*)(out + d) = w;
          }
        }
      if (lane < 32) (a.lse + row_off(a, b, h, s))[i] = l > 0.0f ? (m + __log2f(l * Hold<T>::drop)) * G10_LN2 : l == 0.0f ? G10_NEG_INF : l;
    }
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------------------------------
static bool aligned(const void* p, const int64_t* st, bool batch) {
  if (!p || ((uintptr_t)p & 15)) return false;
  for (int i = batch ? 0 : 1; i < 3; ++i)
    if (st[i] & 7) return false;
  return st[1] >= 0 && st[1] <= (1 << 22);
}

int attn_args(const g10_attention_args* g, bool back, AttnArgs& a) {
  if (!g) return G10_EINVAL;
  if (g->type != G10_F16 && g->type != G10_BF16) return G10_EINVAL;
  if (!g->dim || g->dim % 8 || g->dim > 128) return G10_EINVAL;
  if (!g->kv_heads || !g->heads || g->heads % g->kv_heads || g->heads > 65536) return G10_EINVAL;
  if ((g->q_start == nullptr) != (g->k_start == nullptr) || (g->q_start && g->k_len)) return G10_EINVAL;
  if (!(g->scale > 0.0f) || !(g->scale < 3e38f)) return G10_EINVAL;
  if (g->causal > 1 || g->seq_q >= (1u << 30) || g->seq_k >= (1u << 30) || g->window >= (1u << 30) || g->sinks >= (1u << 30)) return G10_EINVAL;
  if (g->max_q >= (1u << 30) || g->max_k >= (1u << 30)) return G10_EINVAL;
  if (((uint64_t)g->batch * g->kv_heads + 7) / 8 * 8 * (g->heads / g->kv_heads) + REST > G10_GROUPS_MOST) return G10_EINVAL;   // (a workgroup for each head at least)
  const bool packed = g->q_start != nullptr;
  a = AttnArgs{};
  a.q = g->q; a.k = g->k; a.v = g->v; a.o = g->o; a.lse = g->lse; a.d_o = g->d_o; a.dq = g->dq; a.dk = g->dk; a.dv = g->dv;
  for (int i = 0; i < 3; ++i) {
    a.qs[i] = g->q_stride[i]; a.ks[i] = g->k_stride[i]; a.vs[i] = g->v_stride[i]; a.os[i] = g->o_stride[i];
    a.dos[i] = g->do_stride[i]; a.dqs[i] = g->dq_stride[i]; a.dks[i] = g->dk_stride[i]; a.dvs[i] = g->dv_stride[i];
  }
  a.q_start = g->q_start; a.k_start = g->k_start; a.k_len = g->k_len;
  a.batch = g->batch; a.heads = g->heads; a.kv_heads = g->kv_heads; a.group = g->heads / g->kv_heads; a.dim = g->dim;
  a.seq_q = g->seq_q; a.seq_k = g->seq_k;
  a.max_q = packed ? (g->max_q < g->seq_q ? g->max_q : g->seq_q) : g->seq_q;
  a.max_k = packed ? (g->max_k < g->seq_k ? g->max_k : g->seq_k) : g->seq_k;
  if (packed && g->seq_q && !a.max_q) a.max_q = 1;
  if (packed && g->seq_k && !a.max_k) a.max_k = 1;
  a.causal = g->causal; a.window = g->window; a.sinks = g->sinks;
  a.scale = g->scale; a.scale2 = g->scale * G10_LOG2E;
  const bool some_q = g->batch && g->seq_q, some_k = g->batch && g->seq_k;
  if (some_q && (!aligned(g->q, g->q_stride, !packed) || !aligned(g->o, g->o_stride, !packed) || !g->lse)) return G10_EINVAL;
  if (some_k && (!aligned(g->k, g->k_stride, !packed) || !aligned(g->v, g->v_stride, !packed))) return G10_EINVAL;
  if (back) {
    if (some_q && (!aligned(g->d_o, g->do_stride, !packed) || !aligned(g->dq, g->dq_stride, !packed))) return G10_EINVAL;
    if (some_k && (!aligned(g->dk, g->dk_stride, !packed) || !aligned(g->dv, g->dv_stride, !packed))) return G10_EINVAL;
  }
  return G10_OK;
}

extern "C" int g10_attention_workspace(const g10_attention_args* g, uint64_t* bytes) {
  if (!bytes) return G10_EINVAL;
  AttnArgs a;
  G10_TRY(attn_args(g, false, a));
  *bytes = a.batch && a.seq_q ? attn_split_bytes(a, attn_splits(a)) : 0;
  return G10_OK;
}

extern "C" int g10_attention(const g10_attention_args* g, void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  AttnArgs a;
  G10_TRY(attn_args(g, false, a));
  if (!a.batch || !a.seq_q) return G10_OK;
  hipStream_t s = (hipStream_t)hip_stream;
  if (const u32 splits = attn_splits(a)) {
    const u64 need = attn_split_bytes(a, splits);
    if (need && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < need)) return G10_EINVAL;
    return attn_forward_split(a, splits, workspace, g->type, s);
  }
  constexpr int nw = 4;
  const u32 units = a.batch * a.kv_heads;
  a.tiles = tiles_in(units, a.group, (a.max_q + 32 * nw - 1) / (32 * nw));
  const dim3 grid(with_rest(a, unit_grid(units, a.group * a.tiles)));
  if (g->type == G10_BF16) {
    if (a.dim <= 64) k_attn_fwd<__bf16, 64, nw><<<grid, 64 * nw, 0, s>>>(a);
    else k_attn_fwd<__bf16, 128, nw><<<grid, 64 * nw, 0, s>>>(a);
  } else {
    if (a.dim <= 64) k_attn_fwd<_Float16, 64, nw><<<grid, 64 * nw, 0, s>>>(a);
    else k_attn_fwd<_Float16, 128, nw><<<grid, 64 * nw, 0, s>>>(a);
  }
  G10_HIP(hipGetLastError());
  return G10_OK;
}
