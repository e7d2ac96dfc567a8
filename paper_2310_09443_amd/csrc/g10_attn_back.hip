// Attention, backward:  delta = sum(do * o) per query, then one kernel for the gradients of keys and values and one for the
// queries'.  Both work P = 2^(S - lse) and dS = P (do V^T - delta) out again from q, k, v and the forward pass's lse.  Two
// kernels make seven products of the five that are needed; in return every gradient is summed by one wavefront in one order:
// no atomics, and nothing of the size of the scores in memory.
#include "g10_attn.h"

#define BT 64                      // rows of a staged tile
#define BW 128                     // rows of a workgroup, 32 to a wavefront

// In 16-bit floats with a short exponent, P and dS of long rows would fall below the smallest number.  P is held times
// 2^12 (it is at most 1), dS times 8 over the power of two at the largest |do|: both leave by exact powers of two at the end.
template <class T> struct Lift;
template <> struct Lift<__bf16> {
  static constexpr float p2 = 0.0f, p = 1.0f;
  static __device__ __forceinline__ float ds(const u32*) { return 1.0f; }
};
template <> struct Lift<_Float16> {
  static constexpr float p2 = 12.0f, p = 4096.0f;
  static __device__ __forceinline__ float ds(const u32* amax) {
    const int e = clampi((int)(*amax >> 23) - 127, -60, 60);
    return __uint_as_float((u32)(127 + 3 - e) << 23);
  }
};

__global__ void k_attn_clear(u32* x) { *x = 0; }

// delta, 16 lanes to a row; one read of do and o.
template <class T>
__global__ __launch_bounds__(256) void k_attn_delta(const AttnArgs a, u64 rows, u32* amax) {
  typedef typename Vec<T>::x8 x8;
  const u64 row = (u64)blockIdx.x * 16 + threadIdx.x / 16;
  const u32 c = threadIdx.x % 16;
  float sum = 0.0f, big = 0.0f;
  u64 at = 0;
  if (row < rows) {
    const u32 h = (u32)(row % a.heads);
    const u64 tok = row / a.heads;
    const u64 b = a.q_start ? 0 : tok / a.seq_q, i = a.q_start ? tok : tok % a.seq_q;
    at = (b * a.heads + h) * a.seq_q + i;
    if (c * 8 < a.dim) {
      const x8 x = *(const x8*)((const T*)a.d_o + (int64_t)b * a.dos[0] + (int64_t)i * a.dos[1] + (int64_t)h * a.dos[2] + c * 8);
      const x8 y = *(const x8*)((const T*)a.o + (int64_t)b * a.os[0] + (int64_t)i * a.os[1] + (int64_t)h * a.os[2] + c * 8);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        sum += (float)x[j] * (float)y[j];
        big = fmaxf(big, fabsf((float)x[j]));
      }
    }
  }
#pragma unroll
  for (int d = 8; d; d /= 2) sum += __shfl_xor(sum, d, 16);
  if (row < rows && !c) ((float*)a.delta)[at] = sum;
  if (amax) {
    const u32 top = wave_max(__float_as_uint(big));
    if (!lane_id() && top > __hip_atomic_load(amax, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) atomicMax(amax, top);
  }
}

// Gradients of 128 keys and values, 32 to a wavefront, which holds their rows and sums in registers and walks over the
// queries that see them, of all heads of the group:  S = Q K^T,  dP = dO V^T  come out with a key to a lane;
// dV^T += dO^T P,  dK^T += Q^T dS  read the tiles of queries once more, transposed.
template <class T, int DP>
__global__ __launch_bounds__(256) void k_attn_dkdv(const AttnArgs a) {
  __shared__ __attribute__((aligned(16))) T lds[2][2][BT * DP];
  __shared__ float row_lse[2][BT], row_delta[2][BT];
  typedef typename Vec<T>::x8 x8;
  u32 unit, at;
  if (!unit_of(a.batch * a.kv_heads, a.tiles, unit, at)) return;
  const u32 b = unit / a.kv_heads, hk = unit % a.kv_heads;
  const Seq s = seq_of(a, b);
  const int off = s.nk - s.nq;
  const u32 wave = uniform(wave_id()), lane = lane_id();
  const T* K = (const T*)a.k + batch_off(a, b, a.ks[0]) + s.k0 * a.ks[1] + (int64_t)hk * a.ks[2];
  const T* V = (const T*)a.v + batch_off(a, b, a.vs[0]) + s.k0 * a.vs[1] + (int64_t)hk * a.vs[2];
  T* dK = (T*)a.dk + batch_off(a, b, a.dks[0]) + s.k0 * a.dks[1] + (int64_t)hk * a.dks[2];
  T* dV = (T*)a.dv + batch_off(a, b, a.dvs[0]) + s.k0 * a.dvs[1] + (int64_t)hk * a.dvs[2];
  const int nk_all = a.q_start ? s.nk : (int)a.seq_k;                // rows of dk and dv to be written
  Stage<DP, BT, 256> sq, sd;
  sq.init(threadIdx.x, a.dim, a.qs[1]);
  sd.init(threadIdx.x, a.dim, a.dos[1]);
  const u32 lq[2] = {lds_addr(lds[0][0]) + wave * 1024, lds_addr(lds[1][0]) + wave * 1024};
  const u32 ld[2] = {lds_addr(lds[0][1]) + wave * 1024, lds_addr(lds[1][1]) + wave * 1024};
  const float lift = Lift<T>::ds(a.amax), lift_ds = lift / Lift<T>::p;
  for (int kt = (int)(at % a.tiles); kt * BW < nk_all; kt += (int)a.tiles) {
    const int j0 = kt * BW + (int)wave * 32, j = j0 + (int)(lane & 31);
    f32x16 dk[DP / 32] = {}, dv[DP / 32] = {};
    int lo = 0, hi = -1;                                             // queries that see any key of the workgroup
    const int e1 = (kt + 1) * BW < s.nk ? (kt + 1) * BW - 1 : s.nk - 1;
    if (kt * BW < s.nk) query_range(a, kt * BW, e1, s, lo, hi);
    if (hi >= lo) {
      const int wj1 = j0 + 31 < s.nk ? j0 + 31 : s.nk - 1;
      int wlo = 0, whi = -1, ilo = 0, ihi = -1;                      // ... of the wavefront, of the lane
      if (j0 < s.nk) query_range(a, j0, wj1, s, wlo, whi);
      if (j < s.nk) query_range(a, j, j, s, ilo, ihi);
      const u32 span = ihi >= ilo ? (u32)(ihi - ilo + 1) : 0u;
      x8 kf[DP / 16], vf[DP / 16];
      frags_global<T, DP>(kf, K, a.ks[1], j, s.nk - 1, a.dim);
      frags_global<T, DP>(vf, V, a.vs[1], j, s.nk - 1, a.dim);
      const int t0 = lo / BT, nt = hi / BT - t0 + 1, all = nt * (int)a.group;
      float mine = 0.0f;
      // what the thread brings of a tile's lse and delta
      auto fetch = [&](int t) {
        const u32 h = hk * a.group + (u32)(t / nt);
        const int i0 = (t0 + t % nt) * BT;
        const T* Q = (const T*)a.q + batch_off(a, b, a.qs[0]) + s.q0 * a.qs[1] + (int64_t)h * a.qs[2];
        const T* D = (const T*)a.d_o + batch_off(a, b, a.dos[0]) + s.q0 * a.dos[1] + (int64_t)h * a.dos[2];
        sq.load(Q, a.qs[1], i0, s.nq, lq[t & 1]);
        sd.load(D, a.dos[1], i0, s.nq, ld[t & 1]);
        if (threadIdx.x < 2 * BT) {
          const int i = i0 + (int)(threadIdx.x % BT), c = i < s.nq ? i : s.nq - 1;
          const int64_t r = row_off(a, b, h, s) + c;
          mine = threadIdx.x < BT ? a.lse[r] : a.delta[r];
        }
      };
      __syncthreads();
      fetch(0);
      for (int t = 0; t < all; ++t) {
        const int i0 = (t0 + t % nt) * BT, buf = t & 1;
        loads_done();
        if (threadIdx.x < BT) row_lse[buf][threadIdx.x] = mine * G10_LOG2E - Lift<T>::p2;
        else if (threadIdx.x < 2 * BT) row_delta[buf][threadIdx.x - BT] = mine;
        __syncthreads();
        if (t + 1 < all) fetch(t + 1);
        if (whi < i0 || wlo >= i0 + BT) continue;
        const T *tq = lds[buf][0], *td = lds[buf][1];
#pragma unroll
        for (int n = 0; n < BT / 32; ++n) {
          f32x16 sc = {}, dp = {};
#pragma unroll
          for (int ks = 0; ks < DP / 16; ++ks) sc = Vec<T>::mfma(frag_rows<T, DP>(tq, 32 * n, ks), kf[ks], sc);
#pragma unroll
          for (int ks = 0; ks < DP / 16; ++ks) dp = Vec<T>::mfma(frag_rows<T, DP>(td, 32 * n, ks), vf[ks], dp);
          const bool full = j0 + 31 < s.nk && i0 + 32 * n + 31 < s.nq &&
                            all_see(a, i0 + 32 * n + off, i0 + 32 * n + 31 + off, j0, j0 + 31, s.nk);
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const f32x4 le = *(const f32x4*)&row_lse[buf][32 * n + 8 * g + 4 * (lane >> 5)];
            const f32x4 de = *(const f32x4*)&row_delta[buf][32 * n + 8 * g + 4 * (lane >> 5)];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              float p = exp2_fast(sc[4 * g + r] * a.scale2 - le[r]);
              if (!full) p = (u32)(i0 + 32 * n + 8 * g + 4 * (int)(lane >> 5) + r - ilo) < span ? p : 0.0f;
              sc[4 * g + r] = p;
              dp[4 * g + r] = full || p != 0.0f ? p * (dp[4 * g + r] - de[r]) * lift_ds : 0.0f;
            }
          }
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const x8 pf = pack8<T>(sc, k), df = pack8<T>(dp, k);
#pragma unroll
            for (int db = 0; db < DP / 32; ++db) {
              dv[db] = Vec<T>::mfma(frag_tr<T, DP>(td, 32 * n + 16 * k, db), pf, dv[db]);
              dk[db] = Vec<T>::mfma(frag_tr<T, DP>(tq, 32 * n + 16 * k, db), df, dk[db]);
            }
          }
        }
      }
    }
    if (j < nk_all) {
      const float fk = a.scale / lift, fv = 1.0f / Lift<T>::p;
#pragma unroll
      for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int d = 32 * db + 8 * g + 4 * (int)(lane >> 5);
          if (d < (int)a.dim) {
            typename Vec<T>::x4 x, y;
#pragma unroll
            for (int r = 0; r < 4; ++r) { x[r] = (T)(dk[db][4 * g + r] * fk); y[r] = (T)(dv[db][4 * g + r] * fv); }
            *(typename Vec<T>::x4*)(dK + (int64_t)j * a.dks[1] + d) = x;
            *(typename Vec<T>::x4*)(dV + (int64_t)j * a.dvs[1] + d) = y;
          }
        }
    }
  }
}

// Gradients of 128 queries, 32 to a wavefront, as in the forward pass:  S^T = K Q^T,  dP^T = V dO^T  come out with a query
// to a lane;  dQ^T += K^T dS^T.
template <class T, int DP>
__global__ __launch_bounds__(256, 2) void k_attn_dq(const AttnArgs a) {
  __shared__ __attribute__((aligned(16))) T lds[2][2][BT * DP];
  typedef typename Vec<T>::x8 x8;
  u32 unit, at;
  if (!unit_of(a.batch * a.kv_heads, a.group * a.tiles, unit, at)) return;
  const u32 b = unit / a.kv_heads, hk = unit % a.kv_heads, h = hk * a.group + at / a.tiles;
  const Seq s = seq_of(a, b);
  const int off = s.nk - s.nq;
  const u32 wave = uniform(wave_id()), lane = lane_id();
  const T* Q = (const T*)a.q + batch_off(a, b, a.qs[0]) + s.q0 * a.qs[1] + (int64_t)h * a.qs[2];
  const T* D = (const T*)a.d_o + batch_off(a, b, a.dos[0]) + s.q0 * a.dos[1] + (int64_t)h * a.dos[2];
  const T* K = (const T*)a.k + batch_off(a, b, a.ks[0]) + s.k0 * a.ks[1] + (int64_t)hk * a.ks[2];
  const T* V = (const T*)a.v + batch_off(a, b, a.vs[0]) + s.k0 * a.vs[1] + (int64_t)hk * a.vs[2];
  T* dQ = (T*)a.dq + batch_off(a, b, a.dqs[0]) + s.q0 * a.dqs[1] + (int64_t)h * a.dqs[2];
  Stage<DP, BT, 256> sk, sv;
  sk.init(threadIdx.x, a.dim, a.ks[1]);
  sv.init(threadIdx.x, a.dim, a.vs[1]);
  const u32 lk[2] = {lds_addr(lds[0][0]) + wave * 1024, lds_addr(lds[1][0]) + wave * 1024};
  const u32 lv[2] = {lds_addr(lds[0][1]) + wave * 1024, lds_addr(lds[1][1]) + wave * 1024};
  const float lift = Lift<T>::ds(a.amax), lift_ds = lift;
  for (int qt = (int)(a.tiles - 1 - at % a.tiles); qt * BW < s.nq; qt += (int)a.tiles) {
    const int i0 = qt * BW + (int)wave * 32, i = i0 + (int)(lane & 31);
    const Seen seen = keys_of(a, i + off, s.nk);
    const int wp0 = i0 + off, wp1 = (i0 + 31 < s.nq ? i0 + 31 : s.nq - 1) + off;
    const int e1 = (qt + 1) * BW - 1 < s.nq ? (qt + 1) * BW - 1 : s.nq - 1;
    const Tiles tiles = key_tiles<BT>(a, qt * BW + off, e1 + off, s.nk);
    x8 q[DP / 16], dout[DP / 16];
    frags_global<T, DP>(q, Q, a.qs[1], i, s.nq - 1, a.dim);
    frags_global<T, DP>(dout, D, a.dos[1], i, s.nq - 1, a.dim);
    const int64_t r0 = row_off(a, b, h, s) + (i < s.nq ? i : s.nq - 1);
    const float le = a.lse[r0] * G10_LOG2E, de = a.delta[r0];
    f32x16 dq[DP / 32] = {};
    if (tiles.count) {
      __syncthreads();
      sk.load(K, a.ks[1], tiles.at(0) * BT, s.nk, lk[0]);
      sv.load(V, a.vs[1], tiles.at(0) * BT, s.nk, lv[0]);
    }
    for (int t = 0; t < tiles.count; ++t) {
      const int j0 = tiles.at(t) * BT, buf = t & 1;
      loads_done();
      __syncthreads();
      if (t + 1 < tiles.count) {
        sk.load(K, a.ks[1], tiles.at(t + 1) * BT, s.nk, lk[buf ^ 1]);
        sv.load(V, a.vs[1], tiles.at(t + 1) * BT, s.nk, lv[buf ^ 1]);
      }
      const T *tk = lds[buf][0], *tv = lds[buf][1];
      const bool full = all_see(a, wp0, wp1, j0, j0 + BT - 1, s.nk);
#pragma unroll
      for (int n = 0; n < BT / 32; ++n) {
        f32x16 sc = {}, dp = {};
#pragma unroll
        for (int ks = 0; ks < DP / 16; ++ks) sc = Vec<T>::mfma(frag_rows<T, DP>(tk, 32 * n, ks), q[ks], sc);
#pragma unroll
        for (int ks = 0; ks < DP / 16; ++ks) dp = Vec<T>::mfma(frag_rows<T, DP>(tv, 32 * n, ks), dout[ks], dp);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float p = exp2_fast(sc[r] * a.scale2 - le);
          if (!full) p = seen.key(j0 + 32 * n + res_row(r)) ? p : 0.0f;
          dp[r] = full || p != 0.0f ? p * (dp[r] - de) * lift_ds : 0.0f;
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const x8 df = pack8<T>(dp, k);
#pragma unroll
          for (int db = 0; db < DP / 32; ++db) dq[db] = Vec<T>::mfma(frag_tr<T, DP>(tk, 32 * n + 16 * k, db), df, dq[db]);
        }
      }
    }
    if (i < s.nq) {
      const float f = a.scale / lift;
#pragma unroll
      for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int d = 32 * db + 8 * g + 4 * (int)(lane >> 5);
          if (d < (int)a.dim) {
            typename Vec<T>::x4 w;
#pragma unroll
            for (int r = 0; r < 4; ++r) w[r] = (T)(dq[db][4 * g + r] * f);
            *(typename Vec<T>::x4*)(dQ + (int64_t)i * a.dqs[1] + d) = w;
          }
        }
    }
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------------------------------
static uint64_t rows_of(const AttnArgs& a) { return (uint64_t)(a.q_start ? 1 : a.batch) * a.heads * a.seq_q; }

extern "C" int g10_attention_backward_workspace(const g10_attention_args* g, uint64_t* bytes) {
  if (!bytes) return G10_EINVAL;
  AttnArgs a;
  G10_TRY(attn_args(g, true, a));
  *bytes = rows_of(a) * 4 + 256;                                     // delta, the largest |do|
  return G10_OK;
}

extern "C" int g10_attention_backward(const g10_attention_args* g, void* workspace, uint64_t workspace_bytes, void* hip_stream) {
  AttnArgs a;
  G10_TRY(attn_args(g, true, a));
  if (!a.batch) return G10_OK;
  const uint64_t rows = rows_of(a), units = (uint64_t)a.batch * a.kv_heads;
  if (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < rows * 4 + 256) return G10_EINVAL;
  const uint64_t qt = (a.max_q + BW - 1) / BW, kt = (a.max_k + BW - 1) / BW;
  if ((units + 7) * a.group * qt >= (1ull << 31) || (units + 7) * kt >= (1ull << 31) || rows / 16 >= (1ull << 31) - 1) return G10_EINVAL;
  hipStream_t s = (hipStream_t)hip_stream;
  a.amax = (const u32*)workspace;
  a.delta = (const float*)((char*)workspace + 256);
  u32* const amax = g->type == G10_F16 ? (u32*)workspace : nullptr;
  if (amax) k_attn_clear<<<1, 1, 0, s>>>(amax);
  if (rows) {
    const dim3 grid((u32)((rows + 15) / 16));
    if (g->type == G10_BF16) k_attn_delta<__bf16><<<grid, 256, 0, s>>>(a, rows, amax);
    else k_attn_delta<_Float16><<<grid, 256, 0, s>>>(a, rows, amax);
  }
  const bool narrow = a.dim <= 64, bf = g->type == G10_BF16;
  if (kt) {
    a.tiles = (u32)kt;
    const dim3 grid(unit_grid((u32)units, a.tiles));
    if (bf && narrow) k_attn_dkdv<__bf16, 64><<<grid, 256, 0, s>>>(a);
    else if (bf) k_attn_dkdv<__bf16, 128><<<grid, 256, 0, s>>>(a);
    else if (narrow) k_attn_dkdv<_Float16, 64><<<grid, 256, 0, s>>>(a);
    else k_attn_dkdv<_Float16, 128><<<grid, 256, 0, s>>>(a);
  }
  if (qt) {
    a.tiles = (u32)qt;
    const dim3 grid(unit_grid((u32)units, a.group * a.tiles));
    if (bf && narrow) k_attn_dq<__bf16, 64><<<grid, 256, 0, s>>>(a);
    else if (bf) k_attn_dq<__bf16, 128><<<grid, 256, 0, s>>>(a);
    else if (narrow) k_attn_dq<_Float16, 64><<<grid, 256, 0, s>>>(a);
    else k_attn_dq<_Float16, 128><<<grid, 256, 0, s>>>(a);
  }
  G10_HIP(hipGetLastError());
  return G10_OK;
}
