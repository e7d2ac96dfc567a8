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

struct Piece { float *o, *ml; };   // unfinished output of a row and a split: [dim] and {maximum, sum}

__device__ __forceinline__ Piece piece_of(const AttnArgs& a, u32 b, const Seq& s, int i, u32 h, u32 split) {
  const u64 row = ((a.q_start ? (u64)s.q0 : (u64)b * a.seq_q) + (u64)i) * a.heads + h;
  Piece p;
  p.o = a.part + (row * a.splits + split) * a.dim;
  p.ml = a.part_ml + (row * a.splits + split) * 2;
  return p;
}

template <class T, int DP>
__global__ __launch_bounds__(64 * SW) void k_attn_split(const AttnArgs a) {
  // [wavefront][buffer][keys, values]; afterwards the wavefronts' outputs
  __shared__ __attribute__((aligned(256))) T lds[SW][2][2][ST * DP];
  __shared__ float ms[SW][32], ls[SW][32];
  typedef typename Vec<T>::x8 x8;
  const u32 wave = uniform(wave_id()), lane = lane_id();
  u32 unit, at;
  if (!unit_of(a.batch * a.kv_heads, a.tiles * a.splits, unit, at)) return;
  const u32 b = unit / a.kv_heads, hk = unit % a.kv_heads, split = at % a.splits;
  const Seq s = seq_of(a, b);
  const int off = s.nk - s.nq, rows = s.nq * (int)a.group;
  const Unseen unseen = unseen_keys(a, s);
  const T* K = (const T*)a.k + batch_off(a, b, a.ks[0]) + s.k0 * a.ks[1] + (int64_t)hk * a.ks[2];
  const T* V = (const T*)a.v + batch_off(a, b, a.vs[0]) + s.k0 * a.vs[1] + (int64_t)hk * a.vs[2];
  Stage<DP, ST, 64> sk, sv;
  sk.init(lane, a.dim, a.ks[1]);
  sv.init(lane, a.dim, a.vs[1]);
  u32 lk[2], lv[2];
  for (int i = 0; i < 2; ++i) { lk[i] = lds_addr(lds[wave][i][0]); lv[i] = lds_addr(lds[wave][i][1]); }
  for (int rb = (int)(at / a.splits); rb * 32 < rows; rb += (int)a.tiles) {
    const int r0 = rb * 32, r1 = r0 + 31 < rows ? r0 + 31 : rows - 1;
    const int row = r0 + (int)(lane & 31), c = row < rows ? row : rows - 1;
    const int i = c / (int)a.group;
    const u32 h = hk * a.group + (u32)(c % (int)a.group);
    const Seen seen = keys_of(a, i + off, s.nk);
    const int p0 = r0 / (int)a.group + off, p1 = r1 / (int)a.group + off;
    const Tiles tiles = key_tiles<ST>(a, p0, p1, s.nk);
    const int t0 = (int)((int64_t)tiles.count * split / a.splits), t1 = (int)((int64_t)tiles.count * (split + 1) / a.splits);
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
        sc[r] = exp2_fast(sc[r] * a.scale2 - base);
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
      const Piece piece = piece_of(a, b, s, oi, oh, split);
      T* out = (T*)a.o + batch_off(a, b, a.os[0]) + (s.q0 + oi) * a.os[1] + (int64_t)oh * a.os[2];
      for (int d = (int)threadIdx.x % 8; d < (int)a.dim / 4; d += 8) {
        const float* src = (const float*)&lds[0][0][0][0] + col * DP + ((d ^ (col & 7)) << 2);
        f32x4 x = *(const f32x4*)src;
        for (int w = 1; w < SW; ++w) x += *(const f32x4*)(src + w * 32 * DP);
        if (a.splits > 1) *(f32x4*)(piece.o + 4 * d) = x;
        else {
          typename Vec<T>::x4 y;
          for (int r = 0; r < 4; ++r) y[r] = (T)times(inv, x[r]);
          *(typename Vec<T>::x4*)(out + 4 * d) = y;
        }
      }
      if (threadIdx.x % 8 == 0) {
        if (a.splits > 1) { piece.ml[0] = cm; piece.ml[1] = cl; }
        else (a.lse + row_off(a, b, oh, s))[oi] = cl > 0.0f ? (cm + __log2f(cl)) * G10_LN2 : cl == 0.0f ? G10_NEG_INF : cl;
      }
    }
    __syncthreads();                                                // (the next rows' tiles go where the parts lie)
  }
}

// A row's splits joined, a wavefront to a row, eight parts on their way at once: bound by the memory's latency (splits of
// 8 sequences of 32768 keys, 16 to a row: XX us; part by part it was 17).
template <class T>
__global__ __launch_bounds__(256) void k_attn_join(const AttnArgs a) {
  const u32 unit = blockIdx.x / a.tiles, b = unit / a.kv_heads, hk = unit % a.kv_heads, lane = lane_id();
  const Seq s = seq_of(a, b);
  const int rows = s.nq * (int)a.group;
  for (int r = (int)((blockIdx.x % a.tiles) * 4 + wave_id()); r < rows; r += (int)a.tiles * 4) {
    const int i = r / (int)a.group;
    const u32 h = hk * a.group + (u32)(r % (int)a.group);
    const Piece p = piece_of(a, b, s, i, h, 0);
    float big = G10_NEG_INF;
    for (u32 k = lane; k < a.splits; k += 64) big = fmaxf(big, p.ml[2 * k]);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) big = fmaxf(big, __shfl_xor(big, d, 64));
    float x0 = 0.0f, x1 = 0.0f, l = 0.0f;
    const bool has = 2 * lane < a.dim;
    for (u32 k0 = 0; k0 < a.splits; k0 += 64) {                      // a lane to a split for the weights, then a lane to two values
      const u32 n = a.splits - k0 < 64 ? a.splits - k0 : 64;
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
    if (!lane) (a.lse + row_off(a, b, h, s))[i] = l > 0.0f ? (big + __log2f(l)) * G10_LN2 : l == 0.0f ? G10_NEG_INF : l;
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------------------------------
// How many workgroups share a row's keys; 0: the work is not for these kernels.
//   - Up to 64 columns (a row's heads times its queries) half or more of a query tile of k_attn_fwd would be empty.
//   - The workgroups hold 128 KB of LDS each, one to a compute unit: four rounds of 256 even out sequences of unlike lengths.
//   - A split has 256 keys or more, two tiles for each wavefront: less does not pay for the joining.
// (Packed sequences go by their mean lengths, which are known here; max_q and max_k only cut the grid.)
u32 attn_splits(const AttnArgs& a) {
  const u64 nq = a.q_start ? ((u64)a.seq_q + a.batch - 1) / a.batch : a.seq_q, nk = a.q_start ? ((u64)a.seq_k + a.batch - 1) / a.batch : a.seq_k;
  const u64 cols = nq * a.group;
  if (cols > 64) return 0;
  u64 keys = nk;
  if (a.window) {
    const u64 near = (u64)a.window * (a.causal ? 1 : 2) + nq + a.sinks;
    if (near < keys) keys = near;
  }
  const u64 units = (u64)a.batch * a.kv_heads * ((cols + 31) / 32);
  u64 n = (1024 + units - 1) / units;
  const u64 most = (keys + 255) / 256;
  if (n > most) n = most;
  if (n > 512) n = 512;
  return n ? (u32)n : 1u;
}
u64 attn_split_bytes(const AttnArgs& a, u32 splits) {
  if (splits <= 1) return 0;
  const u64 rows = (u64)(a.q_start ? 1 : a.batch) * a.seq_q * a.heads;
  return rows * splits * (a.dim + 2) * 4;
}

template <class T>
static void launch(AttnArgs a, hipStream_t s) {
  const u32 units = a.batch * a.kv_heads;
  a.tiles = (u32)(((u64)a.max_q * a.group + 31) / 32);
  const dim3 grid(unit_grid(units, a.tiles * a.splits));
  if (a.dim <= 64) k_attn_split<T, 64><<<grid, 64 * SW, 0, s>>>(a);
  else k_attn_split<T, 128><<<grid, 64 * SW, 0, s>>>(a);
  if (a.splits > 1) {
    a.tiles = (u32)(((u64)a.max_q * a.group + 3) / 4);
    k_attn_join<T><<<units * a.tiles, 256, 0, s>>>(a);
  }
}

int attn_forward_split(AttnArgs a, u32 splits, void* workspace, u32 type, hipStream_t s) {
  a.splits = splits;
  const u64 rows = (u64)(a.q_start ? 1 : a.batch) * a.seq_q * a.heads;
  a.part = (float*)workspace;
  a.part_ml = splits > 1 ? a.part + rows * splits * a.dim : nullptr;
  if (type == G10_BF16) launch<__bf16>(a, s);
  else launch<_Float16>(a, s);
  G10_HIP(hipGetLastError());
  return G10_OK;
}
