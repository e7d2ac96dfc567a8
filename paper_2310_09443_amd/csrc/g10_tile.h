// Matrix products of 16-bit factors in tiles: C[m][n] = sum over k of A[m][k] B[k][n], summed in 32 bits.
//
// A workgroup of WM x WN wavefronts makes a tile of 32 TM WM rows by 64 WN columns, a wavefront 32 TM rows by twice 32 columns: 32 of the
// tile's first panel of 32 WN columns and the same 32 of its second one.  The panels of B need not lie side by side: a gated product takes
// one panel of each weight, and a value's two factors come out in one lane's registers.
//
// Both factors go through LDS in steps of KS = 64 or 32 along k, straight from memory (no registers), in panels of one of two layouts, as they
// lie in memory: rows of KS values along k (ALONG), read as fragments of 8 values, or KS rows of 128 or 64 values across (ACROSS), read
// with the transposing LDS read.  Both orders of k are the same, so any two layouts meet.  The places of 16-byte pieces in a row are exchanged
// so that each read takes all banks once.
//
// One barrier a step: behind it the step's panels are there (each wavefront has waited for its own loads) and the panels of the
// step before are read, so the loads of the step STAGES - 1 ahead go there at once and have as many steps to arrive.  A wavefront reads the
// fragments of the next 16 values of k while it multiplies the present ones; over the barrier it still multiplies the last ones of
// the step before.
#pragma once

#include "g10_attn.h"

// All but the wavefront's last N loads to LDS, and all its accesses to LDS.  (A barrier alone does not wait for reads whose values are used
// behind it; the other wavefronts' next loads go where they read.)
template <int N>
__device__ __forceinline__ void lds_settled() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | ((N >> 4) << 14));
  asm volatile("" ::: "memory");
}

enum { ALONG = 0, ACROSS = 1 };

// Exchanges of a row's pieces.
__device__ __forceinline__ u32 swz32(u32 r) { return (r >> 2) & 3; }                     // 4 pieces to a row of 32 values
__device__ __forceinline__ u32 swz64(u32 r) { return (r >> 1) & 7; }                     // 8 pieces to a row of 64
__device__ __forceinline__ u32 swz64a(u32 r) { return ((r & 2) << 1) | ((r >> 2) & 3); } // 8 pieces to a row of 64 across, read transposed
__device__ __forceinline__ u32 swz128(u32 r) { return ((r & 3) << 2) | ((r >> 2) & 3); } // 16 pieces to a row of 128

// A panel of ROWS places across (KS values of k each) by NT threads: what each loads, and where it looks.
template <int LAYOUT, int ROWS, int NT, int KS>
struct Panel {
  static constexpr int PIECES = ROWS * KS / 8, IT = PIECES / NT, BYTES = PIECES * 16;
  static_assert(PIECES % NT == 0, "whole rounds");
  static constexpr int PER = LAYOUT == ALONG ? KS / 8 : ROWS / 8;                        // pieces to a row in LDS
  static __device__ __forceinline__ u32 swz(u32 row) { return LAYOUT == ACROSS ? (ROWS == 128 ? swz128(row) : swz64a(row)) : KS == 64 ? swz64(row) : swz32(row); }
  static_assert(LAYOUT == ALONG || ROWS == 128 || ROWS == 64, "rows of 128 or 64 across");
  u32 off[IT];
  u32 k[IT];                       // the first value of k of each piece
  // first, n: the panel's first place across, and how many there are in all (places past them repeat the last row or piece: who uses them
  // does not keep what comes of it)
  __device__ __forceinline__ void init(u32 t, int64_t stride, u32 first, u32 n) {
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const u32 p = i * NT + t, row = p / PER, place = p % PER;
      if (LAYOUT == ALONG) {
        const u32 c = place ^ swz(row), left = n - first, r = row < left ? row : left - 1;
        off[i] = (u32)((int64_t)r * stride + c * 8) * 2;
        k[i] = c * 8;
      } else {
        u32 c = place ^ swz(row);
        if (first + c * 8 >= n) c = 0;
        off[i] = (u32)((int64_t)row * stride + c * 8) * 2;
        k[i] = row;
      }
    }
  }
  // Where the panel at `first` and step `step` lies in an operand: rows [across][k] with ALONG, [k][across] with ACROSS.
  static __device__ __forceinline__ const char* start(const void* p, int64_t stride, u32 first, u32 step) {
    return (const char*)p + (LAYOUT == ALONG ? (int64_t)first * stride : (int64_t)first) * 2 + step * bytes(stride);
  }
  static __device__ __forceinline__ int64_t bytes(int64_t stride) { return (LAYOUT == ALONG ? (int64_t)KS : KS * stride) * 2; }
  // lds: the panel + this wavefront's first piece
  __device__ __forceinline__ void load(int i, const char* at, u32 lds) const { load_piece(at, off[i], lds + (u32)(i * NT * 16)); }
  // left: values of k from the step's first on; pieces past them become zeros
  __device__ __forceinline__ void load_short(int i, const char* at, u32 lds, u32 left) const {
    if (k[i] < left) load_piece(at, off[i], lds + (u32)(i * NT * 16));
    else *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(lds + (u32)(i * NT * 16) + lane_id() * 16) = u32x4{};
  }
  // The base address of a lane's fragments.
  static __device__ __forceinline__ u32 base(u32 panel) {
    const u32 l = lane_id();
    if (LAYOUT == ALONG) return panel + (l & 31) * (KS * 2) + (((l >> 5) ^ swz(l & 31)) << 4);
    const u32 row = 8 * (l >> 5) + ((l & 15) >> 2), c = 2 * ((l >> 4) & 1) + ((l & 3) >> 1);
    return panel + row * (ROWS * 2) + ((c ^ swz(row)) << 4) + (l & 1) * 8;
  }
  // 32 places from 32 blk on, values 16 kk + 8 (l / 32) + 0..7 of k
  template <class T>
  static __device__ __forceinline__ typename Vec<T>::x8 frag(u32 base, int blk, int kk) {
    if constexpr (LAYOUT == ALONG) {
      return *(__attribute__((address_space(3))) const typename Vec<T>::x8*)(uintptr_t)((base ^ (u32)(kk << 5)) + (u32)(blk * 32 * KS * 2));
    } else {
      const u32 at = base ^ (u32)(blk << 6);
      const typename Vec<T>::x4 a = Vec<T>::read_tr(at + (u32)(kk * 16 * ROWS * 2)), b = Vec<T>::read_tr((at ^ 16) + (u32)((kk * 16 + 4) * ROWS * 2));
      return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }
};

// The sums of one tile.  acc[j][i]: panel j, rows 32 i of the wavefront; lane l holds row l % 32, columns res_row(r).
template <class T, int LA, int LB, int WM, int WN, int TM, int KS, int STAGES>
struct Tile {
  static constexpr int NT = 64 * WM * WN, BM = 32 * TM * WM, WIDE = 32 * WN;
  static constexpr int AROWS = LA == ALONG ? BM : 128, APANELS = BM / AROWS;
  typedef Panel<LA, AROWS, NT, KS> PA;
  typedef Panel<LB, WIDE, NT, KS> PB;
  static constexpr int A_BYTES = APANELS * PA::BYTES, STAGE = A_BYTES + 2 * PB::BYTES, LDS = STAGES * STAGE;
  static constexpr int LOADS = APANELS * PA::IT + 2 * PB::IT;                            // of a wavefront and step
  typedef typename Vec<T>::x8 x8;

  // Where the next step's panels lie.
  struct Walk {
    const char *a[APANELS], *b[2];
    u32 left;                      // values of k still to load of this source
  };

  // `steps` steps; sa, sb: bytes from one to the next.  next(w) is called where a source has no more values of k.  whole: no step but the last one is a
  // short one (a wavefront with nothing to load for its zeros has fewer loads to count).
  template <class NEXT>
  static __device__ __forceinline__ void run(f32x16 (&acc)[2][TM], u32 lds0, int steps, const PA (&pa)[APANELS], const PB (&pb)[2], Walk w, int64_t sa, int64_t sb,
                                             bool whole, NEXT&& next) {
    const u32 wave = uniform(wave_id()), wm = wave / WN, wn = wave % WN;
    int loaded = 0;
    u32 to = lds0;
    // one load of a step's LOADS; the last one goes on to the next step
    auto load = [&](int n) {
      const u32 at = to + wave * 1024;
#pragma unroll
      for (int i = 0; i < APANELS; ++i)
        if (n / PA::IT == i && n < APANELS * PA::IT) pa[i].load(n % PA::IT, w.a[i], at + i * PA::BYTES);
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (n >= APANELS * PA::IT && (n - APANELS * PA::IT) / PB::IT == j) pb[j].load((n - APANELS * PA::IT) % PB::IT, w.b[j], at + A_BYTES + j * PB::BYTES);
    };
    auto load_short = [&]() {
      const u32 at = to + wave * 1024;
#pragma unroll
      for (int i = 0; i < APANELS; ++i)
#pragma unroll
        for (int n = 0; n < PA::IT; ++n) pa[i].load_short(n, w.a[i], at + i * PA::BYTES, w.left);
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int n = 0; n < PB::IT; ++n) pb[j].load_short(n, w.b[j], at + A_BYTES + j * PB::BYTES, w.left);
    };
    auto loaded_one = [&]() {
#pragma unroll
      for (int i = 0; i < APANELS; ++i) w.a[i] += sa;
#pragma unroll
      for (int j = 0; j < 2; ++j) w.b[j] += sb;
      if (w.left > KS) w.left -= KS; else next(w);
      ++loaded;
      to = to + STAGE < lds0 + LDS ? to + STAGE : lds0;
    };
    const u32 a_off = LA == ALONG ? wm * (32 * TM * KS * 2) : ((wm * TM * 32) / 128) * (u32)PA::BYTES, a_blk = LA == ALONG ? 0 : (wm * TM) % 4;
    const u32 ab = PA::base(lds0 + a_off) ^ (a_blk << 6), bb = PB::base(lds0 + A_BYTES) ^ (LB == ALONG ? 0 : wn << 6);
    const u32 b_off = LB == ALONG ? wn * (32 * KS * 2) : 0;
    x8 fa[2][TM] = {}, fb[2][2] = {};
    auto read = [&](int s, u32 at, int kk) {
#pragma unroll
      for (int j = 0; j < 2; ++j) fb[s][j] = PB::template frag<T>(bb + at + b_off + j * PB::BYTES, 0, kk);
#pragma unroll
      for (int i = 0; i < TM; ++i) fa[s][i] = PA::template frag<T>(ab + at, i, kk);
    };
    auto multiply = [&](int s) {
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[j][i] = Vec<T>::mfma(fb[s][j], fa[s][i], acc[j][i]);
    };
    for (int i = 0; i < STAGES - 1 && loaded < steps; ++i) {
      if (w.left >= KS) {
#pragma unroll
        for (int n = 0; n < LOADS; ++n) load(n);
      } else {
        load_short();
      }
      loaded_one();
    }
    u32 from = 0;
    for (int step = 0; step < steps; ++step) {
      // (fewer loads are on their way at the end: all are waited for there)
      if (STAGES > 2 && whole && loaded < steps) lds_settled<LOADS * (STAGES - 2)>(); else lds_settled<0>();
      __syncthreads();
      read(0, from, 0);
      hold();
      // the last products of the step before (at first of zeros), with the next loads between them: a wavefront that issues all loads at a stretch
      // leaves the matrix unit without work
      const bool more = loaded < steps, full = more && w.left >= KS;
      if (more && !full) load_short();
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        if (full) {
#pragma unroll
          for (int n = i * LOADS / TM; n < (i + 1) * LOADS / TM; ++n) load(n);
        }
        hold();
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[j][i] = Vec<T>::mfma(fb[1][j], fa[1][i], acc[j][i]);
        hold();
      }
      if (more) loaded_one();
#pragma unroll
      for (int kk = 1; kk < KS / 16; ++kk) {
        hold();
        read(kk & 1, from, kk);
        hold();
        multiply((kk & 1) ^ 1);
      }
      hold();
      from = from + STAGE < LDS ? from + STAGE : 0;
    }
    if (steps) multiply(1);
  }
};
