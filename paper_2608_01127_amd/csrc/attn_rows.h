// Attention of the rows of one key head over a list of keys that is not the rows' own
// sequence: cross attention (an encoder's states) and cached attention over pages of
// 8-bit keys and values (gfx950).
//
// Rows.  The G = H / Hkv query heads of a key head share its keys, so they are the rows
// of one tile: row r of key head hk is token r / G of query head hk G + r % G.  With one
// token and G heads a tile then reads the keys once for all of them.
//
// Keys.  A workgroup visits key steps of BK keys: cached tokens of its sequence (PAGED) and
// bf16 keys (the states, or the queued tokens' own keys).  Each kind starts a step of its
// own and its last step may be partly filled.  The steps that every row sees whole come
// first, cached ones, then bf16 ones; then the partly filled cached step and the bf16 steps
// that some rows see in part.  Rows of a staged tile behind the last key repeat it (codes at
// D = 72: zeros), so that nothing behind the data is read and the masked products meet
// finite values.  D = 72 contracts 80 columns: the last eight of a key row in LDS are the
// next row's first ones, against zeros in Q, so that a key a row does not see has to be
// finite as its value has.
//
// Cached tokens are e4m3 codes with a power-of-two scale for each 64 tokens and head: a
// step never straddles a page, and a code times its scale is exact in bf16, so a tile is
// converted once on its way into LDS (global load, v_cvt_scalef32_pk_bf16_fp8, LDS
// write) and the products are the bf16 ones on the cache's very values.
#pragma once

#include <type_traits>

#include "mw_device.h"
#include "mw_kernels.h"

namespace mw {

typedef int i32x2 __attribute__((ext_vector_type(2)));

// Sequence of each batch member (paged calls), by value: a call keeps no memory of the caller's.
template <bool PAGED>
struct RowsSeqs {
  int seq[PAGED ? kMaxSeqs : 1];
};

// Address of row r of key head hk in a [B, H, T, D] view.
__device__ __forceinline__ long long row_offset(const Strides& s, int b, int hk, int G, int r) {
  const int t = G == 1 ? r : (int)((unsigned)r / (unsigned)G);
  return b * s.b + (long long)(hk * G + (r - t * G)) * s.h + t * s.t;
}

// Barrier that waits for this wave's LDS accesses and leaves its global loads in flight.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// A wave's 32 x D result (accumulator layout: lane l, register i of block db holds column 32 db + 8 (i / 4) +
// 4 (l / 32) + i % 4 of row l % 32; at D = 72 `tail` holds the last eight) as bf16 rows in memory, by way of `x`, the
// wave's own 32 rows of an LDS tile: 16 bytes a lane, whole rows at once.  Storing from the accumulators, 8 bytes a
// lane and 16 to a row, cost 10 of 51 us at 12 heads x 19200 rows x 128 keys (D = 128).  `mul` scales the lane's row;
// `row_ptr(r)` is the address of row r of the block, of which there are n.
template <int D, class RowPtr>
__device__ __forceinline__ void store_rows(const f32x16 (&acc)[D / 32], const f32x4 (&tail)[2], bf16_t* x, int n, int lane,
                                           float mul, RowPtr row_ptr) {
  constexpr int DB = D / 32, PPR = D / 8;
  const int row = lane & 31;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      bf16x4 w;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = to_bf16(acc[db][4 * g + j] * mul);
      *reinterpret_cast<bf16x4*>(x + Tile<D>::off(row, db * 32 + 8 * g + 4 * (lane >> 5))) = w;
    }
  if constexpr (D % 32 != 0) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = 16 * e + (lane & 15);
      const float m = __shfl(mul, r);
      bf16x4 w;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = to_bf16(tail[e][j] * m);
      if (lane < 32) *reinterpret_cast<bf16x4*>(x + Tile<D>::off(r, 64 + 4 * (lane >> 4))) = w;
    }
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the wave's own rows: no barrier)
#pragma unroll
  for (int p0 = 0; p0 < 32 * PPR; p0 += 64) {
    const int p = p0 + lane, r = p / PPR, slot = p - r * PPR;
    if (r < n) {  // (n <= 32)
      const u32x4 w = *reinterpret_cast<const u32x4*>(x + r * D + slot * 8);
      *reinterpret_cast<u32x4*>(row_ptr(r) + (slot ^ Tile<D>::swz(r)) * 8) = w;
    }
  }
}

// Online softmax and output of 32 rows of a wave (row = lane % 32), as S^T = K Q^T and
// O^T += V^T P^T (layouts at the top of mw_device.h).
template <int D, int BN>
struct RowBlock {
  static constexpr int KK = (D + 15) / 16, DB = D / 32, KB = BN / 32;
  static constexpr bool TAIL = D % 32 != 0;
  // The running maximum moves when a step raises it by more than this many powers of two;
  // until then probabilities are taken against the old one and stay below 2^8.
  static constexpr float kRaise = 8.f;
  f32x16 o[DB];
  f32x4 ot[2];  // (TAIL) columns 64.. of rows 0..15 and 16..31
  float m, l;

  __device__ __forceinline__ void init() {
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = zero16();
    ot[0] = ot[1] = zero4();
    m = -INFINITY;
    l = 0.f;
  }

  // One step of BN staged keys; `key0` + i is the place of key i, and (MASKED) a row sees
  // places lo <= place < hi.  `mid` is called between the scores and the softmax.
  //
  // Matrix phases go first: of two waves on a SIMD one is then in its softmax while the other multiplies (12 heads x
  // 19200 rows x 2048 keys, D = 128: 261 -> 246 us).  Over pages (CODES) the conversion of the next tile, in `mid`, and
  // what lies between two steps come last as well (12 heads x 2400 rows over 15000 cached tokens: D = 128 327 -> 300 us,
  // D = 64 214 -> 177 us; with the conversion in front of the step 316 and 208); with bf16 keys, whose steps are staged
  // by a few instructions, that is 5% slower.
  template <bool MASKED, bool CODES, class Mid>
  __device__ __forceinline__ void step(Mid mid, const bf16_t* Kt, const bf16_t* Vt, const FragOffsets<D>& fo, const Tail72& ft,
                                       const bf16x8 (&qf)[KK], float c, int key0, int lo, int hi, int lane) {
    // fragments read in groups ahead of their products: 1 to 2% faster, but at D = 64 over pages up to 7% slower
    constexpr bool GROUPS = D != 64 || !CODES;
    f32x16 s[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) s[kb] = zero16();
    // K fragments of two contraction steps at a time, read while the two before them multiply (as in add())
    constexpr int STEP = GROUPS ? 2 : KK;
    bf16x8 kf[2][STEP][KB];
    auto read = [&](int g) {
#pragma unroll
      for (int j = 0; j < STEP; ++j)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
          if (STEP * g + j < KK) kf[g & 1][j][kb] = fo.row8(Kt, kb * 32, STEP * g + j);
    };
    if constexpr (CODES) __builtin_amdgcn_s_setprio(1);
    read(0);
#pragma unroll
    for (int g = 0; STEP * g < KK; ++g) {
      if (STEP * (g + 1) < KK) read(g + 1);
      if constexpr (GROUPS) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < STEP; ++j)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
          if (STEP * g + j < KK) s[kb] = mfma32(kf[g & 1][j][kb], qf[STEP * g + j], s[kb]);
      if constexpr (GROUPS) __builtin_amdgcn_sched_barrier(0);
    }
    auto vf = [&](int kb, int t, int db) { return fo.tr8(Vt, kb * 32, t, db); };
    bf16x8 ahead[DB];
    ahead_of(ahead, 0, vf);
    if constexpr (MASKED) hide(s, key0, lo, hi, lane);
    __builtin_amdgcn_s_setprio(0);
    mid();
    weigh(s, c, lane);
    __builtin_amdgcn_s_setprio(1);
    add<GROUPS>(s, ahead, vf, [&](int kb) { return ft.read(Vt, kb * 32); });
    if constexpr (CODES) __builtin_amdgcn_s_setprio(0);
  }

  // Scores of keys that the row does not see: -inf.
  __device__ __forceinline__ static void hide(f32x16 (&s)[KB], int key0, int lo, int hi, int lane) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = key0 + kb * 32 + acc_row(i, lane);
        s[kb][i] = ((key >= lo) & (key < hi)) ? s[kb][i] : -INFINITY;
      }
  }

  // Scores -> probabilities against the running maximum; their sum.
  __device__ __forceinline__ void weigh(f32x16 (&s)[KB], float c, int lane) {
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[kb][i]);
    mx = max_halves(mx) * c;
    const bool raise = mx > m + kRaise;
    if (wave_any(raise)) {
      // rows that keep their maximum (it may be -inf still) keep a factor of 1
      const float a = raise ? fast_exp2(m - mx) : 1.f;
      l *= a;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] *= a;
      if constexpr (TAIL) {
#pragma unroll
        for (int e = 0; e < 2; ++e) ot[e] *= __shfl(a, 16 * e + (lane & 15));
      }
      m = raise ? mx : m;
    }
    const float nm = m == -INFINITY ? 0.f : -m;
    float sum = 0.f;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[kb][i] = fast_exp2(fmaf(s[kb][i], c, nm));
        sum += s[kb][i];
      }
    l += sum;
  }

  // O^T += V^T P^T; the probabilities go to the matrix product in bf16 (their sum stays in 32 bits).  vf(kb, t, db):
  // V fragment of 16-key step t and column block db of key block kb; vt(kb): (TAIL) that of columns 64...
  // `ahead` holds the first step's fragments (ahead_of), read before the softmax.  With GROUPS each step's fragments
  // are read while the one before it multiplies; left alone, the compiler reads a fragment right before its product.
  template <class VF>
  __device__ __forceinline__ static void ahead_of(bf16x8 (&v)[DB], int step, VF vf) {
#pragma unroll
    for (int db = 0; db < DB; ++db) v[db] = vf(step / 2, step % 2, db);
  }
  template <bool GROUPS, class VF, class VT>
  __device__ __forceinline__ void add(const f32x16 (&s)[KB], bf16x8 (&ahead)[DB], VF vf, VT vt) {
    bf16x8 v[2][DB], p[2];
#pragma unroll
    for (int db = 0; db < DB; ++db) v[0][db] = ahead[db];
#pragma unroll
    for (int step = 0; step < 2 * KB; ++step) {
      if (step + 1 < 2 * KB) ahead_of(v[(step + 1) & 1], step + 1, vf);
      p[step & 1] = pack8(s[step / 2], step % 2);
      if constexpr (GROUPS) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] = mfma32(v[step & 1][db], p[step & 1], o[db]);
      if constexpr (GROUPS) __builtin_amdgcn_sched_barrier(0);
      if (TAIL && step % 2) {
        const bf16x8 x = vt(step / 2);
        tail_operands(p[0], p[1]);
#pragma unroll
        for (int e = 0; e < 2; ++e) ot[e] = mfma16(x, p[e], ot[e]);
      }
    }
  }

  // Floats of LDS that merge() takes.
  template <int KG, int NWR>
  static constexpr int merge_floats() {
    return (KG - 1) * NWR * (DB * 16 + 2 + (TAIL ? 8 : 0)) * 64;
  }
  // The key groups' results of the same rows, joined in group 0 (in group order): with M the
  // largest m_g, O = sum 2^(m_g - M) O_g and l likewise.  Every wave of the workgroup calls it
  // after the last read of `x`; afterwards only group 0 holds the result.
  template <int KG, int NWR>
  __device__ __forceinline__ void merge(int kg, int rw, int lane, float* x) {
    constexpr int N = DB * 16 + 2 + (TAIL ? 8 : 0);
    if (kg > 0) {
      float* y = x + ((kg - 1) * NWR + rw) * N * 64 + lane;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) y[(db * 16 + i) * 64] = o[db][i];
      y[DB * 16 * 64] = m;
      y[(DB * 16 + 1) * 64] = l;
      if constexpr (TAIL) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[(DB * 16 + 2 + i) * 64] = ot[i / 4][i % 4];
      }
    }
    __syncthreads();
    if (kg > 0) return;  // (the caller's barrier follows)
    float M = m, w[KG];
#pragma unroll
    for (int g = 1; g < KG; ++g) {
      w[g] = x[((g - 1) * NWR + rw) * N * 64 + DB * 16 * 64 + lane];
      M = fmaxf(M, w[g]);
    }
    w[0] = m;
#pragma unroll
    for (int g = 0; g < KG; ++g) w[g] = w[g] == -INFINITY ? 0.f : fast_exp2(w[g] - M);
    l *= w[0];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] *= w[0];
    if constexpr (TAIL) {
#pragma unroll
      for (int e = 0; e < 2; ++e) ot[e] *= __shfl(w[0], 16 * e + (lane & 15));
    }
#pragma unroll
    for (int g = 1; g < KG; ++g) {
      const float* y = x + ((g - 1) * NWR + rw) * N * 64 + lane;
      l = fmaf(w[g], y[(DB * 16 + 1) * 64], l);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] = fmaf(w[g], y[(db * 16 + i) * 64], o[db][i]);
      if constexpr (TAIL) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float wt = __shfl(w[g], 16 * e + (lane & 15));
#pragma unroll
          for (int i = 0; i < 4; ++i) ot[e][i] = fmaf(wt, y[(DB * 16 + 2 + 4 * e + i) * 64], ot[e][i]);
        }
      }
    }
    m = M;
  }
};

// Results of rows t0.. of key head bh = (b, hk): of one key range of several as an unnormalised fp32 O and the pair
// (m, l), else O and LSE.  x: LDS scratch of 32 rows.
template <int D, int BN>
__device__ __forceinline__ void finish_rows(const RowsParams& p, const RowBlock<D, BN>& rb, int split, int bh, int b, int hk,
                                            int t0, bf16_t* x, int lane) {
  constexpr int DB = D / 32;
  constexpr bool TAIL = D % 32 != 0;
  const int row = t0 + (lane & 31), G = p.G;
  const float l = sum_halves(rb.l);
  if (p.n_splits > 1) {
    const long long prow = ((long long)split * p.B * p.Hkv + bh) * p.R;
    if constexpr (TAIL) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = t0 + 16 * e + (lane & 15);
        if (lane < 32 && r < p.R) *reinterpret_cast<f32x4*>(p.part + (prow + r) * D + 64 + 4 * (lane >> 4)) = rb.ot[e];
      }
    }
    if (row >= p.R) return;
    float* po = p.part + (prow + row) * D;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = rb.o[db][4 * g + j];
        *reinterpret_cast<f32x4*>(po + db * 32 + 8 * g + 4 * (lane >> 5)) = w;
      }
    if (lane < 32) {
      float* ml = p.part + (long long)p.n_splits * p.B * p.Hkv * p.R * D + 2 * (prow + row);
      ml[0] = rb.m;
      ml[1] = l;
    }
    return;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;  // a row that saw no key gives zeros
  store_rows<D>(rb.o, rb.ot, x, min(32, p.R - t0), lane, inv,
                [&](int r) { return p.o + row_offset(p.so, b, hk, G, t0 + r); });
  if (p.lse != nullptr && lane < 32 && row < p.R) {
    const int t = row / G;
    p.lse[((long long)b * p.Hkv * G + hk * G + (row - t * G)) * p.T + t] =
        l == 0.f ? -INFINITY : (rb.m + __log2f(l)) * 0.69314718055994530942f;
  }
}

// Eight codes (two words) -> bf16 values at a power-of-two scale.
__device__ __forceinline__ bf16x8 decode(unsigned w0, unsigned w1, float scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A tile of 64 cached tokens of one head on its way into LDS: this thread's pieces of 16 K and V codes in registers.
// The tile's codes are contiguous in the page; NT threads a round.  D = 72: 288 pieces, the 32 that 256 threads leave
// over of K and of V are the last wave's, K's by its first half; a piece may end in the next row, and so do its two
// slots of the (dense) LDS tile.
template <int D, int NT>
struct CodeTile {
  static constexpr bool ODD = D == 72;
  static constexpr int PPR = D / 16;  // pieces per row (D = 64, 128)
  static constexpr int ROUNDS = ODD ? 1 : 64 * PPR / NT;
  static_assert(ODD ? NT == 256 : 64 * PPR % NT == 0, "whole rounds");
  u32x4 k[ROUNDS], v[ROUNDS], rest;
  float ks, vs;
  int last;

  // The tile at `kp`, `vp` (row 0 of the tile in its page), of which rows 0..last hold tokens.  What is behind them
  // is replaced: the last row again, or (D = 72) zeros.
  __device__ __forceinline__ void fetch(const uint8_t* kp, const uint8_t* vp, const float* k_scale,
                                        const float* v_scale, int last_row, int tid) {
    ks = *k_scale;
    vs = *v_scale;
    last = last_row;
    if constexpr (ODD) {
      k[0] = reinterpret_cast<const u32x4*>(kp)[tid];
      v[0] = reinterpret_cast<const u32x4*>(vp)[tid];
      if (tid >= 192) rest = reinterpret_cast<const u32x4*>((tid & 32) ? vp : kp)[256 + (tid & 31)];
    } else {
#pragma unroll
      for (int it = 0; it < ROUNDS; ++it) {
        const int p = it * NT + tid, row = p / PPR, at = min(row, last) * PPR + (p - row * PPR);
        k[it] = reinterpret_cast<const u32x4*>(kp)[at];
        v[it] = reinterpret_cast<const u32x4*>(vp)[at];
      }
    }
  }

  // (D = 72) piece p of a tile into its two LDS slots
  __device__ __forceinline__ void put(bf16_t* tile, int p, const u32x4& x, float scale) const {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const bool in = (2 * p + j) / 9 <= last;
      *reinterpret_cast<bf16x8*>(tile + (2 * p + j) * 8) = decode(in ? x[2 * j] : 0u, in ? x[2 * j + 1] : 0u, scale);
    }
  }

  // The tile in bf16 into LDS rows row0.. of the K and V tiles.
  __device__ __forceinline__ void commit(bf16_t* Kt, bf16_t* Vt, int row0, int tid) const {
    if constexpr (ODD) {
      put(Kt + row0 * D, tid, k[0], ks);
      put(Vt + row0 * D, tid, v[0], vs);
      if (tid >= 192) put(((tid & 32) ? Vt : Kt) + row0 * D, 256 + (tid & 31), rest, (tid & 32) ? vs : ks);
    } else {
#pragma unroll
      for (int it = 0; it < ROUNDS; ++it) {
        const int p = it * NT + tid, row = p / PPR, col = (p - row * PPR) * 16;
        // a piece fills two neighbouring 16-byte slots: odd rows write the upper one first, so that two rows'
        // writes together cover every bank
        const bool up = row & 1;
        const unsigned k0 = k[it][0], k1 = k[it][1], k2 = k[it][2], k3 = k[it][3];
        const unsigned v0 = v[it][0], v1 = v[it][1], v2 = v[it][2], v3 = v[it][3];
        const int first = Tile<D>::off(row0 + row, up ? col + 8 : col), second = Tile<D>::off(row0 + row, up ? col : col + 8);
        *reinterpret_cast<bf16x8*>(Kt + first) = decode(up ? k2 : k0, up ? k3 : k1, ks);
        *reinterpret_cast<bf16x8*>(Vt + first) = decode(up ? v2 : v0, up ? v3 : v1, vs);
        *reinterpret_cast<bf16x8*>(Kt + second) = decode(up ? k0 : k2, up ? k1 : k3, ks);
        *reinterpret_cast<bf16x8*>(Vt + second) = decode(up ? v0 : v2, up ? v1 : v3, vs);
      }
    }
  }
};

// NW waves in KG key groups of NW / KG waves of 32 rows each; a step stages KG * BN keys,
// of which a group takes its BN.  WPS: waves per SIMD the registers are allocated for.
// Bound by a SIMD's two or three waves: over long keys the matrix units are busy 40 to 53% of the time, and waves at work
// on a vector or matrix instruction (softmax; over pages the conversion too) 45 to 51% of a SIMD; the two overlap only
// between waves.  12 heads x 19200 rows x 2048 keys, D = 128: 240 to 245 us, 987 to 1007 TF (a plain product of 8192^3:
// 1246); 16 heads x 4800 rows, one chunk that sees 15000 cached tokens and itself, 852 to 879 us, 886 to 914 TF.
template <int D, bool PAGED, int NW, int BN, int KG, int WPS>
__global__ __launch_bounds__(64 * NW, WPS) void attn_rows_kernel(RowsParams p, RowsSeqs<PAGED> seqs) {
  constexpr int NWR = NW / KG, BM = 32 * NWR, NT = 64 * NW, BK = BN * KG, NB = BK / 64;
  static_assert(NW % KG == 0 && BK % 64 == 0, "whole 64-token blocks a step");
  using RB = RowBlock<D, BN>;
  using Codes = CodeTile<D, NT>;
  constexpr int KK = RB::KK, DB = RB::DB;
  constexpr bool TAIL = RB::TAIL;
  constexpr int TE = stage_elems<D, BK, NT>();
  __shared__ __attribute__((aligned(16))) bf16_t lds[2][2][TE];  // K, V x two stages
  static_assert(RB::template merge_floats<KG, NWR>() * 4 <= (int)sizeof(lds), "the merge fits the stages");
  bf16_t(*Ks)[TE] = lds[0];
  bf16_t(*Vs)[TE] = lds[1];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % NWR, kg = wave / NWR;
  // Consecutive workgroups are dealt to the 8 XCDs in turn: each gets one contiguous range of (key head, key range,
  // batch member, row tile).  The row tiles of a range share one L2; members, whose lengths differ, take turns, or the
  // XCDs with the long ones would finish last (members one after another: 8 chunks of 600 rows, 2 x 12 heads over 14700
  // and 11025 cached tokens 1120 us, so 1037; 3 x 16 heads x 999 rows over 3601, 3001 and 2401, D = 72, 125 and 111).
  int item;
  {
    const int n = gridDim.x, x = blockIdx.x % 8, q = n / 8, rem = n % 8;
    item = x * q + min(x, rem) + blockIdx.x / 8;
  }
  const int group = item / p.n_rtiles, rt = p.n_rtiles - 1 - (item - group * p.n_rtiles);  // late rows see more
  const int range = group / p.B, b = group - range * p.B;
  const int hk = range / p.n_splits, split = range - hk * p.n_splits, bh = b * p.Hkv + hk;
  const int G = p.G;
  const int r0 = rt * BM;

  // this lane's row and its Q fragments; rows behind the last and columns past D are zeros
  const int row = r0 + rw * 32 + (lane & 31);
  bf16x8 qf[KK];
  {
    const bf16_t* qp = p.q + row_offset(p.sq, b, hk, G, min(row, p.R - 1)) + 8 * (lane >> 5);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      if (row < p.R && (D % 16 == 0 || 16 * kk + 8 * (lane >> 5) < D)) {
        qf[kk] = *reinterpret_cast<const bf16x8*>(qp + 16 * kk);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) qf[kk][j] = (__bf16)0.f;
      }
    }
  }

  // the bf16 keys: n_new of them; a row sees [lo, hi)
  int n_new = p.M, len = 0;
  if (p.kv_len != nullptr) n_new = max(0, min(p.M, p.kv_len[b]));
  int lo = 0, hi = n_new, first = 0, last = n_new, lo_all = 0, hi_all = n_new;  // of the row, of any row, of every row
  if (PAGED && p.mode != ROWS_SEE_ALL) {
    const int r1 = min(r0 + BM, p.R) - 1;
    const int c0 = r0 / G / p.qlen, c1 = r1 / G / p.qlen, c = min(row, p.R - 1) / G / p.qlen;
    const bool own = p.mode == ROWS_SEE_OWN;
    hi = (c + 1) * p.qlen;
    lo = own ? c * p.qlen : 0;
    last = (c1 + 1) * p.qlen;
    first = own ? c0 * p.qlen : 0;
    hi_all = (c0 + 1) * p.qlen;
    lo_all = own ? c1 * p.qlen : 0;
  }
  int seq = 0;
  if constexpr (PAGED) {
    seq = seqs.seq[b];
    if constexpr (TAIL) {
      // D = 72: the last row's reads run into the slack behind the tile and meet zeros in Q; it
      // has to be finite, and only the bf16 staging fills it
      constexpr int SLACK = TE - BK * D;
      for (int i = tid; i < 4 * SLACK; i += NT) (&lds[0][0][0])[(i / SLACK) * TE + BK * D + i % SLACK] = 0;
    }
    len = max(0, min(p.lens[seq], p.W * p.L));
  }
  // The key steps, those that every row sees whole first, so that the mask is evaluated in a
  // loop of its own: cached steps [0, old_full), bf16 steps [full0, full1), then the partly
  // filled cached step (old_part of them) and the bf16 steps [new0, full0) and [full1, new1).
  const int old_full = len / BK, old_part = len > old_full * BK;
  const int new0 = first / BK, new1 = last > first ? (last + BK - 1) / BK : new0;
  const int full0 = min(max((lo_all + BK - 1) / BK, new0), new1), full1 = min(max(hi_all / BK, full0), new1);
  const int n_full = old_full + full1 - full0, n_all = n_full + old_part + (full0 - new0) + (new1 - full1);
  const int beg = (int)((long long)n_all * split / p.n_splits), end = (int)((long long)n_all * (split + 1) / p.n_splits);
  // Step i: cached step x as x, bf16 step x as ~x.
  auto place = [&](int i) {
    if (i < n_full) return i < old_full ? i : ~(full0 + i - old_full);
    const int j = i - n_full - old_part;
    if (j < 0) return old_full;
    return ~(j < full0 - new0 ? new0 + j : full1 + j - (full0 - new0));
  };

  const long long kbase = b * p.sk.b + hk * p.sk.h, vbase = b * p.sv.b + hk * p.sv.h;
  const RowOffsets<D, BK, NT> ro_k(p.sk.t, tid), ro_v(p.sv.t, tid);
  // bf16 keys from k0 on straight into LDS
  auto stage_new = [&](int k0, int buf) {
    if (k0 + BK <= n_new) {
      stage_rows_s<D, BK, NT>(Ks[buf], p.k + kbase + k0 * p.sk.t, ro_k, tid);
      stage_rows_s<D, BK, NT>(Vs[buf], p.v + vbase + k0 * p.sv.t, ro_v, tid);
    } else {
      stage_kv_rows_direct<D, BK, NT>(Ks[buf], Vs[buf], [&](int r) -> RowPair {
        const long long j = min(k0 + r, n_new - 1);
        return {p.k + kbase + j * p.sk.t, p.v + vbase + j * p.sv.t};
      }, tid);
    }
  };
  // Cached tokens of a step into registers (and from there into LDS).  Their pages are looked up one
  // step before that.
  Codes codes[PAGED ? NB : 1];
  int page_of[PAGED ? NB : 1];
  auto block_at = [&](int x, int nb) { return min(x * NB + nb, (len - 1) >> 6); };  // one behind the last repeats it
  auto look = [&](int x) {
    if constexpr (PAGED) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const unsigned w = __umulhi((unsigned)block_at(x, nb), p.per_page_magic);
        page_of[nb] = p.table[(long long)seq * p.W + (int)(p.per_page == 1 ? block_at(x, nb) : w)];
      }
    }
  };
  auto fetch = [&](int x) {
    if constexpr (PAGED) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int blk = block_at(x, nb);
        const int off = p.per_page == 1 ? 0 : blk - (int)__umulhi((unsigned)blk, p.per_page_magic) * p.per_page;
        const long long head = (long long)page_of[nb] * p.Hkv + hk;
        const long long e = head * p.per_page + off, at = e * (64 * D);
        codes[nb].fetch(p.k_pages + at, p.v_pages + at, p.k_scales + e, p.v_scales + e, len - 1 - 64 * blk, tid);
      }
    }
  };
  auto commit = [&](int buf) {
    if constexpr (PAGED) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) codes[nb].commit(Ks[buf], Vs[buf], nb * 64, tid);
    }
  };

  const FragOffsets<D> fo(lane, kg * BN * D);
  const Tail72 ft(lane, kg * BN * D);
  const float c = p.scale_log2;
  RB rb;
  rb.init();
  int buf = 0;
  if (beg < end) {
    // Two LDS stages.  A cached step is in registers one step before it is written to LDS, and in LDS one step
    // before it is used; a bf16 step goes to LDS during the step before it.
    int x = place(beg), next = beg + 1 < end ? place(beg + 1) : -1;  // this step and the one behind it
    int after = PAGED && beg + 2 < end ? place(beg + 2) : -1;
    if (PAGED && x >= 0) {
      look(x);
      fetch(x);
      commit(0);
    } else {
      stage_new(~x * BK, 0);
      wait_vmem();
    }
    if (PAGED && next >= 0) {
      look(next);
      fetch(next);
    }
    if (PAGED && after >= 0) look(after);
    lds_barrier();
    int i = beg;
    auto run = [&](auto masked, int stop) {
      for (; i < stop; ++i) {
        const int later = PAGED && i + 3 < end ? place(i + 3) : -1;
        const bool more = i + 1 < end;
        if (!PAGED && more) next = place(i + 1);
        const bool direct = more && (!PAGED || next < 0);
        if (direct) stage_new(~next * BK, buf ^ 1);
        auto mid = [&] {
          if constexpr (PAGED) {
            if (more && !direct) commit(buf ^ 1);
            if (after >= 0) fetch(after);
            if (later >= 0) look(later);
          }
        };
        const bool old = PAGED && x >= 0;
        const int k0 = (old ? x : ~x) * BK + kg * BN;
        rb.template step<decltype(masked)::value, PAGED>(mid, Ks[buf], Vs[buf], fo, ft, qf, c, k0, old ? 0 : lo,
                                                         old ? len : hi, lane);
        if (direct) wait_vmem();
        lds_barrier();
        buf ^= 1;
        x = next;
        next = after;
        after = later;
      }
    };
    run(std::false_type{}, min(n_full, end));
    run(std::true_type{}, end);
  }
  if constexpr (KG > 1) {
    rb.template merge<KG, NWR>(kg, rw, lane, reinterpret_cast<float*>(&lds[0][0][0]));
    __syncthreads();     // (the stages are written again below)
    if (kg > 0) return;  // no barrier follows
  }

  // scratch: a half stage holds the rows of BK / 32 waves (every wave has passed the last barrier)
  constexpr int PER = BK / 32;
  const int half = rw / PER;
  finish_rows<D, BN>(p, rb, split, bh, b, hk, r0 + rw * 32, (half & 1 ? Vs : Ks)[half >> 1] + (rw - half * PER) * 32 * D, lane);
}

// Sequences of a call of few rows, and their key ranges: those of batch member b are numbers first[b] .. first[b + 1].
struct PageRanges {
  int seq[kMaxSeqs];
  int first[kMaxSeqs + 1];
};

// Few rows over pages (RB blocks of 32 rows): bound by reading the codes, so nothing is shared and nothing waits but
// for them.  Each of NW waves streams units of 32 tokens of its own, every NW-th of the workgroup's key range, through
// NSTG private LDS stages: codes go there as they are (32 rows of a head are contiguous in a page), NSTG - 1 units
// ahead, and are converted as the fragments are read; no barrier separates the steps.  K: 16 codes of a row a lane,
// eight for each of two contraction steps (Q's fragments follow that order).  V: ds_read_b64_tr_b8 gives a lane the
// codes of eight keys of its column (in each group of 16 lanes, byte j of lane i is byte i % 8 of the 8 bytes
// addressed by lane 2 j + i / 8).  The waves' results are joined at the end.
// One token of 8 sequences over up to 15840 tokens, 4 key heads (D = 128), 100 MB of codes: 21 us, 4.8 TB/s (a copy of
// 1 GiB: 5.0); 64 rows of 16 heads over 15840, 65 MB, 26 us: by then the conversion and the softmax bound it.
template <int D>
struct RawTile {  // 32 rows of D codes, 16-byte slots permuted so that row and transposing reads spread over the banks
  static constexpr int SLOTS = D / 16;
  static constexpr int ROUNDS = (32 * D + 1023) / 1024;  // 1 KB loads of a tile
  static constexpr int BYTES = ROUNDS * 1024;
  __device__ __forceinline__ static int swz(int row) {
    if constexpr (D == 128) return (row & 7) ^ ((row >> 1) & 4);
    if constexpr (D == 64) return (row >> 2) & 3;
    return 0;  // D = 72: rows are dense, 18 banks apart
  }
  __device__ __forceinline__ static int off(int row, int col) {  // col: a multiple of 8
    if constexpr (D == 72) return row * D + col;
    return row * D + (((col >> 4) ^ swz(row)) << 4) + (col & 15);
  }
  // byte of the (unswizzled) tile that lane `lane` of load `it` fetches; rows behind `last` repeat it
  __device__ __forceinline__ static unsigned source(int it, int lane, int last) {
    if constexpr (D == 72) {
      // (144 pieces of 16 bytes do not end with a row: two halves of 8 could; `last` is met by the reader instead)
      (void)last;
      return (unsigned)min(it * 64 + lane, 32 * D / 16 - 1) * 16u;
    } else {
      const int p = it * 64 + lane, row = p / SLOTS, slot = p - row * SLOTS;
      return (unsigned)(min(row, last) * D + ((slot ^ swz(row)) << 4));
    }
  }
};

constexpr int kMetaBlocks = 256;  // blocks of 64 tokens whose page and scales are looked up at a time

template <int D, int RB, int NW, int NSTG>
__global__ __launch_bounds__(64 * NW, RB == 1 ? 2 : 1) void attn_pages_kernel(RowsParams p, PageRanges seqs, int chunk) {
  using RT = RawTile<D>;
  using Rows = RowBlock<D, 32>;
  constexpr int KK = Rows::KK, DB = Rows::DB, LOADS = 2 * RT::ROUNDS;
  constexpr bool TAIL = Rows::TAIL;
  static_assert(NSTG >= 2 && NSTG <= 4 && LOADS * (NSTG - 1) <= 63, "the wait counts the units in flight");
  constexpr int STAGE = 2 * RT::BYTES;
  constexpr int MERGE = RB * NW * (DB * 16 + 2 + (TAIL ? 8 : 0)) * 64 * 4;
  constexpr int STREAM = NW * NSTG * STAGE;
  __shared__ __attribute__((aligned(16))) unsigned char lds[STREAM > MERGE ? STREAM : MERGE];
  __shared__ int meta_block[kMetaBlocks];
  static_assert(64 * NW == kMetaBlocks, "a thread looks up one block");
  __shared__ float meta_k[kMetaBlocks], meta_v[kMetaBlocks];

  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Workgroup = (range number, key head).  No two read the same codes, so they go round the XCDs as they come.
  const int range = blockIdx.x / p.Hkv, hk = blockIdx.x - range * p.Hkv;
  int b = -1;  // the last member whose first range is not behind this one
  for (int i = 0; i < p.B; i += 64) {
    const int first = seqs.first[min(i + lane, p.B)];
    b += __builtin_popcountll(__builtin_amdgcn_ballot_w64(i + lane < p.B && first <= range));
  }
  b = __builtin_amdgcn_readfirstlane(b);
  const int split = range - seqs.first[b], n_ranges = seqs.first[b + 1] - seqs.first[b];
  const int bh = b * p.Hkv + hk, G = p.G;
  const int seq = seqs.seq[b];
  // The pages of the range's first blocks are looked up before the length is known (an entry of the row is
  // always readable; what lies behind the length is not used): one memory latency less before the codes stream.
  auto entry = [&](int blk) {
    const int w = p.per_page == 1 ? blk : (int)__umulhi((unsigned)blk, p.per_page_magic);
    return make_int2(p.table[(long long)seq * p.W + min(w, p.W - 1)], blk - w * p.per_page);
  };
  int2 my_entry = entry(split * chunk + tid);
  const int len = max(0, min(p.lens[seq], p.W * p.L));
  // this workgroup's blocks: `chunk` of them, the last range whatever is left
  const int n_blk = (len + 63) >> 6;
  const int blk0 = min(n_blk, split * chunk), blk1 = split + 1 == n_ranges ? n_blk : min(n_blk, blk0 + chunk);

  bf16x8 qf[RB][KK];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = rb * 32 + (lane & 31);
    const bf16_t* qp = p.q + row_offset(p.sq, b, hk, G, min(row, p.R - 1));
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      // steps 2 j and 2 j + 1: columns 32 j + 16 h + 0..7 and + 8..15; (D = 72) step 4: columns 64..71 and zeros
      const int col = TAIL && kk == KK - 1 ? 64 : 32 * (kk / 2) + 16 * h + 8 * (kk & 1);
      if (row < p.R && !(TAIL && kk == KK - 1 && h)) {
        qf[rb][kk] = *reinterpret_cast<const bf16x8*>(qp + col);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) qf[rb][kk][j] = (__bf16)0.f;
      }
    }
  }
  Rows rows[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) rows[rb].init();

  unsigned char* mine = lds + wave * NSTG * STAGE;
  const float c = p.scale_log2;
  // this lane's part of the transposing reads: row and column within 32 keys x 32 columns
  const int tr_row = 4 * h + (((lane & 15) >> 1) & 3) + 8 * ((lane & 15) >> 3), tr_col = 16 * ((lane >> 4) & 1) + 8 * (lane & 1);

  for (int m0 = blk0; m0 < blk1; m0 += kMetaBlocks) {
    const int m1 = min(blk1, m0 + kMetaBlocks);
    if (m0 > blk0) {
      __syncthreads();
      my_entry = entry(m0 + tid);
    }
    // (the page's block of this head: below 2^31, P H L / 64 is checked)
    const int my_block = (int)(((long long)my_entry.x * p.Hkv + hk) * p.per_page + my_entry.y);
    const bool known = tid < m1 - m0;
    if (known) meta_block[tid] = my_block;
    __syncthreads();
    // Q is waited for here, not by the compiler's count inside the loop, which does not know of the loads into LDS
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) asm volatile("" : "+v"(qf[rb][kk]));
    // units of 32 tokens of these blocks: every NW-th is this wave's
    const int units = (min(len, m1 * 64) - m0 * 64 + 31) >> 5;
    auto issue = [&](int u, int st) {
      const long long at = ((long long)__builtin_amdgcn_readfirstlane(meta_block[u >> 1]) * 64 + 32 * (u & 1)) * D;
      const int last = min(31, len - 1 - m0 * 64 - u * 32);
      const unsigned to = lds_addr(mine) + st * STAGE;
#pragma unroll
      for (int it = 0; it < RT::ROUNDS; ++it) {
        const unsigned src = RT::source(it, lane, last);
        dma_lds_16_s(p.k_pages + at, src, __builtin_amdgcn_readfirstlane(to + it * 1024));
        dma_lds_16_s(p.v_pages + at, src, __builtin_amdgcn_readfirstlane(to + RT::BYTES + it * 1024));
      }
    };
    // the blocks' scales, a thread each, ahead of the codes
    dma_lds_4(p.k_scales + (known ? my_block : 0), lds_addr(meta_k) + wave * 256);
    dma_lds_4(p.v_scales + (known ? my_block : 0), lds_addr(meta_v) + wave * 256);
    int ahead = 0, u_in = wave, st_in = 0, st = 0;
#pragma unroll
    for (int i = 0; i < NSTG - 1; ++i)
      if (u_in < units) {
        issue(u_in, st_in);
        u_in += NW;
        ++st_in;
        ++ahead;
      }
    if (st_in == NSTG) st_in = 0;
    wait_vmem_upto<LOADS, NSTG - 1>(ahead);  // the scales; the first codes are on their way
    lds_barrier();
    for (int u = wave; u < units; u += NW) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the stage to be filled has been read
      if (u_in < units) {
        issue(u_in, st_in);
        u_in += NW;
        st_in = st_in + 1 == NSTG ? 0 : st_in + 1;
        ++ahead;
      }
      --ahead;
      wait_vmem_upto<LOADS, NSTG - 1>(ahead);
      asm volatile("" ::: "memory");
      const unsigned char* Kt = mine + st * STAGE;
      const unsigned char* Vt = Kt + RT::BYTES;
      const float ks = meta_k[u >> 1], vs = meta_v[u >> 1];
      const int last = len - 1 - m0 * 64 - u * 32;  // last token of the unit, if below 31
      // (D = 72: rows behind it hold whatever the page does)
      const int krow = TAIL ? min(lane & 31, last) : lane & 31;
      f32x16 s[RB][1];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) s[rb][0] = zero16();
#pragma unroll
      for (int j = 0; j < KK / 2; ++j) {
        unsigned w[4];
        if constexpr (TAIL) {
          const u32x2 x = *reinterpret_cast<const u32x2*>(Kt + krow * D + 32 * j + 16 * h);
          const u32x2 y = *reinterpret_cast<const u32x2*>(Kt + krow * D + 32 * j + 16 * h + 8);
          w[0] = x[0], w[1] = x[1], w[2] = y[0], w[3] = y[1];
        } else {
          const u32x4 x = *reinterpret_cast<const u32x4*>(Kt + RT::off(krow, 32 * j + 16 * h));
          w[0] = x[0], w[1] = x[1], w[2] = x[2], w[3] = x[3];
        }
        const bf16x8 k0 = decode(w[0], w[1], ks), k1 = decode(w[2], w[3], ks);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          s[rb][0] = mfma32(k0, qf[rb][2 * j], s[rb][0]);
          s[rb][0] = mfma32(k1, qf[rb][2 * j + 1], s[rb][0]);
        }
      }
      if constexpr (TAIL) {
        const u32x2 x = *reinterpret_cast<const u32x2*>(Kt + krow * D + 64);
        const bf16x8 k0 = decode(h ? 0u : x[0], h ? 0u : x[1], ks);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) s[rb][0] = mfma32(k0, qf[rb][KK - 1], s[rb][0]);
      }
      const bool ragged = last < 31;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        if (ragged) Rows::hide(s[rb], 0, 0, last + 1, lane);
        rows[rb].weigh(s[rb], c, lane);
      }
      // each V fragment is read and converted once for all row blocks
      bf16x8 pb[RB][2];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int t = 0; t < 2; ++t) pb[rb][t] = pack8(s[rb][0], t);
      auto read_v = [&](int row, int col) {
        const unsigned char* at = Vt + (TAIL ? min(row, last) * D + col : RT::off(row, col));
        const auto x = __builtin_amdgcn_ds_read_tr8_b64_v2i32((MW_LDS i32x2*)(at));
        return decode((unsigned)x[0], (unsigned)x[1], vs);
      };
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const bf16x8 vf = read_v(16 * t + tr_row, 32 * db + tr_col);
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) rows[rb].o[db] = mfma32(vf, pb[rb][t], rows[rb].o[db]);
        }
      if constexpr (TAIL) {
        // lane group g holds rows row(g % 2, 8 (g / 2) + j) of columns 64..71 (Tail72); its other eight are not kept
        const int g = lane >> 4, i = lane & 15;
        const bf16x8 vf = read_v(16 * (g & 1) + 4 * (g >> 1) + ((i >> 1) & 3) + 8 * (i >> 3), 64);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          tail_operands(pb[rb][0], pb[rb][1]);
#pragma unroll
          for (int e = 0; e < 2; ++e) rows[rb].ot[e] = mfma16(vf, pb[rb][e], rows[rb].ot[e]);
        }
      }
      st = st + 1 == NSTG ? 0 : st + 1;
    }
  }

  // the queued tokens' own keys, 32 at a time, by the waves of the first range in turn
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  if (split == 0) {
    bf16_t* Vt = reinterpret_cast<bf16_t*>(mine);
    const FragOffsets<D> fo(lane, 0);
    const Tail72 ft(lane, 0);
    const long long kbase = b * p.sk.b + hk * p.sk.h, vbase = b * p.sv.b + hk * p.sv.h;
    for (int k0 = wave * 32; k0 < p.M; k0 += 32 * NW) {
      const bf16_t* kp = p.k + kbase + (long long)min(k0 + (lane & 31), p.M - 1) * p.sk.t;
      f32x16 s[RB][1];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) s[rb][0] = zero16();
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        const int col = TAIL && kk == KK - 1 ? 64 : 32 * (kk / 2) + 16 * h + 8 * (kk & 1);
        const bf16x8 kf = *reinterpret_cast<const bf16x8*>(kp + col);  // (D = 72: Q is zero where h = 1 repeats column 64)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) s[rb][0] = mfma32(kf, qf[rb][kk], s[rb][0]);
      }
#pragma unroll
      for (int it = 0; it < (32 * D / 8 + 63) / 64; ++it) {
        const int q = it * 64 + lane, r = q / (D / 8), slot = q - r * (D / 8);
        if (r < 32)
          *reinterpret_cast<u32x4*>(Vt + Tile<D>::off(r, slot * 8)) =
              *reinterpret_cast<const u32x4*>(p.v + vbase + (long long)min(k0 + r, p.M - 1) * p.sv.t + slot * 8);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const int c0 = min(rb * 32 + (lane & 31), p.R - 1) / G / p.qlen;
        const int hi = p.mode == ROWS_SEE_ALL ? p.M : min(p.M, (c0 + 1) * p.qlen), lo = p.mode == ROWS_SEE_OWN ? c0 * p.qlen : 0;
        Rows::hide(s[rb], k0, lo, hi, lane);
        rows[rb].weigh(s[rb], c, lane);
        auto vf = [&](int, int t, int db) { return fo.tr8(Vt, 0, t, db); };
        bf16x8 ahead[DB];
        Rows::ahead_of(ahead, 0, vf);
        rows[rb].template add<false>(s[rb], ahead, vf, [&](int) { return ft.read(Vt, 0); });
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
  }

  // Join of the waves' results: column block db of every row block (and the tail) is one wave's to add up, with the
  // weights 2^(m_w - M), and to store.
  __syncthreads();
  float* x = reinterpret_cast<float*>(lds) + lane;
  constexpr int N = DB * 16 + 2 + (TAIL ? 8 : 0);
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    float* y = x + (rb * NW + wave) * N * 64;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) y[(db * 16 + i) * 64] = rows[rb].o[db][i];
    y[DB * 16 * 64] = rows[rb].m;
    y[(DB * 16 + 1) * 64] = rows[rb].l;
    if constexpr (TAIL) {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[(DB * 16 + 2 + i) * 64] = rows[rb].ot[i / 4][i % 4];
    }
  }
  __syncthreads();
  static_assert(DB + TAIL <= NW, "a column block a wave");
  if (wave >= DB + TAIL) return;  // no barrier follows
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const float* y = x + rb * NW * N * 64;
    float w[NW], M = -INFINITY, l = 0.f;
#pragma unroll
    for (int g = 0; g < NW; ++g) {
      w[g] = y[(g * N + DB * 16) * 64];
      M = fmaxf(M, w[g]);
    }
#pragma unroll
    for (int g = 0; g < NW; ++g) {
      w[g] = w[g] == -INFINITY ? 0.f : fast_exp2(w[g] - M);
      l = fmaf(w[g], y[(g * N + DB * 16 + 1) * 64], l);
    }
    l = sum_halves(l);
    const int row = rb * 32 + (lane & 31);
    const bool one = p.n_splits == 1;
    const float inv = one ? (l == 0.f ? 0.f : 1.f / l) : 1.f;  // a row that saw no key gives zeros
    const long long prow = ((long long)split * p.B * p.Hkv + bh) * p.R;
    auto put = [&](int r, int col, const f32x4& v) {  // four columns of row r
      if (one) {
        bf16x4 u;
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = to_bf16(v[j]);
        *reinterpret_cast<bf16x4*>(p.o + row_offset(p.so, b, hk, G, r) + col) = u;
      } else {
        *reinterpret_cast<f32x4*>(p.part + (prow + r) * D + col) = v;
      }
    };
    if (!TAIL || wave < DB) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f32x4 v = zero4();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
          for (int g = 0; g < NW; ++g) v[j] = fmaf(w[g], y[(g * N + wave * 16 + 4 * q + j) * 64], v[j]);
          v[j] *= inv;
        }
        if (row < p.R) put(row, wave * 32 + 8 * q + 4 * h, v);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 16 * e + (lane & 15);
        f32x4 v = zero4();
#pragma unroll
        for (int g = 0; g < NW; ++g) {
          const float wg = __shfl(w[g], r);
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = fmaf(wg, y[(g * N + DB * 16 + 2 + 4 * e + j) * 64], v[j]);
        }
        const float iv = __shfl(inv, r);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] *= iv;
        if (lane < 32 && rb * 32 + r < p.R) put(rb * 32 + r, 64 + 4 * (lane >> 4), v);
      }
    }
    if (wave == 0 && lane < 32 && row < p.R) {
      if (!one) {
        float* ml = p.part + (long long)p.n_splits * p.B * p.Hkv * p.R * D + 2 * (prow + row);
        ml[0] = M;
        ml[1] = l;
      } else if (p.lse != nullptr) {
        const int t = row / G;
        p.lse[((long long)b * p.Hkv * G + hk * G + (row - t * G)) * p.T + t] =
            l == 0.f ? -INFINITY : (M + __log2f(l)) * 0.69314718055994530942f;
      }
    }
  }
}

// Join of the key ranges' partials: with M the largest m_s, O = sum 2^(m_s - M) O_s / sum 2^(m_s - M) l_s
// and LSE = (M + log2 of that sum) ln 2.  One thread for four columns of a row.
// A call of few rows over pages (PAGES) has ranges of its own for each batch member.
template <int D, bool PAGES>
__global__ __launch_bounds__(256) void attn_rows_join_kernel(RowsParams p, std::conditional_t<PAGES, PageRanges, int> seqs) {
  constexpr int TPR = D / 4;
  const long long rows = (long long)p.B * p.Hkv * p.R;
  const long long gid = (long long)blockIdx.x * 256 + threadIdx.x;
  const long long pr = gid / TPR;
  if (pr >= rows) return;
  const int col = (int)(gid - pr * TPR) * 4;
  const int bh = (int)(pr / p.R), r = (int)(pr - (long long)bh * p.R);
  const int b = bh / p.Hkv, hk = bh - b * p.Hkv;
  const float* ml = p.part + (long long)p.n_splits * rows * D;
  int n = p.n_splits;
  if constexpr (PAGES) n = seqs.first[b + 1] - seqs.first[b];
  float M = -INFINITY, L = 0.f;
  f32x4 acc = zero4();
  constexpr int U = 8;  // ranges in flight
  for (int s0 = 0; s0 < n; s0 += U) {
    float mv[U], lv[U];
    f32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool in = s0 + u < n;
      const long long x = (long long)(in ? s0 + u : s0) * rows + pr;
      mv[u] = in ? ml[2 * x] : -INFINITY;
      lv[u] = ml[2 * x + 1];
      v[u] = *reinterpret_cast<const f32x4*>(p.part + x * D + col);
    }
    float Mn = M;
#pragma unroll
    for (int u = 0; u < U; ++u) Mn = fmaxf(Mn, mv[u]);
    const float a = M == -INFINITY ? 0.f : fast_exp2(M - Mn);
    L *= a;
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] *= a;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float w = mv[u] == -INFINITY ? 0.f : fast_exp2(mv[u] - Mn);  // an empty range
      L = fmaf(w, lv[u], L);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = fmaf(w, v[u][j], acc[j]);
    }
    M = Mn;
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  bf16x4 w;
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = to_bf16(acc[j] * inv);
  *reinterpret_cast<bf16x4*>(p.o + row_offset(p.so, b, hk, p.G, r) + col) = w;
  if (p.lse != nullptr && col == 0) {
    const int t = r / p.G;
    p.lse[((long long)b * p.Hkv * p.G + hk * p.G + (r - t * p.G)) * p.T + t] =
        L == 0.f ? -INFINITY : (M + __log2f(L)) * 0.69314718055994530942f;
  }
}

}  // namespace mw
