// Backward of the cross attention (gfx950): with P recomputed from Q, K and the forward's LSE,
//   dV = sum_r P_r^T dO_r,  dP = dO V^T,  Delta = rowsum(dO O),  dS = P (dP - Delta),
//   dQ = scale dS K,  dK = scale sum_r dS_r^T Q_r
// over the rows r of a key head (its query heads' tokens, attn_rows.h), so that the gradients of
// shared heads are sums over more rows and need nothing else.
//
//   dQ kernel    : a wave owns 32 rows and walks the keys; it has the rows' dO in registers, so it also
//                  forms Delta (and LSE log2 e) for the other kernel; where one step holds all keys, as sum_j P_j dP_j.  Few rows over many keys: the keys are cut
//                  into ranges that leave fp32 dQ.
//   dK/dV kernel : a wave owns 32 keys and walks rows staged in LDS.  The rows are many and the keys few, so the
//                  rows of a key tile are cut into slices that fill the card and leave fp32 dK, dV.
//   join kernel  : adds ranges and slices in their order.  No atomics: the result is deterministic.
#include <algorithm>
#include <type_traits>

#include "attn_rows.h"

namespace mw {

namespace {

constexpr int kD = MW_CROSS_HEAD_DIM;

// Valid keys of batch member b.
__device__ __forceinline__ int valid_keys(const CrossBwdParams& p, int b) {
  return p.kv_len == nullptr ? p.M : max(0, min(p.M, p.kv_len[b]));
}

// Consecutive workgroups are dealt to the 8 XCDs in turn: each gets one contiguous range of the work, whose order is
// (key head, slice or range, batch member, tile): members of different lengths take turns on every XCD (3 x 64 heads on
// 8, 391 rows, up to 3087 ragged states, D = 64, forward and backward: 359 -> 284 us; equal lengths: within 1%).
__device__ __forceinline__ int xcd_range(int id, int n) {
  const int x = id % 8, q = n / 8, rem = n % 8;
  return x * q + min(x, rem) + id / 8;
}

// dK/dV: NWK key waves of 32 keys each (K fragments, dK^T and dV^T in registers) in QG row groups; a step stages
// BM * QG rows, of which a group takes its BM, and the groups' gradients are added through LDS at the end.  The
// first VL V fragments are read from LDS, where they lie as in the registers (D = 128: two waves per SIMD need
// the registers).  Lanes behind the last key repeat it and store zeros.
// Bound by the matrix units' share of a SIMD's two waves and by LDS reads (48% and 35% of the time busy): 12 heads x
// 19200 rows x 512 keys, D = 128: 127 to 130 us, 930 to 954 TF.
template <int D, int NWK, int QG, int BM, int VL>
__global__ __launch_bounds__(64 * NWK * QG, 2) void cross_dkdv_kernel(CrossBwdParams p, int n_ktiles) {
  constexpr int NW = NWK * QG, BN = 32 * NWK, NT = 64 * NW, BS = BM * QG, KK = (D + 15) / 16, DB = D / 32;
  constexpr bool TAIL = D % 32 != 0;
  static_assert(16 * VL <= D, "the V fragments in LDS have no columns past D");
  using LD = KeyTileLds<D, NWK, QG, BM, VL>;
  constexpr int TE = LD::TE, RT = LD::RT;
  __shared__ __attribute__((aligned(16))) unsigned char lds[LD::BYTES];
  bf16_t(*Qs)[TE] = reinterpret_cast<bf16_t(*)[TE]>(lds);
  bf16_t(*Os)[TE] = reinterpret_cast<bf16_t(*)[TE]>(lds + 4 * TE);
  float(*lse_s)[RT] = reinterpret_cast<float(*)[RT]>(lds + 8 * TE);
  float(*dlt_s)[RT] = reinterpret_cast<float(*)[RT]>(lds + 8 * TE + 8 * RT);
  bf16_t* Vs = reinterpret_cast<bf16_t*>(lds + LD::STAGES);
  const int item = xcd_range(blockIdx.x, gridDim.x);
  const int group = item / n_ktiles, kt = item - group * n_ktiles, part = group / p.B, b = group - part * p.B;
  const int hk = part / p.n_slices, slice = part - hk * p.n_slices, bh = b * p.Hkv + hk;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kw = wave % NWK, qg = wave / NWK, gq = qg * BM;
  const int G = p.G, R = p.R;
  const int k0 = kt * BN, key = k0 + kw * 32 + (lane & 31), n = valid_keys(p, b);
  f32x16 dk[DB], dv[DB];
  f32x4 tail[4] = {zero4(), zero4(), zero4(), zero4()};  // (TAIL) dV^T, dK^T of keys 0..15 and 16..31
#pragma unroll
  for (int db = 0; db < DB; ++db) dk[db] = dv[db] = zero16();

  if (k0 < n) {
    bf16x8 kf[KK], vf[KK];
    const bf16_t* vfrag = Vs + (kw * VL * 64 + lane) * 8;
    auto load_keys = [&] {
      const long long kr = min(key, n - 1);
      const bf16_t* ka = p.k + b * p.sk.b + hk * p.sk.h + kr * p.sk.t + 8 * (lane >> 5);
      const bf16_t* va = p.v + b * p.sv.b + hk * p.sv.h + kr * p.sv.t + 8 * (lane >> 5);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        if (D % 16 == 0 || 16 * kk + 8 * (lane >> 5) < D) {
          kf[kk] = *reinterpret_cast<const bf16x8*>(ka + 16 * kk);
          vf[kk] = *reinterpret_cast<const bf16x8*>(va + 16 * kk);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) kf[kk][j] = vf[kk][j] = (__bf16)0.f;
        }
        if (kk < VL && qg == 0) *reinterpret_cast<bf16x8*>(Vs + ((kw * VL + kk) * 64 + lane) * 8) = vf[kk];
      }
    };
    const FragOffsets<D> fo(lane, gq * D);
    const Tail72 ft(lane, gq * D);
    const RowOffsets<D, BS, NT> ro_q(p.sq.t, tid), ro_o(p.sdo.t, tid);
    const long long qb = b * p.sq.b + hk * p.sq.h, ob = b * p.sdo.b + hk * p.sdo.h;
    const float* lse2 = p.lse2 + (long long)bh * R;
    const float* dlt = p.delta + (long long)bh * R;
    const int n_steps = (R + BS - 1) / BS;
    const int beg = (int)((long long)n_steps * slice / p.n_slices) * BS;
    const int end = min(R, (int)((long long)n_steps * (slice + 1) / p.n_slices) * BS);
    auto stage = [&](int r0, int buf) {
      if (G == 1 && r0 + BS <= R) {
        stage_rows_s<D, BS, NT>(Qs[buf], p.q + qb + r0 * p.sq.t, ro_q, tid);
        stage_rows_s<D, BS, NT>(Os[buf], p.d_o + ob + r0 * p.sdo.t, ro_o, tid);
      } else {
        stage_rows_direct<D, BS, NT>(Qs[buf], [&](int r) { return p.q + row_offset(p.sq, b, hk, G, min(r0 + r, R - 1)); },
                                     tid);
        stage_rows_direct<D, BS, NT>(Os[buf],
                                     [&](int r) { return p.d_o + row_offset(p.sdo, b, hk, G, min(r0 + r, R - 1)); }, tid);
      }
#pragma unroll
      for (int c = wave; c < 2 * (RT / 64); c += NW) {
        const int part = c % (RT / 64);
        if (c < RT / 64) {
          stage_f32x64_direct(lse_s[buf] + 64 * part, lse2, r0 + 64 * part, R, lane);
        } else {
          stage_f32x64_direct(dlt_s[buf] + 64 * part, dlt, r0 + 64 * part, R, lane);
        }
      }
    };
    const float c = p.scale_log2;
    // Matrix phases go first where a step is matrix products only (24 heads on 8, 9600 rows x 2048 keys, D = 64: the whole
    // backward 487 -> 468 us; D = 128, 12 heads: 429 -> 422 us); with the tail's lane exchanges, D = 72, it is 1% slower.
    constexpr bool PRIO = !TAIL;
    auto step = [&](auto ragged, int r0, int buf) {
#pragma unroll
      for (int qb = 0; qb < BM / 32; ++qb) {
        // the dP products start from -Delta of their rows
        f32x16 s = zero16(), dp;
        if constexpr (PRIO) __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 d4 = *reinterpret_cast<const f32x4*>(&dlt_s[buf][gq + qb * 32 + 8 * g + 4 * (lane >> 5)]);
#pragma unroll
          for (int j = 0; j < 4; ++j) dp[4 * g + j] = d4[j];
        }
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          s = mfma32(fo.row8(Qs[buf], qb * 32, kk), kf[kk], s);
          const bf16x8 vk = kk < VL ? *reinterpret_cast<const bf16x8*>(vfrag + kk * 512) : vf[kk];
          dp = mfma32(fo.row8(Os[buf], qb * 32, kk), vk, dp);
        }
        if constexpr (PRIO) __builtin_amdgcn_s_setprio(0);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int rr = gq + qb * 32 + 8 * g + 4 * (lane >> 5);
          const f32x4 l4 = *reinterpret_cast<const f32x4*>(&lse_s[buf][rr]);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int i = 4 * g + j;
            float pv = fast_exp2(fmaf(s[i], c, -l4[j]));
            if constexpr (decltype(ragged)::value) pv = r0 + rr + j < R ? pv : 0.f;
            s[i] = pv;
            dp[i] *= pv;
          }
        }
        // P, then dS, to the matrix products in bf16
        bf16x8 h[2] = {pack8(s, 0), pack8(s, 1)};
        if constexpr (PRIO) __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int db = 0; db < DB; ++db) dv[db] = mfma32(fo.tr8(Os[buf], qb * 32, t, db), h[t], dv[db]);
        if constexpr (TAIL) {
          tail_operands(h[0], h[1]);
          const bf16x8 x = ft.read(Os[buf], qb * 32);
#pragma unroll
          for (int e = 0; e < 2; ++e) tail[e] = mfma16(x, h[e], tail[e]);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          h[t] = pack8(dp, t);
#pragma unroll
          for (int db = 0; db < DB; ++db) dk[db] = mfma32(fo.tr8(Qs[buf], qb * 32, t, db), h[t], dk[db]);
        }
        if constexpr (TAIL) {
          tail_operands(h[0], h[1]);
          const bf16x8 x = ft.read(Qs[buf], qb * 32);
#pragma unroll
          for (int e = 0; e < 2; ++e) tail[2 + e] = mfma16(x, h[e], tail[2 + e]);
        }
      }
    };
    if (beg < end) {
      stage(beg, 0);  // ahead of the keys, whose V fragments are waited for on their way into LDS
      load_keys();
      wait_vmem();
      __syncthreads();
      int buf = 0;
      int r0 = beg;
      auto run = [&](auto ragged, int stop) {
        for (; r0 < stop; r0 += BS) {
          if (r0 + BS < end) stage(r0 + BS, buf ^ 1);
          if (k0 + kw * 32 < n) step(ragged, r0, buf);
          if constexpr (PRIO) __builtin_amdgcn_s_setprio(0);
          wait_vmem();
          __syncthreads();
          buf ^= 1;
        }
      };
      run(std::false_type{}, min(end, R / BS * BS));
      run(std::true_type{}, end);
    }
  }

  if constexpr (QG > 1) {
    float* m = reinterpret_cast<float*>(lds);
    add_groups<QG, NWK>(dv, qg, kw, lane, m);
    add_groups<QG, NWK>(dk, qg, kw, lane, m);
    if constexpr (TAIL) {
      f32x16 all[1];
#pragma unroll
      for (int i = 0; i < 16; ++i) all[0][i] = tail[i / 4][i % 4];
      add_groups<QG, NWK>(all, qg, kw, lane, m);
#pragma unroll
      for (int i = 0; i < 16; ++i) tail[i / 4][i % 4] = all[0][i];
    }
    if (qg > 0) return;  // no barrier follows
  }
  if (p.n_slices > 1) {
    const long long half = (long long)p.B * p.Hkv * p.M * D;
    float* pk = p.part + slice * 2 * half + (long long)bh * p.M * D;  // dK; dV half further on
    if constexpr (TAIL) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int kr = k0 + kw * 32 + 16 * e + (lane & 15);
        if (lane < 32 && kr < n) {
          float* x = pk + (long long)kr * D + 64 + 4 * (lane >> 4);
          *reinterpret_cast<f32x4*>(x) = tail[2 + e];
          *reinterpret_cast<f32x4*>(x + half) = tail[e];
        }
      }
    }
    if (key >= n) return;  // (the last kernel reads valid keys only)
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 wk, wv;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          wk[j] = dk[db][4 * g + j];
          wv[j] = dv[db][4 * g + j];
        }
        float* x = pk + (long long)key * D + db * 32 + 8 * g + 4 * (lane >> 5);
        *reinterpret_cast<f32x4*>(x) = wk;
        *reinterpret_cast<f32x4*>(x + half) = wv;
      }
    return;
  }
  if constexpr (TAIL) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int kr = k0 + kw * 32 + 16 * e + (lane & 15), col = 64 + 4 * (lane >> 4);
      if (lane < 32 && kr < p.M) {
        bf16x4 wk, wv;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          wk[j] = to_bf16(kr < n ? tail[2 + e][j] * p.scale : 0.f);
          wv[j] = to_bf16(kr < n ? tail[e][j] : 0.f);
        }
        *reinterpret_cast<bf16x4*>(p.dk + b * p.sdk.b + hk * p.sdk.h + kr * p.sdk.t + col) = wk;
        *reinterpret_cast<bf16x4*>(p.dv + b * p.sdv.b + hk * p.sdv.h + kr * p.sdv.t + col) = wv;
      }
    }
  }
  if (key >= p.M) return;
  bf16_t* dkr = p.dk + b * p.sdk.b + hk * p.sdk.h + key * p.sdk.t;
  bf16_t* dvr = p.dv + b * p.sdv.b + hk * p.sdv.h + key * p.sdv.t;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      bf16x4 wk, wv;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        wk[j] = to_bf16(key < n ? dk[db][4 * g + j] * p.scale : 0.f);
        wv[j] = to_bf16(key < n ? dv[db][4 * g + j] : 0.f);
      }
      const int col = db * 32 + 8 * g + 4 * (lane >> 5);
      *reinterpret_cast<bf16x4*>(dkr + col) = wk;
      *reinterpret_cast<bf16x4*>(dvr + col) = wv;
    }
}

// dQ: NW waves of 32 rows each (Q and dO fragments, dQ^T in registers), walking the keys of range `split`, BN a step.
// Few keys a row and long prologues (Q, dO and O of every row are read once): the same 12 heads 115 us, 790 TF, the
// matrix units busy 41% of it.  (D = 72 at three waves a SIMD spills six registers, 28 bytes a lane.)
template <int D, int NW, int BN, int WPS>
__global__ __launch_bounds__(64 * NW, WPS) void cross_dq_kernel(CrossBwdParams p, int n_rtiles) {
  constexpr int BM = 32 * NW, NT = 64 * NW, KK = (D + 15) / 16, DB = D / 32;
  constexpr bool TAIL = D % 32 != 0;
  constexpr int TE = stage_elems<D, BN, NT>();
  __shared__ __attribute__((aligned(16))) bf16_t lds[2][2][TE];
  bf16_t(*Ks)[TE] = lds[0];
  bf16_t(*Vs)[TE] = lds[1];
  const int item = xcd_range(blockIdx.x, gridDim.x);
  const int group = item / n_rtiles, rt = item - group * n_rtiles, part = group / p.B, b = group - part * p.B;
  const int hk = part / p.n_ranges, split = part - hk * p.n_ranges, bh = b * p.Hkv + hk;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = p.G, R = p.R;
  const int row = rt * BM + wave * 32 + (lane & 31), rc = min(row, R - 1);
  // This row's Q, dO and O, asked for before anything that waits (the number of keys, the first keys): their latencies
  // then pass together.
  bf16x8 qf[KK], of[KK], y[KK];
  {
    const bf16_t* qa = p.q + row_offset(p.sq, b, hk, G, rc) + 8 * (lane >> 5);
    const bf16_t* da = p.d_o + row_offset(p.sdo, b, hk, G, rc) + 8 * (lane >> 5);
    const bf16_t* oa = p.o + row_offset(p.so, b, hk, G, rc) + 8 * (lane >> 5);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      if (D % 16 == 0 || 16 * kk + 8 * (lane >> 5) < D) {
        of[kk] = *reinterpret_cast<const bf16x8*>(da + 16 * kk);
        y[kk] = *reinterpret_cast<const bf16x8*>(oa + 16 * kk);
        qf[kk] = *reinterpret_cast<const bf16x8*>(qa + 16 * kk);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) qf[kk][j] = of[kk][j] = y[kk][j] = (__bf16)0.f;
      }
    }
  }
  const int row_t = rc / G;
  const float lse = p.lse[((long long)b * p.Hkv * G + hk * G + (rc - row_t * G)) * p.T + row_t];
  const int n = valid_keys(p, b);
  f32x16 dq[DB];
  f32x4 tail[2] = {zero4(), zero4()};
#pragma unroll
  for (int db = 0; db < DB; ++db) dq[db] = zero16();
  // (a batch member without a key has no use for the row terms either)
  const int steps = (n + BN - 1) / BN;
  const int beg = (int)((long long)steps * split / p.n_ranges) * BN;
  const int end = min(n, (int)((long long)steps * (split + 1) / p.n_ranges) * BN);
  if (n > 0) {
    const FragOffsets<D> fo(lane, 0);
    const Tail72 ft(lane, 0);
    const long long kb = b * p.sk.b + hk * p.sk.h, vb = b * p.sv.b + hk * p.sv.h;
    const RowOffsets<D, BN, NT> ro_k(p.sk.t, tid), ro_v(p.sv.t, tid);
    auto stage = [&](int k0, int buf) {
      if (k0 + BN <= n) {
        stage_rows_s<D, BN, NT>(Ks[buf], p.k + kb + k0 * p.sk.t, ro_k, tid);
        stage_rows_s<D, BN, NT>(Vs[buf], p.v + vb + k0 * p.sv.t, ro_v, tid);
      } else {
        stage_kv_rows_direct<D, BN, NT>(Ks[buf], Vs[buf], [&](int r) -> RowPair {
          const long long j = min(k0 + r, n - 1);
          return {p.k + kb + j * p.sk.t, p.v + vb + j * p.sv.t};
        }, tid);
      }
    };
    if (beg < end) stage(beg, 0);
    float dot = 0.f;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int j = 0; j < 8; ++j) dot = fmaf((float)of[kk][j], (float)y[kk][j], dot);
    float ndlt = -sum_halves(dot);
    const float c = p.scale_log2, lse2 = lse * 1.4426950408889634f;
    wait_vmem();
    __syncthreads();
    // Keys of a single step: Delta = sum_j P_j dP_j of the probabilities at hand.  rowsum(dO O) has O's rounding to bf16,
    // which next to few keys' dP - Delta is no longer small (2 keys: dK 0.0043 off, relative to its norm; so 0.0023,
    // which is the rounding of dS and of dK itself; from 64 keys on it is below a tenth of those).
    const bool few = n <= BN;
    if (few && beg < end) {
      float sum = 0.f;
#pragma unroll 1
      for (int kq = 0; kq < BN / 32; ++kq) {
        f32x16 s = zero16(), dp = zero16();
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          s = mfma32(fo.row8(Ks[0], kq * 32, kk), qf[kk], s);
          dp = mfma32(fo.row8(Vs[0], kq * 32, kk), of[kk], dp);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const bool in = kq * 32 + acc_row(i, lane) < n;
          sum = fmaf(in ? fast_exp2(fmaf(s[i], c, -lse2)) : 0.f, in ? dp[i] : 0.f, sum);
        }
      }
      ndlt = -sum_halves(sum);
    }
    if ((few ? beg < end : split == 0) && lane < 32 && row < R) {
      p.delta[(long long)bh * R + row] = ndlt;
      p.lse2[(long long)bh * R + row] = lse2;
    }
    f32x16 nd;
#pragma unroll
    for (int i = 0; i < 16; ++i) nd[i] = ndlt;
    auto step = [&](auto ragged, int k0, int buf) {
#pragma unroll
      for (int kq = 0; kq < BN / 32; ++kq) {
        if (decltype(ragged)::value && k0 + kq * 32 >= n) break;
        f32x16 s = zero16(), dp = nd;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          s = mfma32(fo.row8(Ks[buf], kq * 32, kk), qf[kk], s);
          dp = mfma32(fo.row8(Vs[buf], kq * 32, kk), of[kk], dp);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float pv = fast_exp2(fmaf(s[i], c, -lse2));
          if constexpr (decltype(ragged)::value) pv = k0 + kq * 32 + acc_row(i, lane) < n ? pv : 0.f;
          dp[i] *= pv;
        }
        bf16x8 h[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          h[t] = pack8(dp, t);
#pragma unroll
          for (int db = 0; db < DB; ++db) dq[db] = mfma32(fo.tr8(Ks[buf], kq * 32, t, db), h[t], dq[db]);
        }
        if constexpr (TAIL) {
          const bf16x8 x = ft.read(Ks[buf], kq * 32);
          tail_operands(h[0], h[1]);
#pragma unroll
          for (int e = 0; e < 2; ++e) tail[e] = mfma16(x, h[e], tail[e]);
        }
      }
    };
    int buf = 0, k0 = beg;
    auto run = [&](auto ragged, int stop) {
      for (; k0 < stop; k0 += BN) {
        if (k0 + BN < end) stage(k0 + BN, buf ^ 1);
        step(ragged, k0, buf);
        wait_vmem();
        __syncthreads();
        buf ^= 1;
      }
    };
    run(std::false_type{}, min(end, n / BN * BN));
    run(std::true_type{}, end);
  }
  if (p.n_ranges > 1) {  // fp32 dQ of this key range
    float* part = p.part_q + ((long long)split * p.B * p.Hkv + bh) * R * D;
    if constexpr (TAIL) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = rt * BM + wave * 32 + 16 * e + (lane & 15);
        if (lane < 32 && r < R) *reinterpret_cast<f32x4*>(part + (long long)r * D + 64 + 4 * (lane >> 4)) = tail[e];
      }
    }
    if (row >= R) return;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = dq[db][4 * g + j];
        *reinterpret_cast<f32x4*>(part + (long long)row * D + db * 32 + 8 * g + 4 * (lane >> 5)) = w;
      }
    return;
  }
  // (every wave has passed the last barrier: a half stage holds the rows of BN / 32 waves)
  static_assert(NW <= 2 * (BN / 32), "one stage holds the rows of every wave");
  const int r0 = rt * BM + wave * 32, half = wave / (BN / 32);
  store_rows<D>(dq, tail, (half ? Vs : Ks)[0] + (wave - half * (BN / 32)) * 32 * D, min(32, R - r0), lane, p.scale,
                [&](int r) { return p.dq + row_offset(p.sdq, b, hk, G, r0 + r); });
}

// Sums of the slices (dK, dV; zeros for the padding keys) and of the key ranges (dQ), each in order.  One thread
// for four columns of a row; the first n_kv workgroups take the keys.
template <int D>
__global__ __launch_bounds__(256) void cross_join_kernel(CrossBwdParams p, int n_kv) {
  constexpr int TPR = D / 4;
  if ((int)blockIdx.x < n_kv) {
    const long long rows = (long long)p.B * p.Hkv * p.M, gid = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long kr = gid / TPR;
    if (kr >= rows) return;
    const int col = (int)(gid - kr * TPR) * 4;
    const int bh = (int)(kr / p.M), key = (int)(kr - (long long)bh * p.M), b = bh / p.Hkv, hk = bh - b * p.Hkv;
    f32x4 k = zero4(), v = zero4();
    if (key < valid_keys(p, b)) {
      const long long half = rows * D;
      const float* x = p.part + kr * D + col;
#pragma unroll 4
      for (int s = 0; s < p.n_slices; ++s) {
        k += *reinterpret_cast<const f32x4*>(x + 2 * s * half);
        v += *reinterpret_cast<const f32x4*>(x + (2 * s + 1) * half);
      }
    }
    bf16x4 wk, wv;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      wk[j] = to_bf16(k[j] * p.scale);
      wv[j] = to_bf16(v[j]);
    }
    *reinterpret_cast<bf16x4*>(p.dk + b * p.sdk.b + hk * p.sdk.h + key * p.sdk.t + col) = wk;
    *reinterpret_cast<bf16x4*>(p.dv + b * p.sdv.b + hk * p.sdv.h + key * p.sdv.t + col) = wv;
    return;
  }
  const long long rows = (long long)p.B * p.Hkv * p.R, gid = (long long)(blockIdx.x - n_kv) * 256 + threadIdx.x;
  const long long rr = gid / TPR;
  if (rr >= rows) return;
  const int col = (int)(gid - rr * TPR) * 4;
  const int bh = (int)(rr / p.R), r = (int)(rr - (long long)bh * p.R), b = bh / p.Hkv, hk = bh - b * p.Hkv;
  f32x4 q = zero4();
#pragma unroll 4
  for (int s = 0; s < p.n_ranges; ++s) q += *reinterpret_cast<const f32x4*>(p.part_q + (s * rows + rr) * D + col);
  bf16x4 w;
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = to_bf16(q[j] * p.scale);
  *reinterpret_cast<bf16x4*>(p.dq + row_offset(p.sdq, b, hk, p.G, r) + col) = w;
}

template <int NWK, int QG, int BM, int VL>
hipError_t launch_dkdv(const CrossBwdParams& p, hipStream_t stream) {
  const int n_ktiles = (p.M + 32 * NWK - 1) / (32 * NWK);
  const long long grid = (long long)p.B * p.Hkv * n_ktiles * p.n_slices;
  if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
  hipLaunchKernelGGL((cross_dkdv_kernel<kD, NWK, QG, BM, VL>), dim3((unsigned)grid), dim3(64 * NWK * QG), 0, stream, p,
                     n_ktiles);
  return hipGetLastError();
}

}  // namespace

#define MW_CAT_(a, b) a##b
#define MW_CAT(a, b) MW_CAT_(a, b)
hipError_t MW_CAT(launch_cross_bwd_, MW_CROSS_HEAD_DIM)(const CrossBwdParams& p, hipStream_t stream) {
  constexpr int NW = 4;
  const int n_rtiles = (p.R + 32 * NW - 1) / (32 * NW);
  const long long grid = (long long)p.B * p.Hkv * n_rtiles * p.n_ranges;
  if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
  hipLaunchKernelGGL((cross_dq_kernel<kD, NW, 64, kD == 128 ? 2 : 3>), dim3((unsigned)grid), dim3(64 * NW), 0, stream, p,
                     n_rtiles);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  e = p.key_waves == 2 ? launch_dkdv<2, 4, 32, kD == 128 ? 7 : 0>(p, stream) : launch_dkdv<4, 2, 32, kD == 128 ? 6 : 0>(p, stream);
  if (e != hipSuccess || (p.n_slices == 1 && p.n_ranges == 1)) return e;
  const long long bhkv = (long long)p.B * p.Hkv;
  const long long n_kv = p.n_slices > 1 ? (bhkv * p.M * (kD / 4) + 255) / 256 : 0;
  const long long n_q = p.n_ranges > 1 ? (bhkv * p.R * (kD / 4) + 255) / 256 : 0;
  hipLaunchKernelGGL(cross_join_kernel<kD>, dim3((unsigned)(n_kv + n_q)), dim3(256), 0, stream, p, (int)n_kv);
  return hipGetLastError();
}

#if MW_CROSS_HEAD_DIM == 128
// Key waves and row slices of the dK/dV kernel and key ranges of the dQ kernel, by a price for each choice.  A round of
// the workgroups that are resident together begins with `begin` us; a step of 64 keys (or 32 * 8 / key waves rows) takes
// `lone` us where a workgroup has its CU for itself and `shared` us of the CU for each where it has not.  The join costs a
// launch, its partials' transfer and time for each slice and range.  The constants are a least-squares fit to 55160
// timings of 5712 shapes (1 to 64 key heads, up to 60000 rows and 12000 keys): the plans taken are on average 0.6% (at
// the 90th percentile 2.3%) off the fastest; one dK/dV workgroup and two dQ workgroups a CU as a rule were 5% (12%).
struct BwdPrice {
  int occ_q, occ_k;
  double begin_q, lone_q, shared_q, begin_k, lone_k[2], shared_k[2];  // [0]: two key waves, [1]: four
  double join, per_mb, per_part;
};
const BwdPrice& bwd_price(int D) {
  static const BwdPrice d64 = {3, 2, 8.16, 1.11, 0.81, 4.92, {1.32, 0.97}, {1.32, 0.94}, 2.79, 0.379, 0.124};
  static const BwdPrice d72 = {3, 1, 9.17, 1.33, 0.97, 4.14, {1.49, 1.15}, {1.49, 1.15}, 2.77, 0.268, 0.103};
  static const BwdPrice d128 = {2, 1, 10.52, 1.76, 1.39, 5.42, {2.16, 1.61}, {2.16, 1.61}, 3.69, 0.321, 0.101};
  return D == 64 ? d64 : (D == 72 ? d72 : d128);
}

// Time of `n` workgroups of `steps` steps each.
double rounds_us(long long n, long long steps, int occ, double begin, double lone, double shared) {
  const double busiest = (double)((n + 255) / 256), k = std::min(busiest, (double)occ);
  return busiest / k * (begin + steps * std::max(lone, k * shared));
}

CrossBwdPlan cross_bwd_plan(int D, int BHkv, int R, int M) {
  const BwdPrice& c = bwd_price(D);
  // the best without and with parts, of either kernel
  struct Best {
    double us = 1e300;
    int parts = 1, key_waves = 4;
  } dq[2], dkv[2];
  const auto offer = [](Best& x, double us, int parts, int key_waves) {
    if (us < x.us) x = {us, parts, key_waves};
  };
  const long long q_steps = (M + 63) / 64, q_tiles = (long long)BHkv * ((R + 127) / 128);
  const double q_mb = (double)BHkv * R * D * 4e-6, kv_mb = (double)BHkv * M * D * 8e-6;
  for (int n = 1; n <= std::min(64LL, q_steps); ++n) {
    const double t = rounds_us(q_tiles * n, (q_steps + n - 1) / n, c.occ_q, c.begin_q, c.lone_q, c.shared_q);
    offer(dq[n > 1], n > 1 ? t + n * (c.per_mb * q_mb + c.per_part) : t, n, 0);
  }
  for (const int kw : {2, 4}) {
    const int rows = 32 * (8 / kw), i = kw / 2 - 1;
    const long long steps = (R + rows - 1) / rows, tiles = (long long)BHkv * ((M + 32 * kw - 1) / (32 * kw));
    for (int n = 1; n <= std::min(64LL, steps); ++n) {
      const double t = rounds_us(tiles * n, (steps + n - 1) / n, c.occ_k, c.begin_k, c.lone_k[i], c.shared_k[i]);
      offer(dkv[n > 1], n > 1 ? t + n * (c.per_mb * kv_mb + c.per_part) : t, n, kw);
    }
  }
  CrossBwdPlan plan{4, 1, 1};
  double best = 1e300;
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2; ++j) {
      const double t = dq[i].us + dkv[j].us + (i + j > 0 ? c.join : 0.0);
      if (t < best) {
        best = t;
        plan = {dkv[j].key_waves, dkv[j].parts, dq[i].parts};
      }
    }
  return plan;
}
#endif

}  // namespace mw
