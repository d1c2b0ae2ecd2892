// Backward of the cross attention (gfx950): with P recomputed from Q, K and the forward's LSE,
//   dV = sum_r P_r^T dO_r,  dP = dO V^T,  Delta = rowsum(dO O),  dS = P (dP - Delta),
//   dQ = scale dS K,  dK = scale sum_r dS_r^T Q_r
// over the rows r of a key head (its query heads' tokens, attn_rows.h), so that the gradients of
// shared heads are sums over more rows and need nothing else.
//
//   row terms  : -Delta and LSE log2 e, one pass over O and dO;
//   one grid   : dK/dV work (a tile of keys held in registers walks a slice of the rows) and
//                dQ work (a tile of rows walks the keys);
//   slices     : the rows are many and the keys few, so the rows of a key tile are cut into
//                slices that fill the card; each leaves fp32 dK, dV, which the last kernel adds in
//                slice order.  No atomics: the result is deterministic.
#include <algorithm>
#include <type_traits>

#include "attn_rows.h"

namespace mw {

namespace {

constexpr int kD = MW_CROSS_HEAD_DIM;

template <int D>
__global__ __launch_bounds__(256) void cross_rowterms_kernel(CrossBwdParams p) {
  constexpr int CPR = D == 64 ? 8 : 16;  // lanes per row (D = 72: nine of 16 have a piece)
  const long long gid = (long long)blockIdx.x * 256 + threadIdx.x, n_rows = (long long)p.B * p.Hkv * p.R;
  const long long rr = gid / CPR;
  const int c = (int)(gid % CPR);
  float acc = 0.f;
  int b = 0, h = 0, t = 0;
  if (rr < n_rows) {
    const long long bh = rr / p.R;
    const int r = (int)(rr - bh * p.R);
    t = r / p.G;
    b = (int)(bh / p.Hkv);
    h = (int)(bh - (long long)b * p.Hkv) * p.G + (r - t * p.G);
    if (c < D / 8) {
      const bf16x8 x = *reinterpret_cast<const bf16x8*>(p.o + b * p.so.b + h * p.so.h + t * p.so.t + c * 8);
      const bf16x8 y = *reinterpret_cast<const bf16x8*>(p.d_o + b * p.sdo.b + h * p.sdo.h + t * p.sdo.t + c * 8);
#pragma unroll
      for (int j = 0; j < 8; ++j) acc = fmaf((float)x[j], (float)y[j], acc);
    }
  }
#pragma unroll
  for (int w = CPR / 2; w >= 1; w >>= 1) acc += __shfl_xor(acc, w);
  if (rr < n_rows && c == 0) {
    const float l = p.lse[((long long)b * p.Hkv * p.G + h) * p.T + t];
    p.delta[rr] = -acc;
    p.lse2[rr] = l == -INFINITY ? INFINITY : l * 1.4426950408889634f;  // a row without a key: P = 0
  }
}

// Valid keys of batch member b.
__device__ __forceinline__ int valid_keys(const CrossBwdParams& p, int b) {
  return p.kv_len == nullptr ? p.M : max(0, min(p.M, p.kv_len[b]));
}

// Work items [0, n) of a part of the grid that starts at a multiple of 8: XCD x gets one contiguous range.
__device__ __forceinline__ int xcd_range(int id, int n) {
  const int x = id % 8, q = n / 8, rem = n % 8;
  return x * q + min(x, rem) + id / 8;
}

template <int D, int NW, int BM>
struct CrossLds {
  static constexpr int TE = stage_elems<D, BM, 64 * NW>();
  static constexpr int RT = BM < 64 ? 64 : BM;
  static constexpr int BYTES = 2 * 2 * TE * 2 + 2 * 2 * RT * 4;
};

// dK/dV work: a wave owns 32 keys (K and V fragments, dK^T and dV^T in registers) and walks rows
// [beg, end) of the key head, BM a step, staged in LDS.  Lanes behind the last key repeat it and
// store zeros.
template <int D, int NW, int BM>
__device__ __forceinline__ void dkdv_work(const CrossBwdParams& p, int bh, int kt, int slice, unsigned char* lds) {
  constexpr int BN = 32 * NW, NT = 64 * NW, KK = (D + 15) / 16, DB = D / 32;
  constexpr bool TAIL = D % 32 != 0;
  using LD = CrossLds<D, NW, BM>;
  constexpr int TE = LD::TE, RT = LD::RT;
  bf16_t(*Qs)[TE] = reinterpret_cast<bf16_t(*)[TE]>(lds);
  bf16_t(*Os)[TE] = reinterpret_cast<bf16_t(*)[TE]>(lds + 4 * TE);
  float(*lse_s)[RT] = reinterpret_cast<float(*)[RT]>(lds + 8 * TE);
  float(*dlt_s)[RT] = reinterpret_cast<float(*)[RT]>(lds + 8 * TE + 8 * RT);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int b = bh / p.Hkv, hk = bh - b * p.Hkv, G = p.G, R = p.R;
  const int k0 = kt * BN, key = k0 + wave * 32 + (lane & 31), n = valid_keys(p, b);
  f32x16 dk[DB], dv[DB];
  f32x4 tail[4] = {zero4(), zero4(), zero4(), zero4()};  // (TAIL) dV^T, dK^T of keys 0..15 and 16..31
#pragma unroll
  for (int db = 0; db < DB; ++db) dk[db] = dv[db] = zero16();

  if (k0 < n) {
    bf16x8 kf[KK], vf[KK];
    {
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
      }
    }
    const FragOffsets<D> fo(lane, 0);
    const Tail72 ft(lane, 0);
    const RowOffsets<D, BM, NT> ro_q(p.sq.t, tid), ro_o(p.sdo.t, tid);
    const long long qb = b * p.sq.b + hk * p.sq.h, ob = b * p.sdo.b + hk * p.sdo.h;
    const float* lse2 = p.lse2 + (long long)bh * R;
    const float* dlt = p.delta + (long long)bh * R;
    const int n_steps = (R + BM - 1) / BM;
    const int beg = (int)((long long)n_steps * slice / p.n_slices) * BM;
    const int end = min(R, (int)((long long)n_steps * (slice + 1) / p.n_slices) * BM);
    auto stage = [&](int r0, int buf) {
      if (G == 1 && r0 + BM <= R) {
        stage_rows_s<D, BM, NT>(Qs[buf], p.q + qb + r0 * p.sq.t, ro_q, tid);
        stage_rows_s<D, BM, NT>(Os[buf], p.d_o + ob + r0 * p.sdo.t, ro_o, tid);
      } else {
        stage_rows_direct<D, BM, NT>(Qs[buf], [&](int r) { return p.q + row_offset(p.sq, b, hk, G, min(r0 + r, R - 1)); },
                                     tid);
        stage_rows_direct<D, BM, NT>(Os[buf],
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
    auto step = [&](auto ragged, int r0, int buf) {
#pragma unroll
      for (int qb = 0; qb < BM / 32; ++qb) {
        // the dP products start from -Delta of their rows
        f32x16 s = zero16(), dp;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 d4 = *reinterpret_cast<const f32x4*>(&dlt_s[buf][qb * 32 + 8 * g + 4 * (lane >> 5)]);
#pragma unroll
          for (int j = 0; j < 4; ++j) dp[4 * g + j] = d4[j];
        }
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          s = mfma32(fo.row8(Qs[buf], qb * 32, kk), kf[kk], s);
          dp = mfma32(fo.row8(Os[buf], qb * 32, kk), vf[kk], dp);
        }
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int rr = qb * 32 + 8 * g + 4 * (lane >> 5);
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
      stage(beg, 0);
      wait_vmem();
      __syncthreads();
      int buf = 0;
      for (int r0 = beg; r0 < end; r0 += BM) {
        if (r0 + BM < end) stage(r0 + BM, buf ^ 1);
        if (r0 + BM <= R) {
          step(std::false_type{}, r0, buf);
        } else {
          step(std::true_type{}, r0, buf);
        }
        wait_vmem();
        __syncthreads();
        buf ^= 1;
      }
    }
  }

  if (p.n_slices > 1) {
    const long long half = (long long)p.B * p.Hkv * p.M * D;
    float* pk = p.part + slice * 2 * half + (long long)bh * p.M * D;  // dK; dV half further on
    if constexpr (TAIL) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int kr = k0 + wave * 32 + 16 * e + (lane & 15);
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
      const int kr = k0 + wave * 32 + 16 * e + (lane & 15), col = 64 + 4 * (lane >> 4);
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

// dQ work: a wave owns 32 rows (Q and dO fragments, dQ^T in registers) and walks the keys, BN a step.
template <int D, int NW, int BN>
__device__ __forceinline__ void dq_work(const CrossBwdParams& p, int bh, int rt, unsigned char* lds) {
  constexpr int BM = 32 * NW, NT = 64 * NW, KK = (D + 15) / 16, DB = D / 32;
  constexpr bool TAIL = D % 32 != 0;
  constexpr int TE = stage_elems<D, BN, NT>();
  bf16_t(*Ks)[TE] = reinterpret_cast<bf16_t(*)[TE]>(lds);
  bf16_t(*Vs)[TE] = reinterpret_cast<bf16_t(*)[TE]>(lds + 4 * TE);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int b = bh / p.Hkv, hk = bh - b * p.Hkv, G = p.G, R = p.R;
  const int row = rt * BM + wave * 32 + (lane & 31), rc = min(row, R - 1), n = valid_keys(p, b);
  f32x16 dq[DB];
  f32x4 tail[2] = {zero4(), zero4()};
#pragma unroll
  for (int db = 0; db < DB; ++db) dq[db] = zero16();
  if (n > 0) {
    bf16x8 qf[KK], of[KK];
    const bf16_t* qa = p.q + row_offset(p.sq, b, hk, G, rc) + 8 * (lane >> 5);
    const bf16_t* oa = p.d_o + row_offset(p.sdo, b, hk, G, rc) + 8 * (lane >> 5);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      if (D % 16 == 0 || 16 * kk + 8 * (lane >> 5) < D) {
        qf[kk] = *reinterpret_cast<const bf16x8*>(qa + 16 * kk);
        of[kk] = *reinterpret_cast<const bf16x8*>(oa + 16 * kk);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) qf[kk][j] = of[kk][j] = (__bf16)0.f;
      }
    }
    const float lse2 = p.lse2[(long long)bh * R + rc], ndlt = p.delta[(long long)bh * R + rc], c = p.scale_log2;
    f32x16 nd;
#pragma unroll
    for (int i = 0; i < 16; ++i) nd[i] = ndlt;
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
    auto step = [&](auto ragged, int k0, int buf) {
#pragma unroll
      for (int kq = 0; kq < BN / 32; ++kq) {
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
    stage(0, 0);
    wait_vmem();
    __syncthreads();
    int buf = 0;
    for (int k0 = 0; k0 < n; k0 += BN) {
      if (k0 + BN < n) stage(k0 + BN, buf ^ 1);
      if (k0 + BN <= n) {
        step(std::false_type{}, k0, buf);
      } else {
        step(std::true_type{}, k0, buf);
      }
      wait_vmem();
      __syncthreads();
      buf ^= 1;
    }
  }
  if constexpr (TAIL) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = rt * BM + wave * 32 + 16 * e + (lane & 15);
      if (lane < 32 && r < R) {
        bf16x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = to_bf16(tail[e][j] * p.scale);
        *reinterpret_cast<bf16x4*>(p.dq + row_offset(p.sdq, b, hk, G, r) + 64 + 4 * (lane >> 4)) = w;
      }
    }
  }
  if (row >= R) return;
  bf16_t* dst = p.dq + row_offset(p.sdq, b, hk, G, row);
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      bf16x4 w;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = to_bf16(dq[db][4 * g + j] * p.scale);
      *reinterpret_cast<bf16x4*>(dst + db * 32 + 8 * g + 4 * (lane >> 5)) = w;
    }
}

template <int D, int NW, int BMK, int BNQ, int WPS>
__global__ __launch_bounds__(64 * NW, WPS) void cross_grad_kernel(CrossBwdParams p, int n_dkdv, int first_dq, int n_ktiles,
                                                                  int n_rtiles) {
  constexpr int B1 = CrossLds<D, NW, BMK>::BYTES, B2 = 8 * stage_elems<D, BNQ, 64 * NW>();
  __shared__ __attribute__((aligned(16))) unsigned char lds[B1 > B2 ? B1 : B2];
  const int id = blockIdx.x;
  if (id < first_dq) {
    if (id >= n_dkdv) return;  // (the dQ work starts at a multiple of 8)
    const int item = xcd_range(id, n_dkdv);
    const int per = n_ktiles * p.n_slices, bh = item / per, x = item - bh * per, slice = x / n_ktiles;
    dkdv_work<D, NW, BMK>(p, bh, x - slice * n_ktiles, slice, lds);
  } else {
    const int item = xcd_range(id - first_dq, (int)gridDim.x - first_dq);
    const int bh = item / n_rtiles;
    dq_work<D, NW, BNQ>(p, bh, item - bh * n_rtiles, lds);
  }
}

// dK and dV: the slices' sums in slice order, and zeros for the padding keys.  One thread for four columns.
template <int D>
__global__ __launch_bounds__(256) void cross_join_kernel(CrossBwdParams p) {
  constexpr int TPR = D / 4;
  const long long rows = (long long)p.B * p.Hkv * p.M, gid = (long long)blockIdx.x * 256 + threadIdx.x;
  const long long kr = gid / TPR;
  if (kr >= rows) return;
  const int col = (int)(gid - kr * TPR) * 4;
  const int bh = (int)(kr / p.M), key = (int)(kr - (long long)bh * p.M), b = bh / p.Hkv, hk = bh - b * p.Hkv;
  f32x4 k = zero4(), v = zero4();
  if (key < valid_keys(p, b)) {
    const long long half = rows * D;
    const float* x = p.part + kr * D + col;
    for (int s = 0; s < p.n_slices; ++s, x += 2 * half) {
      k += *reinterpret_cast<const f32x4*>(x);
      v += *reinterpret_cast<const f32x4*>(x + half);
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
}

}  // namespace

#define MW_CAT_(a, b) a##b
#define MW_CAT(a, b) MW_CAT_(a, b)
hipError_t MW_CAT(launch_cross_bwd_, MW_CROSS_HEAD_DIM)(const CrossBwdParams& p, hipStream_t stream) {
  const long long rows = (long long)p.B * p.Hkv * p.R, threads = rows * (kD == 64 ? 8 : 16);
  hipLaunchKernelGGL(cross_rowterms_kernel<kD>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  constexpr int NW = 4;
  const int n_ktiles = (p.M + 32 * NW - 1) / (32 * NW), n_rtiles = (p.R + 32 * NW - 1) / (32 * NW);
  const long long n_dkdv = (long long)p.B * p.Hkv * n_ktiles * p.n_slices, first_dq = (n_dkdv + 7) / 8 * 8;
  const long long grid = first_dq + (long long)p.B * p.Hkv * n_rtiles;
  if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
  hipLaunchKernelGGL((cross_grad_kernel<kD, NW, kD == 128 ? 32 : 64, 64, kD == 128 ? 1 : 2>), dim3((unsigned)grid),
                     dim3(64 * NW), 0, stream, p, (int)n_dkdv, (int)first_dq, n_ktiles, n_rtiles);
  e = hipGetLastError();
  if (e != hipSuccess || p.n_slices == 1) return e;
  const long long n = (long long)p.B * p.Hkv * p.M * (kD / 4);
  hipLaunchKernelGGL(cross_join_kernel<kD>, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, stream, p);
  return hipGetLastError();
}

#if MW_CROSS_HEAD_DIM == 128
int cross_bwd_slices(int D, int BHkv, int R, int M) {
  (void)D;
  const long long tiles = (long long)BHkv * ((M + 127) / 128);
  return (int)std::max(1LL, std::min({(256 + tiles - 1) / tiles, (long long)R / 256, 64LL}));
}
#endif

}  // namespace mw
