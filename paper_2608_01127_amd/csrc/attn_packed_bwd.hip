// Backward of the packed attention (gfx950): with P recomputed from Q, K and the forward's LSE,
//   dV = sum_r P_r^T dO_r,  dP = dO V^T,  Delta = rowsum(dO O),  dS = P (dP - Delta),
//   dQ = scale dS K,  dK = scale sum_r dS_r^T Q_r
// over the rows r of a key head (attn_packed.h).
//
//   terms kernel : Delta and LSE log2 e of each row.
//   grad kernel  : dK and dV, of which a wave owns 32 keys and walks the rows that see them, staged in LDS; and dQ, of which
//                  a wave owns 32 rows and walks the keys they see.
//   join kernel  : adds the parts of tiles that the plan has cut, in their order.  No atomics.
#include <algorithm>
#include <type_traits>

#include "attn_packed.h"

namespace mw {

namespace {

constexpr int kD = MW_PACKED_HEAD_DIM;

// LDS of a row tile's kernels: K and V tiles of BN * KG keys, two stages each; the groups' sums.
template <int D, int NW, int KG, int BN>
struct RowTileLds {
  static constexpr int TE = stage_elems<D, BN * KG, 64 * NW>();
  static constexpr int BYTES = 2 * 2 * TE * 2;
  static_assert(KG == 1 || (KG / 2) * (NW / KG) * (D / 32) * 4096 <= BYTES, "the groups' sums fit the stages");
};

// A sequence's keys and values, staged BS at a time; keys behind the last one repeat it.
template <int D, int BS, int NT>
struct KeyStage {
  const bf16_t *k, *v;
  long long sk, sv;
  int n;
  RowOffsets<D, BS, NT> ro_k, ro_v;
  __device__ __forceinline__ KeyStage(const PackedBwdParams& p, const PackedItem& it, int hk, int tid)
      : k(p.k + (long long)it.k0 * p.sk.t + hk * p.sk.h), v(p.v + (long long)it.k0 * p.sv.t + hk * p.sv.h), sk(p.sk.t),
        sv(p.sv.t), n(it.nk), ro_k(p.sk.t, tid), ro_v(p.sv.t, tid) {}
  __device__ __forceinline__ void stage(int i, bf16_t* Kt, bf16_t* Vt, int tid) const {
    const long long k0 = (long long)i * BS;
    if (k0 + BS <= n) {
      stage_rows_s<D, BS, NT>(Kt, k + k0 * sk, ro_k, tid);
      stage_rows_s<D, BS, NT>(Vt, v + k0 * sv, ro_v, tid);
    } else {
      stage_kv_rows_direct<D, BS, NT>(Kt, Vt, [&](int r) -> RowPair {
        const long long j = min(k0 + r, (long long)n - 1);
        return {k + j * sk, v + j * sv};
      }, tid);
    }
  }
};

// Delta and LSE log2 e of the rows of a tile, for both gradients: rowsum(dO O), which has O's rounding to bf16.  Next to few
// keys' dP - Delta that is not small (cross_dq_kernel): rows of a tile whose first one sees at most 64 keys take sum_j P_j dP_j.
// Bound by reading dO and O: 19200 rows of 12 heads, D = 128, 118 MB in 27 us (31 with a row read by two lanes).
template <int D>
__global__ __launch_bounds__(256) void packed_terms_kernel(PackedBwdParams p, int BM) {
  constexpr int BS = 64, NT = 256, KK = (D + 15) / 16;
  using LD = RowTileLds<D, 4, 1, BS>;
  __shared__ __attribute__((aligned(16))) bf16_t Ks[LD::TE], Vs[LD::TE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int hk;
  PackedItem it;
  if (!work_item(p.list_q, blockIdx.x, p.Hkv, hk, it) || it.beg > 0) return;
  const int G = p.G, R = it.nq * G, n = it.nk, r0 = it.tile * BM;
  const long long terms = ((long long)hk * p.total_q + it.q0) * G;
  auto lse_of = [&](int r) {
    const int t = r / G;
    return p.lse[(long long)(hk * G + (r - t * G)) * p.total_q + it.q0 + t] * 1.4426950408889634f;
  };
  if (it.slot >= 0 || it.beg == it.end || sees(r0, G, it.nq, n, p.L) > 64) {
    // a row is read by eight lanes, or sixteen, a quarter of the tile by a wave
    constexpr int LPR = D == 128 ? 16 : 8, ROWS = 64 / LPR, ITERS = 32 / ROWS, PER = (D / 8 + LPR - 1) / LPR;
    const int part = lane % LPR, first = r0 + wave * (BM / 4) + lane / LPR;
    bf16x8 x[ITERS][PER], y[ITERS][PER];
    float lse2[ITERS];
#pragma unroll
    for (int i = 0; i < ITERS; ++i) {
      if (i * ROWS >= BM / 4) break;
      const int rc = min(first + i * ROWS, R - 1);
      const bf16_t* da = p.d_o + packed_offset(p.sdo, hk, G, it.q0, rc);
      const bf16_t* oa = p.o + packed_offset(p.so, hk, G, it.q0, rc);
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const int col = min(8 * (part + j * LPR), D - 8);  // (D = 72: its last eight columns are one lane's)
        x[i][j] = *reinterpret_cast<const bf16x8*>(da + col);
        y[i][j] = *reinterpret_cast<const bf16x8*>(oa + col);
      }
      lse2[i] = lse_of(rc);
    }
#pragma unroll
    for (int i = 0; i < ITERS; ++i) {
      const int row = first + i * ROWS;
      if (i * ROWS >= BM / 4) break;
      float dot = 0.f;
#pragma unroll
      for (int j = 0; j < PER; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) dot = part + j * LPR < D / 8 ? fmaf((float)x[i][j][e], (float)y[i][j][e], dot) : dot;
#pragma unroll
      for (int m = 1; m < LPR; m <<= 1) dot += __shfl_xor(dot, m);
      if (part == 0 && row < R) {
        p.delta[terms + row] = -dot;
        p.lse2[terms + row] = lse2[i];
      }
    }
    return;
  }
  const int row = r0 + wave * 32 + (lane & 31), rc = min(row, R - 1), hi = sees(rc, G, it.nq, n, p.L);
  const float lse2 = lse_of(rc);
  const bf16_t* qa = p.q + packed_offset(p.sq, hk, G, it.q0, rc) + 8 * (lane >> 5);
  const bf16_t* da = p.d_o + packed_offset(p.sdo, hk, G, it.q0, rc) + 8 * (lane >> 5);
  bf16x8 qf[KK], of[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) {
    if (D % 16 == 0 || 16 * kk + 8 * (lane >> 5) < D) {
      qf[kk] = *reinterpret_cast<const bf16x8*>(qa + 16 * kk);
      of[kk] = *reinterpret_cast<const bf16x8*>(da + 16 * kk);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) qf[kk][j] = of[kk][j] = (__bf16)0.f;
    }
  }
  const FragOffsets<D> fo(lane, 0);
  const KeyStage<D, BS, NT> keys(p, it, hk, tid);
  float sum = 0.f;
  for (int i = it.beg; i < it.end; ++i) {
    if (i > it.beg) __syncthreads();  // (the stage has been read)
    keys.stage(i, Ks, Vs, tid);
    wait_vmem();
    __syncthreads();
#pragma unroll 1
    for (int kq = 0; kq < BS / 32; ++kq) {
      f32x16 s = zero16(), dp = zero16();
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        s = mfma32(fo.row8(Ks, kq * 32, kk), qf[kk], s);
        dp = mfma32(fo.row8(Vs, kq * 32, kk), of[kk], dp);
      }
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const bool in = i * BS + kq * 32 + acc_row(j, lane) < hi;
        sum = fmaf(in ? fast_exp2(fmaf(s[j], p.scale_log2, -lse2)) : 0.f, in ? dp[j] : 0.f, sum);
      }
    }
  }
  sum = sum_halves(sum);
  if (wave * 32 < BM && lane < 32 && row < R) {
    p.delta[terms + row] = -sum;
    p.lse2[terms + row] = lse2;
  }
}

// dK/dV: NWK key waves of 32 keys each (K fragments, dK^T and dV^T in registers) in QG row groups; a step stages
// BM * QG rows, of which a group takes its BM, and the groups' gradients are added through LDS at the end.  The
// first VL V fragments are read from LDS, where they lie as in the registers (D = 128: two waves per SIMD need
// the registers).  Lanes behind the last key repeat it and store nothing.
template <int D, int NWK, int QG, int BM, int VL>
__device__ __forceinline__ void packed_dkdv(const PackedBwdParams& p, const int bid, unsigned char* lds) {
  constexpr int NW = NWK * QG, BN = 32 * NWK, NT = 64 * NW, BS = BM * QG, KK = (D + 15) / 16, DB = D / 32;
  constexpr bool TAIL = D % 32 != 0;
  static_assert(16 * VL <= D, "the V fragments in LDS have no columns past D");
  using LD = KeyTileLds<D, NWK, QG, BM, VL>;
  constexpr int TE = LD::TE, RT = LD::RT;
  bf16_t(*Qs)[TE] = reinterpret_cast<bf16_t(*)[TE]>(lds);
  bf16_t(*Os)[TE] = reinterpret_cast<bf16_t(*)[TE]>(lds + 4 * TE);
  float(*lse_s)[RT] = reinterpret_cast<float(*)[RT]>(lds + 8 * TE);
  float(*dlt_s)[RT] = reinterpret_cast<float(*)[RT]>(lds + 8 * TE + 8 * RT);
  bf16_t* Vs = reinterpret_cast<bf16_t*>(lds + LD::STAGES);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kw = wave % NWK, qg = wave / NWK, gq = qg * BM;
  int hk;
  PackedItem it;
  if (!work_item(p.list_k, bid, p.Hkv, hk, it)) return;
  const int G = p.G, R = it.nq * G, n = it.nk, L = p.L;
  const int k0 = it.tile * BN, key = k0 + kw * 32 + (lane & 31);
  f32x16 dk[DB], dv[DB];
  f32x4 tail[4] = {zero4(), zero4(), zero4(), zero4()};  // (TAIL) dV^T, dK^T of keys 0..15 and 16..31
#pragma unroll
  for (int db = 0; db < DB; ++db) dk[db] = dv[db] = zero16();

  if (it.beg < it.end) {
    // the first row that sees this lane's key; from `all` on every row sees every key of the tile
    const int first = max(0, (int)((unsigned)min(key, n - 1) / (unsigned)L) * L - (n - it.nq)) * G;
    const int all = max(0, (int)((unsigned)(min(k0 + BN, n) - 1) / (unsigned)L) * L - (n - it.nq)) * G;
    bf16x8 kf[KK], vf[KK];
    const bf16_t* vfrag = Vs + (kw * VL * 64 + lane) * 8;
    for (int f = wave; f < NWK * VL; f += NW) {  // V fragments in LDS, one a wave and round, as they lie in registers
      const int w = f / (VL > 0 ? VL : 1), kk = f - w * VL;
      const long long kr = it.k0 + min(k0 + w * 32 + (lane & 31), n - 1);
      dma_lds_16(p.v + hk * p.sv.h + kr * p.sv.t + 16 * kk + 8 * (lane >> 5), lds_addr(Vs) + f * 1024);
    }
    {
      const long long kr = it.k0 + min(key, n - 1);
      const bf16_t* ka = p.k + hk * p.sk.h + kr * p.sk.t + 8 * (lane >> 5);
      const bf16_t* va = p.v + hk * p.sv.h + kr * p.sv.t + 8 * (lane >> 5);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        if (D % 16 == 0 || 16 * kk + 8 * (lane >> 5) < D) {
          kf[kk] = *reinterpret_cast<const bf16x8*>(ka + 16 * kk);
          if (kk >= VL) vf[kk] = *reinterpret_cast<const bf16x8*>(va + 16 * kk);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) kf[kk][j] = vf[kk][j] = (__bf16)0.f;
        }
      }
    }
    const FragOffsets<D> fo(lane, gq * D);
    const Tail72 ft(lane, gq * D);
    // offsets of one query head's rows, held in registers where there are any to spare
    constexpr bool HELD = D != 128 || QG == 1;
    const RowOffsets<D, HELD ? BS : 32, NT> ro_q(p.sq.t, tid), ro_o(p.sdo.t, tid);
    const bf16_t* q0p = p.q + (long long)hk * G * p.sq.h + (long long)it.q0 * p.sq.t;
    const bf16_t* o0p = p.d_o + (long long)hk * G * p.sdo.h + (long long)it.q0 * p.sdo.t;
    const long long row_base = ((long long)hk * p.total_q + it.q0) * G;
    const float* lse2 = p.lse2 + row_base;
    const float* dlt = p.delta + row_base;
    const int beg = it.beg * BS, end = min(R, it.end * BS);
    auto stage = [&](int r0, int buf) {  // rows behind the sequence's last one repeat it
      bool done = false;
      if constexpr (HELD) {
        if (r0 + BS <= R && G == 1) {
          stage_rows_s<D, BS, NT>(Qs[buf], uniform(q0p + r0 * p.sq.t), ro_q, tid);
          stage_rows_s<D, BS, NT>(Os[buf], uniform(o0p + r0 * p.sdo.t), ro_o, tid);
          done = true;
        }
      }
      if (done) {
      } else if (r0 + BS <= R && p.near) {
        stage_group<D, BS, NT>(Qs[buf], q0p, p.sq, r0, G, p.magic, tid);
        stage_group<D, BS, NT>(Os[buf], o0p, p.sdo, r0, G, p.magic, tid);
      } else {
        stage_rows_direct<D, BS, NT>(Qs[buf], [&](int r) { return p.q + packed_offset(p.sq, hk, G, it.q0, min(r0 + r, R - 1)); },
                                     tid);
        stage_rows_direct<D, BS, NT>(Os[buf],
                                     [&](int r) { return p.d_o + packed_offset(p.sdo, hk, G, it.q0, min(r0 + r, R - 1)); }, tid);
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
    constexpr bool PRIO = !TAIL;  // matrix phases go first
    auto step = [&](auto masked, int r0, int buf) {
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
            if constexpr (decltype(masked)::value) pv = ((r0 + rr + j >= first) & (r0 + rr + j < R)) ? pv : 0.f;
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
    stage(beg, 0);
    wait_vmem();
    __syncthreads();
    int buf = 0, r0 = beg;
    auto run = [&](auto masked, int stop) {
      for (; r0 < stop; r0 += BS) {
        if (r0 + BS < end) stage(r0 + BS, buf ^ 1);
        if (k0 + kw * 32 < n) step(masked, r0, buf);
        if constexpr (PRIO) __builtin_amdgcn_s_setprio(0);
        wait_vmem();
        __syncthreads();
        buf ^= 1;
      }
    };
    run(std::true_type{}, min(end, (all + BS - 1) / BS * BS));
    run(std::false_type{}, min(end, R / BS * BS));
    run(std::true_type{}, end);
  }

  if constexpr (QG > 1) {
    float* m = reinterpret_cast<float*>(lds);
    add_groups<QG, NWK>(dv, qg, kw, lane, m);
    add_groups<QG, NWK>(dk, qg, kw, lane, m);
    if constexpr (TAIL) {
      f32x16 rest[1];
#pragma unroll
      for (int i = 0; i < 16; ++i) rest[0][i] = tail[i / 4][i % 4];
      add_groups<QG, NWK>(rest, qg, kw, lane, m);
#pragma unroll
      for (int i = 0; i < 16; ++i) tail[i / 4][i % 4] = rest[0][i];
    }
    if (qg > 0) return;  // no barrier follows
  }
  if (it.slot >= 0) {
    constexpr int HALF = BN * D;
    float* pk = p.part_k + ((long long)it.slot * p.Hkv + hk) * 2 * HALF;  // dK; dV behind it
    if constexpr (TAIL) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int kr = kw * 32 + 16 * e + (lane & 15);
        if (lane < 32 && k0 + kr < n) {
          float* x = pk + kr * D + 64 + 4 * (lane >> 4);
          *reinterpret_cast<f32x4*>(x) = tail[2 + e];
          *reinterpret_cast<f32x4*>(x + HALF) = tail[e];
        }
      }
    }
    if (key >= n) return;
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
        float* x = pk + (key - k0) * D + db * 32 + 8 * g + 4 * (lane >> 5);
        *reinterpret_cast<f32x4*>(x) = wk;
        *reinterpret_cast<f32x4*>(x + HALF) = wv;
      }
    return;
  }
  if constexpr (TAIL) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int kr = k0 + kw * 32 + 16 * e + (lane & 15), col = 64 + 4 * (lane >> 4);
      if (lane < 32 && kr < n) {
        bf16x4 wk, wv;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          wk[j] = to_bf16(tail[2 + e][j] * p.scale);
          wv[j] = to_bf16(tail[e][j]);
        }
        *reinterpret_cast<bf16x4*>(p.dk + hk * p.sdk.h + (long long)(it.k0 + kr) * p.sdk.t + col) = wk;
        *reinterpret_cast<bf16x4*>(p.dv + hk * p.sdv.h + (long long)(it.k0 + kr) * p.sdv.t + col) = wv;
      }
    }
  }
  if (key >= n) return;
  bf16_t* dkr = p.dk + hk * p.sdk.h + (long long)(it.k0 + key) * p.sdk.t;
  bf16_t* dvr = p.dv + hk * p.sdv.h + (long long)(it.k0 + key) * p.sdv.t;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      bf16x4 wk, wv;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        wk[j] = to_bf16(dk[db][4 * g + j] * p.scale);
        wv[j] = to_bf16(dv[db][4 * g + j]);
      }
      const int col = db * 32 + 8 * g + 4 * (lane >> 5);
      *reinterpret_cast<bf16x4*>(dkr + col) = wk;
      *reinterpret_cast<bf16x4*>(dvr + col) = wv;
    }
}

// dQ: NW waves in KG key groups of NW / KG waves of 32 rows each (Q and dO fragments, dQ^T in registers); a step stages
// BN * KG keys, of which a group takes its BN, and the groups' dQ are added through LDS at the end.
template <int D, int NW, int KG, int BN>
__device__ __forceinline__ void packed_dq(const PackedBwdParams& p, const int bid, unsigned char* lds) {
  constexpr int NWR = NW / KG, BM = 32 * NWR, BS = BN * KG, NT = 64 * NW, KK = (D + 15) / 16, DB = D / 32;
  constexpr bool TAIL = D % 32 != 0;
  using LD = RowTileLds<D, NW, KG, BN>;
  constexpr int TE = LD::TE;
  bf16_t(*Ks)[TE] = reinterpret_cast<bf16_t(*)[TE]>(lds);
  bf16_t(*Vs)[TE] = reinterpret_cast<bf16_t(*)[TE]>(lds + 4 * TE);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % NWR, kg = wave / NWR;
  int hk;
  PackedItem it;
  if (!work_item(p.list_q, bid, p.Hkv, hk, it)) return;
  const int G = p.G, R = it.nq * G, n = it.nk, r0 = it.tile * BM;
  const int row = r0 + rw * 32 + (lane & 31), rc = min(row, R - 1);
  bf16x8 qf[KK], of[KK];
  {
    const bf16_t* qa = p.q + packed_offset(p.sq, hk, G, it.q0, rc) + 8 * (lane >> 5);
    const bf16_t* da = p.d_o + packed_offset(p.sdo, hk, G, it.q0, rc) + 8 * (lane >> 5);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      if (D % 16 == 0 || 16 * kk + 8 * (lane >> 5) < D) {
        of[kk] = *reinterpret_cast<const bf16x8*>(da + 16 * kk);
        qf[kk] = *reinterpret_cast<const bf16x8*>(qa + 16 * kk);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) qf[kk][j] = of[kk][j] = (__bf16)0.f;
      }
    }
  }
  const long long at = ((long long)hk * p.total_q + it.q0) * G + rc;
  const float ndlt = p.delta[at], lse2 = p.lse2[at], c = p.scale_log2;
  const int hi = sees(rc, G, it.nq, n, p.L), hi_all = sees(r0, G, it.nq, n, p.L);
  f32x16 dq[DB];
  f32x4 tail[2] = {zero4(), zero4()};
#pragma unroll
  for (int db = 0; db < DB; ++db) dq[db] = zero16();
  const FragOffsets<D> fo(lane, 0);
  const Tail72 ft(lane, 0);
  const KeyStage<D, BS, NT> keys(p, it, hk, tid);
  if (it.beg < it.end) keys.stage(it.beg, Ks[0], Vs[0], tid);
  wait_vmem();
  __syncthreads();
  if (it.beg < it.end) {
    f32x16 nd;
#pragma unroll
    for (int i = 0; i < 16; ++i) nd[i] = ndlt;
    auto step = [&](auto masked, int k0, int buf) {
#pragma unroll
      for (int kq = 0; kq < BN / 32; ++kq) {
        f32x16 s = zero16(), dp = nd;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          s = mfma32(fo.row8(Ks[buf], kg * BN + kq * 32, kk), qf[kk], s);
          dp = mfma32(fo.row8(Vs[buf], kg * BN + kq * 32, kk), of[kk], dp);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float pv = fast_exp2(fmaf(s[i], c, -lse2));
          if constexpr (decltype(masked)::value) pv = k0 + kg * BN + kq * 32 + acc_row(i, lane) < hi ? pv : 0.f;
          dp[i] *= pv;
        }
        bf16x8 h[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          h[t] = pack8(dp, t);
#pragma unroll
          for (int db = 0; db < DB; ++db) dq[db] = mfma32(fo.tr8(Ks[buf], kg * BN + kq * 32, t, db), h[t], dq[db]);
        }
        if constexpr (TAIL) {
          const bf16x8 x = ft.read(Ks[buf], kg * BN + kq * 32);
          tail_operands(h[0], h[1]);
#pragma unroll
          for (int e = 0; e < 2; ++e) tail[e] = mfma16(x, h[e], tail[e]);
        }
      }
    };
    int buf = 0, i = it.beg;
    auto run = [&](auto masked, int stop) {
      for (; i < stop; ++i) {
        if (i + 1 < it.end) keys.stage(i + 1, Ks[buf ^ 1], Vs[buf ^ 1], tid);
        step(masked, i * BS, buf);
        wait_vmem();
        __syncthreads();
        buf ^= 1;
      }
    };
    run(std::false_type{}, min(hi_all / BS, it.end));
    run(std::true_type{}, it.end);
  }
  if constexpr (KG > 1) {
    float* m = reinterpret_cast<float*>(lds);
    add_groups<KG, NWR>(dq, kg, rw, lane, m);
    if constexpr (TAIL) {
      f32x16 rest[1] = {zero16()};
#pragma unroll
      for (int i = 0; i < 8; ++i) rest[0][i] = tail[i / 4][i % 4];
      add_groups<KG, NWR>(rest, kg, rw, lane, m);
#pragma unroll
      for (int i = 0; i < 8; ++i) tail[i / 4][i % 4] = rest[0][i];
    }
    __syncthreads();     // (the stages are written again below)
    if (kg > 0) return;  // no barrier follows
  }
  if (it.slot >= 0) {  // fp32 dQ of this range of the keys
    float* part = p.part_q + (((long long)it.slot * p.Hkv + hk) * BM + rw * 32) * D;
    if constexpr (TAIL) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 16 * e + (lane & 15);
        if (lane < 32 && r0 + rw * 32 + r < R) *reinterpret_cast<f32x4*>(part + r * D + 64 + 4 * (lane >> 4)) = tail[e];
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
        *reinterpret_cast<f32x4*>(part + (lane & 31) * D + db * 32 + 8 * g + 4 * (lane >> 5)) = w;
      }
    return;
  }
  // (every wave has passed the last barrier: a half stage holds the rows of BS / 32 waves)
  static_assert(NWR <= 2 * (BS / 32), "one stage holds the rows of every wave");
  const int half = rw / (BS / 32);
  store_rows<D>(dq, tail, (half ? Vs : Ks)[0] + (rw - half * (BS / 32)) * 32 * D, min(32, R - r0 - rw * 32), lane, p.scale,
                [&](int r) { return p.dq + packed_offset(p.sdq, hk, G, it.q0, r0 + rw * 32 + r); });
}

// Sums of the parts of cut tiles, in order: dK and dV, then dQ.  One thread for four columns of a row.  5 us where little is
// cut, 7 for the text batch below.
template <int D, int BM, int BN>
__global__ __launch_bounds__(256) void packed_bwd_join_kernel(PackedBwdParams p) {
  constexpr int TPR = D / 4, PER_K = join_blocks(BN, D), PER_Q = join_blocks(BM, D);
  const int n_kv = p.list_k[1] * p.Hkv * PER_K, n = n_kv + p.list_q[1] * p.Hkv * PER_Q;
  for (int id = blockIdx.x; id < n; id += gridDim.x) {
    if (id < n_kv) {
      const int job = id / PER_K, j = job / p.Hkv, hk = job - j * p.Hkv;
      const PackedJoin it = p.joins_k[j];
      const int x = (id - job * PER_K) * 256 + threadIdx.x, kr = x / TPR, col = (x - kr * TPR) * 4;
      const int key = it.tile * BN + kr;
      if (kr >= BN || key >= it.nk) continue;
      f32x4 k = zero4(), v = zero4();
#pragma unroll 4
      for (int s = 0; s < it.parts; ++s) {
        const float* y = p.part_k + ((long long)(it.first + s) * p.Hkv + hk) * 2 * BN * D + kr * D + col;
        k += *reinterpret_cast<const f32x4*>(y);
        v += *reinterpret_cast<const f32x4*>(y + BN * D);
      }
      bf16x4 wk, wv;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        wk[c] = to_bf16(k[c] * p.scale);
        wv[c] = to_bf16(v[c]);
      }
      *reinterpret_cast<bf16x4*>(p.dk + hk * p.sdk.h + (long long)(it.k0 + key) * p.sdk.t + col) = wk;
      *reinterpret_cast<bf16x4*>(p.dv + hk * p.sdv.h + (long long)(it.k0 + key) * p.sdv.t + col) = wv;
      continue;
    }
    const int b = id - n_kv, job = b / PER_Q, j = job / p.Hkv, hk = job - j * p.Hkv;
    const PackedJoin it = p.joins_q[j];
    const int x = (b - job * PER_Q) * 256 + threadIdx.x, rt = x / TPR, col = (x - rt * TPR) * 4;
    const int row = it.tile * BM + rt;
    if (rt >= BM || row >= it.nq * p.G) continue;
    f32x4 q = zero4();
#pragma unroll 4
    for (int s = 0; s < it.parts; ++s)
      q += *reinterpret_cast<const f32x4*>(p.part_q + (((long long)(it.first + s) * p.Hkv + hk) * BM + rt) * D + col);
    bf16x4 w;
#pragma unroll
    for (int c = 0; c < 4; ++c) w[c] = to_bf16(q[c] * p.scale);
    *reinterpret_cast<bf16x4*>(p.dq + packed_offset(p.sdq, hk, p.G, it.q0, row) + col) = w;
  }
}

}  // namespace

// A tile's configuration: rows (dQ) and keys (dK, dV) of 128 in four waves, or of 64 in two groups of two.
template <int D, PackedTile T>
struct Config {
  static constexpr bool WIDE = T == PackedTile::wide;
  static constexpr int TILE = WIDE ? 128 : 64, GROUPS = WIDE ? 1 : 2;
  static constexpr int VL = D == 128 ? (WIDE ? 6 : 7) : 0;
  static constexpr int BM = packed_dkv_step(D, T) / GROUPS;
  using Rows = RowTileLds<D, 4, GROUPS, 64 / GROUPS>;
  using Keys = KeyTileLds<D, TILE / 32, GROUPS, BM, VL>;
};

// Both in one grid: the longer dK/dV items first, so that dQ's fill the places that the last of them leave (the text batch
// below 253 us, one after the other, with Delta formed by dQ's, 283; 512 tokens of 8 heads, D = 128, forward and backward 44
// -> 36).
//
// Bound by the matrix products: 14 D a pair for the 10 that the gradients need, because S and dP are formed for both, so that
// neither has to add to memory that others add to.  Clips of 600 to 9600 tokens, 19200 in all, 12 heads, D = 128: 1600 us,
// 1008 TF executed, matrix units 58% busy with two waves a SIMD at 1.65 GHz, which is what the power limit leaves; the text
// batch, 8192 tokens, 24 heads on 8, D = 64, 1005 TF; 4717 tokens of 16 heads, D = 72, 138 us, 884 TF.
template <int D, PackedTile TQ, PackedTile TK>
__global__ __launch_bounds__(256, packed_bwd_per_cu(D, TQ, TK)) void packed_grad_kernel(PackedBwdParams p, int n_keys) {
  using Q = Config<D, TQ>;
  using K = Config<D, TK>;
  constexpr int BYTES = Q::Rows::BYTES > K::Keys::BYTES ? Q::Rows::BYTES : K::Keys::BYTES;
  __shared__ __attribute__((aligned(16))) unsigned char lds[BYTES];
  if ((int)blockIdx.x < n_keys) {
    packed_dkdv<D, K::TILE / 32, K::GROUPS, K::BM, K::VL>(p, blockIdx.x, lds);
  } else {
    packed_dq<D, 4, Q::GROUPS, 64 / Q::GROUPS>(p, blockIdx.x - n_keys, lds);
  }
}

namespace {

template <PackedTile TQ, PackedTile TK>
hipError_t launch_grad(const PackedBwdParams& p, const PackedShape& s, hipStream_t stream) {
  if (s.dq.tile != Config<kD, TQ>::TILE || s.dq.step != 64 || s.dkv.tile != Config<kD, TK>::TILE ||
      s.dkv.step != packed_dkv_step(kD, TK))
    return hipErrorInvalidValue;
  const long long n_rows = (long long)s.dq.max_items * s.Hkv, n_keys = (long long)s.dkv.max_items * s.Hkv;
  if (n_rows + n_keys > 0x7fffffffLL) return hipErrorInvalidValue;
  hipLaunchKernelGGL((packed_terms_kernel<kD>), dim3((unsigned)n_rows), dim3(256), 0, stream, p, s.dq.tile);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((packed_grad_kernel<kD, TQ, TK>), dim3((unsigned)(n_keys + n_rows)), dim3(256), 0, stream, p, (int)n_keys);
  return hipGetLastError();
}

template <int BM, int BN>
hipError_t launch_join(const PackedBwdParams& p, const PackedShape& s, hipStream_t stream) {
  const long long n =
      (long long)s.Hkv * (s.dkv.max_joins * join_blocks(BN, kD) + s.dq.max_joins * join_blocks(BM, kD));
  if (n == 0) return hipSuccess;
  hipLaunchKernelGGL((packed_bwd_join_kernel<kD, BM, BN>), dim3((unsigned)std::min(n, (long long)kJoinGrid)), dim3(256), 0,
                     stream, p);
  return hipGetLastError();
}

}  // namespace

#define MW_CAT_(a, b) a##b
#define MW_CAT(a, b) MW_CAT_(a, b)
// 128 keys in four waves: with two row groups of eight waves, whose barriers hold them all in step, the 1B clips take 1993 for
// 1920 us, forward and backward, the text batch (D = 64) 399 for 381.
hipError_t MW_CAT(launch_packed_bwd_, MW_PACKED_HEAD_DIM)(const PackedBwdParams& p, const PackedShape& s, hipStream_t stream) {
  const bool wide_q = s.dq.kind == PackedTile::wide, wide_k = s.dkv.kind == PackedTile::wide;
  constexpr PackedTile W = PackedTile::wide, P = PackedTile::pairs;
  const hipError_t e = wide_q ? (wide_k ? launch_grad<W, W>(p, s, stream) : launch_grad<W, P>(p, s, stream))
                              : (wide_k ? launch_grad<P, W>(p, s, stream) : launch_grad<P, P>(p, s, stream));
  if (e != hipSuccess) return e;
  if (wide_q) return wide_k ? launch_join<128, 128>(p, s, stream) : launch_join<128, 64>(p, s, stream);
  return wide_k ? launch_join<64, 128>(p, s, stream) : launch_join<64, 64>(p, s, stream);
}

}  // namespace mw
