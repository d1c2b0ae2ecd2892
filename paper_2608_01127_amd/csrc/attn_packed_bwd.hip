// Backward of the packed attention (gfx950): with P recomputed from Q, K and the forward's LSE,
//   dV = sum_r P_r^T dO_r,  dP = dO V^T,  Delta = rowsum(dO O),  dS = P (dP - Delta),
//   dQ = scale dS K,  dK = scale sum_r dS_r^T Q_r
// over the rows r of a key head (attn_packed.hip).
//
//   dQ kernel    : a wave owns 32 rows and walks the keys they see; it forms Delta (and LSE log2 e) for the other one.
//   dK/dV kernel : a wave owns 32 keys and walks the rows that see them, staged in LDS.
//   join kernel  : adds the parts of tiles that the plan has cut, in their order.  No atomics.
#include <algorithm>
#include <type_traits>

#include "attn_packed.h"

namespace mw {

namespace {

constexpr int kD = MW_PACKED_HEAD_DIM;

// dK/dV: NWK key waves of 32 keys each (K fragments, dK^T and dV^T in registers) in QG row groups; a step stages
// BM * QG rows, of which a group takes its BM, and the groups' gradients are added through LDS at the end.  The
// first VL V fragments are read from LDS, where they lie as in the registers (D = 128: two waves per SIMD need
// the registers).  Lanes behind the last key repeat it and store nothing.
//
// Bound by the matrix products, 8 D a pair of the 14 D of the backward (S and dP are formed in both kernels, so that neither
// has to add to memory that others add to), with two waves a SIMD: clips of 600 to 9600 tokens, 19200 in all, 12 heads, D =
// 128, 890 to 970 us, 945 TF executed, matrix units 56% busy at 1.62 GHz, which is what the power limit leaves.  D = 64 (24
// heads on 8, 8192 tokens) 169 us, 860 TF: 1072 workgroups over 768 places.
template <int D, int NWK, int QG, int BM, int VL, int WPS>
__global__ __launch_bounds__(64 * NWK * QG, WPS) void packed_dkdv_kernel(PackedBwdParams p) {
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
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kw = wave % NWK, qg = wave / NWK, gq = qg * BM;
  int hk;
  PackedItem it;
  if (!work_item(p.list_k, p.Hkv, hk, it)) return;
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
// Bound by the matrix products, 6 D a pair, as above: the clips 635 to 690 us, 1011 TF executed, matrix units 60% busy at
// 1.62 GHz; the 8192 tokens of D = 64 115 us, 944 TF; 4717 tokens of 16 heads, D = 72, 65 us, 790 TF.
template <int D, int NW, int KG, int BN, int WPS>
__global__ __launch_bounds__(64 * NW, WPS) void packed_dq_kernel(PackedBwdParams p) {
  constexpr int NWR = NW / KG, BM = 32 * NWR, BS = BN * KG, NT = 64 * NW, KK = (D + 15) / 16, DB = D / 32;
  constexpr bool TAIL = D % 32 != 0;
  constexpr int TE = stage_elems<D, BS, NT>();
  __shared__ __attribute__((aligned(16))) bf16_t lds[2][2][TE];
  bf16_t(*Ks)[TE] = lds[0];
  bf16_t(*Vs)[TE] = lds[1];
  static_assert(KG == 1 || (KG / 2) * NWR * DB * 4096 <= (int)sizeof(lds), "the groups' sums fit the stages");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % NWR, kg = wave / NWR;
  int hk;
  PackedItem it;
  if (!work_item(p.list_q, p.Hkv, hk, it)) return;
  const int G = p.G, R = it.nq * G, n = it.nk, r0 = it.tile * BM;
  const int row = r0 + rw * 32 + (lane & 31), rc = min(row, R - 1);
  // This row's Q, dO and O, asked for before anything that waits: their latencies then pass together.
  bf16x8 qf[KK], of[KK], y[KK];
  {
    const bf16_t* qa = p.q + packed_offset(p.sq, hk, G, it.q0, rc) + 8 * (lane >> 5);
    const bf16_t* da = p.d_o + packed_offset(p.sdo, hk, G, it.q0, rc) + 8 * (lane >> 5);
    const bf16_t* oa = p.o + packed_offset(p.so, hk, G, it.q0, rc) + 8 * (lane >> 5);
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
  const float lse = p.lse[(long long)(hk * G + (rc - row_t * G)) * p.total_q + it.q0 + row_t];
  const int hi = sees(rc, G, it.nq, n, p.L), hi_all = sees(r0, G, it.nq, n, p.L);
  f32x16 dq[DB];
  f32x4 tail[2] = {zero4(), zero4()};
#pragma unroll
  for (int db = 0; db < DB; ++db) dq[db] = zero16();
  const bf16_t* k0p = p.k + (long long)it.k0 * p.sk.t + hk * p.sk.h;
  const bf16_t* v0p = p.v + (long long)it.k0 * p.sv.t + hk * p.sv.h;
  const FragOffsets<D> fo(lane, 0);
  const Tail72 ft(lane, 0);
  const RowOffsets<D, BS, NT> ro_k(p.sk.t, tid), ro_v(p.sv.t, tid);
  auto stage = [&](int i, int buf) {  // keys behind the sequence's last one repeat it
    const long long k0 = (long long)i * BS;
    if (k0 + BS <= n) {
      stage_rows_s<D, BS, NT>(Ks[buf], k0p + k0 * p.sk.t, ro_k, tid);
      stage_rows_s<D, BS, NT>(Vs[buf], v0p + k0 * p.sv.t, ro_v, tid);
    } else {
      stage_kv_rows_direct<D, BS, NT>(Ks[buf], Vs[buf], [&](int r) -> RowPair {
        const long long j = min(k0 + r, (long long)n - 1);
        return {k0p + j * p.sk.t, v0p + j * p.sv.t};
      }, tid);
    }
  };
  if (it.beg < it.end) stage(it.beg, 0);
  float dot = 0.f;
#pragma unroll
  for (int kk = 0; kk < KK; ++kk)
#pragma unroll
    for (int j = 0; j < 8; ++j) dot = fmaf((float)of[kk][j], (float)y[kk][j], dot);
  float ndlt = -sum_halves(dot);
  const float c = p.scale_log2, lse2 = lse * 1.4426950408889634f;
  wait_vmem();
  __syncthreads();
  // Rows of few keys: Delta = sum_j P_j dP_j of the probabilities at hand.  rowsum(dO O) has O's rounding to bf16, which
  // next to few keys' dP - Delta is not small (cross_dq_kernel); a tile whose first row sees at most a step of
  // keys is walked twice.
  if (hi_all <= 64 && it.slot < 0 && it.beg < it.end) {
    float sum = 0.f;
    for (int i = it.beg; i < it.end; ++i) {
      if (i > it.beg) {
        stage(i, 0);
        wait_vmem();
        __syncthreads();
      }
#pragma unroll 1
      for (int kq = 0; kq < BS / 32; ++kq) {  // (each group forms the whole sum)
        f32x16 s = zero16(), dp = zero16();
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          s = mfma32(fo.row8(Ks[0], kq * 32, kk), qf[kk], s);
          dp = mfma32(fo.row8(Vs[0], kq * 32, kk), of[kk], dp);
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const bool in = i * BS + kq * 32 + acc_row(j, lane) < hi;
          sum = fmaf(in ? fast_exp2(fmaf(s[j], c, -lse2)) : 0.f, in ? dp[j] : 0.f, sum);
        }
      }
      __syncthreads();  // (the stage is written again)
    }
    ndlt = -sum_halves(sum);
    if (it.end - it.beg > 1) {
      stage(it.beg, 0);
      wait_vmem();
      __syncthreads();
    }
  }
  if (it.beg == 0 && kg == 0 && lane < 32 && row < R) {
    const long long at = ((long long)hk * p.total_q + it.q0) * G + row;
    p.delta[at] = ndlt;
    p.lse2[at] = lse2;
  }
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
        if (i + 1 < it.end) stage(i + 1, buf ^ 1);
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
    float* m = reinterpret_cast<float*>(&lds[0][0][0]);
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
// cut; 9 for the 8192 tokens above, whose parts (16 MB) it reads at 1.9 TB/s.
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

namespace {

template <int NW, int KG, int WPS>
hipError_t launch_dq(const PackedBwdParams& p, const PackedShape& s, hipStream_t stream) {
  constexpr int BN = 64 / KG;
  if (s.dq.tile != 32 * NW / KG || s.dq.step != 64) return hipErrorInvalidValue;
  const long long grid = (long long)s.dq.max_items * s.Hkv;
  if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
  hipLaunchKernelGGL((packed_dq_kernel<kD, NW, KG, BN, WPS>), dim3((unsigned)grid), dim3(64 * NW), 0, stream, p);
  return hipGetLastError();
}

template <int NWK, int QG, int BM, int VL, int WPS>
hipError_t launch_dkdv(const PackedBwdParams& p, const PackedShape& s, hipStream_t stream) {
  if (s.dkv.tile != 32 * NWK || s.dkv.step != BM * QG) return hipErrorInvalidValue;
  const long long grid = (long long)s.dkv.max_items * s.Hkv;
  if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
  hipLaunchKernelGGL((packed_dkdv_kernel<kD, NWK, QG, BM, VL, WPS>), dim3((unsigned)grid), dim3(64 * NWK * QG), 0, stream, p);
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
  constexpr PackedPass DQ = PackedPass::dq, KV = PackedPass::dkdv;
  hipError_t e = wide_q ? launch_dq<4, 1, packed_per_cu(DQ, kD, W)>(p, s, stream)
                        : launch_dq<4, 2, packed_per_cu(DQ, kD, P)>(p, s, stream);
  if (e != hipSuccess) return e;
  if (wide_k) {
    e = launch_dkdv<4, 1, packed_dkv_step(kD, W), kD == 128 ? 6 : 0, packed_per_cu(KV, kD, W)>(p, s, stream);
  } else {
    e = launch_dkdv<2, 2, 32, kD == 128 ? 7 : 0, packed_per_cu(KV, kD, P)>(p, s, stream);
  }
  if (e != hipSuccess) return e;
  if (wide_q) return wide_k ? launch_join<128, 128>(p, s, stream) : launch_join<128, 64>(p, s, stream);
  return wide_k ? launch_join<64, 128>(p, s, stream) : launch_join<64, 64>(p, s, stream);
}

}  // namespace mw
