// Forward of the packed attention (gfx950); the method stands in attn_packed.h.
#include <algorithm>
#include <type_traits>

#include "attn_packed.h"

namespace mw {

namespace {

constexpr int kD = MW_PACKED_HEAD_DIM;

// 32 rows' results of a wave, row `row` of the tile in this lane: partial ones in place `slot`, or O and LSE.
template <int D, int BM, int BN>
__device__ __forceinline__ void finish_packed(const PackedParams& p, const RowBlock<D, BN>& rb, const PackedItem& it, int hk,
                                              int r_tile, bf16_t* x, int lane) {
  constexpr int DB = D / 32;
  constexpr bool TAIL = D % 32 != 0;
  const int G = p.G, R = it.nq * G, r0 = it.tile * BM + r_tile, row = r0 + (lane & 31);
  const float l = sum_halves(rb.l);
  if (it.slot >= 0) {
    const long long at = ((long long)it.slot * p.Hkv + hk) * BM + r_tile;
    if constexpr (TAIL) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 16 * e + (lane & 15);
        if (lane < 32 && r0 + r < R) *reinterpret_cast<f32x4*>(p.part + (at + r) * D + 64 + 4 * (lane >> 4)) = rb.ot[e];
      }
    }
    if (row >= R) return;
    float* po = p.part + (at + (lane & 31)) * D;
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
      float* ml = p.part + (long long)p.max_slots * p.Hkv * BM * D + 2 * (at + lane);
      ml[0] = rb.m;
      ml[1] = l;
    }
    return;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;  // a row that sees no key gives zeros
  store_rows<D>(rb.o, rb.ot, x, min(32, R - r0), lane, inv,
                [&](int r) { return p.o + packed_offset(p.so, hk, G, it.q0, r0 + r); });
  if (lane < 32 && row < R) {
    const int t = row / G;
    p.lse[(long long)(hk * G + (row - t * G)) * p.total_q + it.q0 + t] =
        l == 0.f ? -INFINITY : (rb.m + __log2f(l)) * 0.69314718055994530942f;
  }
}

}  // namespace

// NW waves in KG key groups of NW / KG waves of 32 rows each; a step stages KG * BN keys, of which a group takes its BN.
// S^T = K Q^T, so that a lane holds scores of one row; the softmax is taken in one pass, its maximum raised only where it
// has to be.  O stays in registers.
//
// Many rows are bound by matrix units and softmax side by side: seven prompts, 19200 tokens in all, 16 heads on 4, D = 128,
// 404 us, 1001 TF executed, matrix units 57% and vector work 55% busy at 1.68 GHz; D = 64 (8192 tokens, 24 heads on 8) 89
// us, vector work 82%: its exponentials are as many as at D = 128, for half the products.  D = 72 (4717 tokens, 16 heads)
// 48 us: products of 80 columns, and LDS conflicts in 31% of the LDS-active cycles.  Few rows are bound by reading keys and
// values: one token of 8 sequences, 147 MB, 26 us and the join, 34 the call, 4.3 TB/s.
template <int D, int NW, int BN, int KG, int WPS>
__global__ __launch_bounds__(64 * NW, WPS) void packed_fwd_kernel(PackedParams p) {
  constexpr int NWR = NW / KG, BM = 32 * NWR, NT = 64 * NW, BK = BN * KG;
  using RB = RowBlock<D, BN>;
  constexpr int KK = RB::KK;
  constexpr int TE = stage_elems<D, BK, NT>();
  __shared__ __attribute__((aligned(16))) bf16_t lds[2][2][TE];  // K, V x two stages
  static_assert(RB::template merge_floats<KG, NWR>() * 4 <= (int)sizeof(lds), "the merge fits the stages");
  bf16_t(*Ks)[TE] = lds[0];
  bf16_t(*Vs)[TE] = lds[1];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % NWR, kg = wave / NWR;
  int hk;
  PackedItem it;
  if (!work_item(p.list, blockIdx.x, p.Hkv, hk, it)) return;
  const int G = p.G, R = it.nq * G, r0 = it.tile * BM;

  // this lane's row and its Q fragments; rows behind the last and columns past D are zeros
  const int row = r0 + rw * 32 + (lane & 31);
  bf16x8 qf[KK];
  {
    const bf16_t* qp = p.q + packed_offset(p.sq, hk, G, it.q0, min(row, R - 1)) + 8 * (lane >> 5);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      if (row < R && (D % 16 == 0 || 16 * kk + 8 * (lane >> 5) < D)) {
        qf[kk] = *reinterpret_cast<const bf16x8*>(qp + 16 * kk);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) qf[kk][j] = (__bf16)0.f;
      }
    }
  }
  const int hi = sees(min(row, R - 1), G, it.nq, it.nk, p.L);
  const int n_full = sees(r0, G, it.nq, it.nk, p.L) / BK;  // steps that every row sees whole

  const bf16_t* k0p = p.k + (long long)it.k0 * p.sk.t + hk * p.sk.h;
  const bf16_t* v0p = p.v + (long long)it.k0 * p.sv.t + hk * p.sv.h;
  const RowOffsets<D, BK, NT> ro_k(p.sk.t, tid), ro_v(p.sv.t, tid);
  auto stage = [&](int step, int buf) {  // keys behind the sequence's last one repeat it
    const long long k0 = (long long)step * BK;
    if (k0 + BK <= it.nk) {
      stage_rows_s<D, BK, NT>(Ks[buf], k0p + k0 * p.sk.t, ro_k, tid);
      stage_rows_s<D, BK, NT>(Vs[buf], v0p + k0 * p.sv.t, ro_v, tid);
    } else {
      stage_kv_rows_direct<D, BK, NT>(Ks[buf], Vs[buf], [&](int r) -> RowPair {
        const long long j = min(k0 + r, (long long)it.nk - 1);
        return {k0p + j * p.sk.t, v0p + j * p.sv.t};
      }, tid);
    }
  };
  const FragOffsets<D> fo(lane, kg * BN * D);
  const Tail72 ft(lane, kg * BN * D);
  RB rb;
  rb.init();
  int buf = 0, i = it.beg;
  if (it.beg < it.end) {
    stage(it.beg, 0);
    wait_vmem();
    lds_barrier();
    auto run = [&](auto masked, int stop) {
      for (; i < stop; ++i) {
        if (i + 1 < it.end) stage(i + 1, buf ^ 1);
        rb.template step<decltype(masked)::value, false>([] {}, Ks[buf], Vs[buf], fo, ft, qf, p.scale_log2, i * BK + kg * BN, 0,
                                                         hi, lane);
        wait_vmem();
        lds_barrier();
        buf ^= 1;
      }
    };
    run(std::false_type{}, min(n_full, it.end));
    run(std::true_type{}, it.end);
  }
  if constexpr (KG > 1) {
    rb.template merge<KG, NWR>(kg, rw, lane, reinterpret_cast<float*>(&lds[0][0][0]));
    __syncthreads();     // (the stages are written again below)
    if (kg > 0) return;  // no barrier follows
  }
  // scratch: a half stage holds the rows of BK / 32 waves (every wave has passed the last barrier)
  constexpr int PER = BK / 32;
  const int half = rw / PER;
  static_assert(NWR <= 2 * PER * 2, "the stages hold every wave's rows");
  finish_packed<D, BM, BN>(p, rb, it, hk, rw * 32, (half & 1 ? Vs : Ks)[half >> 1] + (rw - half * PER) * 32 * D, lane);
}

// Join of a cut tile's partial results, in their order: with M the largest m_s, O = sum 2^(m_s - M) O_s /
// sum 2^(m_s - M) l_s and LSE = (M + log2 of that sum) ln 2.  One thread for four columns of a row.  A launch and two
// reads, one after another: 5 us, also where the plan has cut nothing.
template <int D, int BM>
__global__ __launch_bounds__(256) void packed_join_kernel(PackedParams p) {
  constexpr int TPR = D / 4, BLOCKS = join_blocks(BM, D);
  const int n = p.list[1] * p.Hkv * BLOCKS;
  for (int id = blockIdx.x; id < n; id += gridDim.x) {
    const int job = id / BLOCKS, j = job / p.Hkv, hk = job - j * p.Hkv;
    const PackedJoin it = p.joins[j];
    const int x = (id - job * BLOCKS) * 256 + threadIdx.x, rt = x / TPR, col = (x - rt * TPR) * 4;
    const int row = it.tile * BM + rt, G = p.G;
    if (rt >= BM || row >= it.nq * G) continue;
    const float* ml = p.part + (long long)p.max_slots * p.Hkv * BM * D;
    float M = -INFINITY, l = 0.f;
    f32x4 acc = zero4();
    constexpr int U = 4;  // partial results in flight
    for (int s0 = 0; s0 < it.parts; s0 += U) {
      float mv[U], lv[U];
      f32x4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool in = s0 + u < it.parts;
        const long long at = ((long long)(it.first + (in ? s0 + u : s0)) * p.Hkv + hk) * BM + rt;
        mv[u] = in ? ml[2 * at] : -INFINITY;
        lv[u] = ml[2 * at + 1];
        v[u] = *reinterpret_cast<const f32x4*>(p.part + at * D + col);
      }
      float Mn = M;
#pragma unroll
      for (int u = 0; u < U; ++u) Mn = fmaxf(Mn, mv[u]);
      const float a = M == -INFINITY ? 0.f : fast_exp2(M - Mn);
      l *= a;
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[c] *= a;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float w = mv[u] == -INFINITY ? 0.f : fast_exp2(mv[u] - Mn);
        l = fmaf(w, lv[u], l);
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[c] = fmaf(w, v[u][c], acc[c]);
      }
      M = Mn;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    bf16x4 w;
#pragma unroll
    for (int c = 0; c < 4; ++c) w[c] = to_bf16(acc[c] * inv);
    *reinterpret_cast<bf16x4*>(p.o + packed_offset(p.so, hk, G, it.q0, row) + col) = w;
    if (col == 0) {
      const int t = row / G;
      p.lse[(long long)(hk * G + (row - t * G)) * p.total_q + it.q0 + t] =
          l == 0.f ? -INFINITY : (M + __log2f(l)) * 0.69314718055994530942f;
    }
  }
}

namespace {

template <int NW, int BN, int KG, int WPS>
hipError_t launch_fwd_tile(const PackedParams& p, const PackedList& list, hipStream_t stream) {
  constexpr int BM = 32 * NW / KG;
  if (list.tile != BM || list.step != BN * KG) return hipErrorInvalidValue;
  const long long grid = (long long)list.max_items * p.Hkv;
  const long long joins = std::min((long long)list.max_joins * p.Hkv * join_blocks(BM, kD), (long long)kJoinGrid);
  if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
  hipLaunchKernelGGL((packed_fwd_kernel<kD, NW, BN, KG, WPS>), dim3((unsigned)grid), dim3(64 * NW), 0, stream, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.part == nullptr) return e;
  hipLaunchKernelGGL((packed_join_kernel<kD, BM>), dim3((unsigned)joins), dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

#define MW_CAT_(a, b) a##b
#define MW_CAT(a, b) MW_CAT_(a, b)
hipError_t MW_CAT(launch_packed_fwd_, MW_PACKED_HEAD_DIM)(const PackedParams& p, const PackedList& list, hipStream_t stream) {
  if (list.kind == PackedTile::pairs) return launch_fwd_tile<4, 32, 2, packed_fwd_per_cu(kD, PackedTile::pairs)>(p, list, stream);
  return launch_fwd_tile<4, 64, 1, packed_fwd_per_cu(kD, PackedTile::wide)>(p, list, stream);
}

}  // namespace mw
