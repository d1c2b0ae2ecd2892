// Attention weight of the paged cache's tokens (gfx950): what each cached token gets from a call's rows.  keep.hip evicts
// by it.
#include <algorithm>

#include "attn_rows.h"
#include "mw_kernels.h"

namespace mw {

namespace {

// Sum of 16 values over the 32 lanes of a half wave: lane l of a half holds the sum of value (l % 32) / 2.
__device__ __forceinline__ float sum16_over32(float (&v)[16], int lane) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const bool up = lane & 16;
    const float mine = up ? v[i + 8] : v[i], other = up ? v[i] : v[i + 8];
    v[i] = mine + __shfl_xor(other, 16);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool up = lane & 8;
    const float mine = up ? v[i + 4] : v[i], other = up ? v[i] : v[i + 4];
    v[i] = mine + __shfl_xor(other, 8);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const bool up = lane & 4;
    const float mine = up ? v[i + 2] : v[i], other = up ? v[i] : v[i + 2];
    v[i] = mine + __shfl_xor(other, 4);
  }
  const bool up = lane & 2;
  const float mine = up ? v[1] : v[0], other = up ? v[0] : v[1];
  const float x = mine + __shfl_xor(other, 2);
  return x + __shfl_xor(x, 1);
}

// Eight codes from column 16 kk + 8 (lane / 32) on of the row at `row`, as values: K fragment of contraction step kk
// (zeros for columns past D).
template <int D>
__device__ __forceinline__ bf16x8 key_fragment(const uint8_t* row, int kk, int h, float scale) {
  if (D % 16 != 0 && 16 * kk + 8 * h >= D) return decode(0u, 0u, scale);
  const u32x2 x = *reinterpret_cast<const u32x2*>(row + 16 * kk + 8 * h);
  return decode(x[0], x[1], scale);
}

// Member and first block of block number `range` of a call.
__device__ __forceinline__ int member_of(const WeighParams& p, const WeighSeqs& seqs, int range, int lane) {
  int b = -1;  // the last member whose first block is not behind this one
  for (int i = 0; i < p.B; i += 64) {
    const int first = seqs.first[min(i + lane, p.B)];
    b += __builtin_popcountll(__builtin_amdgcn_ballot_w64(i + lane < p.B && first <= range));
  }
  return __builtin_amdgcn_readfirstlane(b);
}

// This lane's sum over its half wave's rows of the block's 64 keys -> sums[key].
__device__ __forceinline__ void sum_rows(const f32x16 (&acc)[2], float* sums, int lane) {
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = acc[kb][i];
    const float x = sum16_over32(v, lane);
    if (!(lane & 1)) sums[kb * 32 + acc_row((lane & 31) >> 1, lane)] = x;
  }
}

__device__ __forceinline__ void put_sum(const WeighParams& p, const WeighSeqs& seqs, float x, int part, int range, int seq,
                                        int token, int lane) {
  if (p.n_parts > 1) {
    p.part[((long long)part * seqs.first[p.B] + range) * 64 + lane] = x;
  } else {
    float* out = p.weights + (long long)seq * p.W * p.L + token;
    *out = p.add ? *out + x : x;
  }
}

}  // namespace

// w_j = sum over rows r and key heads of exp(scale q_r k_j - LSE_r).  A wave keeps a block of 64 cached tokens' keys of a
// head in registers (S^T = K Q^T, rows of S^T are keys) and adds up the probabilities of its rows there, so that rows are
// summed across lanes once, at the end.  Sums are in 32 bits, in an order that the sizes and the
// workspace decide; no atomics.
//
// Few rows: bound by reading the codes.  A workgroup takes one block and one part of the pairs (key head, tile of 32 rows),
// its waves take pairs in turn and read Q as they need it.  Short workgroups, so the more at once the better (one token of 8
// sequences of up to 15840 tokens, 4 key heads, 51 MB: two waves a SIMD 19.1 us, three 15.9, 3.2 TB/s; four spill).
template <int D, int NW>
__global__ __launch_bounds__(64 * NW, 3) void weigh_kernel(WeighParams p, WeighSeqs seqs) {
  constexpr int KK = (D + 15) / 16;
  constexpr bool TAIL = D % 16 != 0;
  __shared__ float sums[NW][64];
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int part = blockIdx.x % p.n_parts, range = blockIdx.x / p.n_parts;
  const int b = member_of(p, seqs, range, lane);
  const int blk = range - seqs.first[b], seq = seqs.seq[b], G = p.G;
  const int len = max(0, min(p.lens[seq], p.W * p.L));
  const int w = blk / p.per_page, page = p.table[(long long)seq * p.W + w], off = blk - w * p.per_page;
  const int tiles = (p.R + 31) / 32;
  const long long units = (long long)p.Hkv * tiles;
  const int beg = (int)(units * part / p.n_parts), end = (int)(units * (part + 1) / p.n_parts);

  f32x16 acc[2] = {zero16(), zero16()};
  bf16x8 kf[2][KK];
  int loaded = -1;
  for (int u = beg + wave; u < end; u += NW) {
    const int hk = u / tiles, rt = u - hk * tiles;
    // Q and LSE are asked for before the codes, which wait for the page's number
    const int row = rt * 32 + (lane & 31), rc = min(row, p.R - 1), t = G == 1 ? rc : rc / G;
    const bf16_t* qp = p.q + row_offset(p.sq, b, hk, G, rc);
    bf16x8 qf[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)  // (D = 72: K is zero where h = 1 repeats column 64)
      qf[kk] = *reinterpret_cast<const bf16x8*>(qp + (TAIL && kk == KK - 1 ? 64 : 32 * (kk / 2) + 16 * h + 8 * (kk & 1)));
    const float lse = p.lse[((long long)b * p.Hkv * G + hk * G + (rc - t * G)) * p.T + t];
    if (hk != loaded) {
      loaded = hk;
      const long long e = ((long long)page * p.Hkv + hk) * p.per_page + off;
      const float scale = p.k_scales[e];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const uint8_t* at = p.k_pages + (e * 64 + kb * 32 + (lane & 31)) * D;
#pragma unroll
        for (int j = 0; j < KK / 2; ++j) {  // sixteen codes of a row, eight for each of two contraction steps
          if constexpr (TAIL) {
            const u32x2 x = *reinterpret_cast<const u32x2*>(at + 32 * j + 16 * h);
            const u32x2 y = *reinterpret_cast<const u32x2*>(at + 32 * j + 16 * h + 8);
            kf[kb][2 * j] = decode(x[0], x[1], scale);
            kf[kb][2 * j + 1] = decode(y[0], y[1], scale);
          } else {
            const u32x4 x = *reinterpret_cast<const u32x4*>(at + 32 * j + 16 * h);
            kf[kb][2 * j] = decode(x[0], x[1], scale);
            kf[kb][2 * j + 1] = decode(x[2], x[3], scale);
          }
        }
        if constexpr (TAIL) kf[kb][KK - 1] = key_fragment<D>(at, KK - 1, h, scale);  // columns 64..71 and zeros
      }
    }
    // rows behind the last one, and rows that saw nothing, weigh nothing
    const float lse2 = row < p.R && lse != -INFINITY ? lse * 1.4426950408889634f : INFINITY;
    f32x16 s[2] = {zero16(), zero16()};
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) s[kb] = mfma32(kf[kb][kk], qf[kk], s[kb]);
    if (wave_any(lse == -INFINITY)) {  // (whatever their queries hold)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = lse == -INFINITY ? 0.f : s[kb][i];
    }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[kb][i] += fast_exp2(fmaf(s[kb][i], p.scale_log2, -lse2));
  }
  sum_rows(acc, sums[wave], lane);
  __syncthreads();
  if (tid >= 64) return;  // no barrier follows
  float x = 0.f;
#pragma unroll
  for (int i = 0; i < NW; ++i) x += sums[i][tid];
  const int token = blk * 64 + tid;
  if (token < len) put_sum(p, seqs, x, part, range, seq, token, tid);
}

// Many rows: a workgroup takes NW blocks of a member, one a wave, and one part of the pairs (key head, step of 64 rows),
// whose Q it stages in LDS for all of them, a step ahead (reading Q anew for each block: the 1B stream step below 718
// us).  Bound by the exponentials, 16 of 24 cycles of vector work an element, next to 16 of matrix work: vector work 67%,
// matrix units 53% busy, with what a wave waits for between them.  12 heads x 4800 rows of a guidance pair over 14700 and
// 11025 tokens, D = 128: 354 us, 1072 TF.
template <int D, int NW, int WPS>
__global__ __launch_bounds__(64 * NW, WPS) void weigh_rows_kernel(WeighParams p, WeighSeqs seqs) {
  constexpr int KK = (D + 15) / 16, NT = 64 * NW, BS = 64;
  constexpr int TE = stage_elems<D, BS, NT>();
  __shared__ __attribute__((aligned(16))) bf16_t Qs[2][TE];
  __shared__ float sums[NW][64];
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int part = blockIdx.x % p.n_parts, group = blockIdx.x / p.n_parts;
  int b = 0, first = 0;  // this group's member and its first group
  for (;;) {
    const int n = (seqs.first[b + 1] - seqs.first[b] + NW - 1) / NW;
    if (group < first + n) break;
    first += n;
    ++b;
  }
  const int blk = (group - first) * NW + wave, seq = seqs.seq[b], G = p.G;
  const int len = max(0, min(p.lens[seq], p.W * p.L));
  const bool busy = blk < seqs.first[b + 1] - seqs.first[b];
  const int w = (busy ? blk : 0) / p.per_page, page = p.table[(long long)seq * p.W + w], off = (busy ? blk : 0) - w * p.per_page;
  const int steps = (p.R + BS - 1) / BS;
  const long long units = (long long)p.Hkv * steps;
  const int beg = (int)(units * part / p.n_parts), end = (int)(units * (part + 1) / p.n_parts);
  const FragOffsets<D> fo(lane, 0);
  const RowOffsets<D, BS, NT> ro(p.sq.t, tid);
  const float* lse_b = p.lse + (long long)b * p.Hkv * G * p.T;
  float lse_row = 0.f;  // of the staged step's row `lane`
  auto stage = [&](int u, int buf) {
    const int hk = u / steps, r0 = (u - hk * steps) * BS;
    const bf16_t* base = p.q + b * p.sq.b + (long long)hk * G * p.sq.h;
    if (r0 + BS <= p.R && G == 1) {
      stage_rows_s<D, BS, NT>(Qs[buf], base + r0 * p.sq.t, ro, tid);
    } else if (r0 + BS <= p.R && p.near) {
      stage_group<D, BS, NT>(Qs[buf], base, p.sq, r0, G, p.magic, tid);
    } else {
      stage_rows_direct<D, BS, NT>(Qs[buf], [&](int r) { return p.q + row_offset(p.sq, b, hk, G, min(r0 + r, p.R - 1)); }, tid);
    }
    const int t0 = G == 1 ? r0 : (unsigned)r0 / (unsigned)G, x = r0 - t0 * G + min(lane, p.R - 1 - r0);
    const int t = G == 1 ? x : __umulhi((unsigned)x, p.magic);
    lse_row = lse_b[(long long)(hk * G + x - t * G) * p.T + t0 + t];
  };
  f32x16 acc[2] = {zero16(), zero16()};
  bf16x8 kf[2][KK];
  int loaded = -1, buf = 0;
  if (beg < end) stage(beg, 0);
  for (int u = beg; u < end; ++u) {
    const int hk = u / steps, r0 = (u - hk * steps) * BS;
    if (hk != loaded) {
      loaded = hk;
      const long long e = ((long long)page * p.Hkv + hk) * p.per_page + off;
      const float scale = p.k_scales[e];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
          kf[kb][kk] = key_fragment<D>(p.k_pages + (e * 64 + kb * 32 + (lane & 31)) * D, kk, h, scale);
    }
    wait_vmem();
    __syncthreads();  // this step has landed, and the other stage has been read
    const bool none = lse_row == -INFINITY;
    // rows behind the last one, and rows that saw nothing, weigh nothing; both half waves take rows 0..31, then 32..63
    const unsigned bits = __float_as_uint(r0 + lane < p.R && !none ? lse_row * 1.4426950408889634f : INFINITY);
    const auto lse2 = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);
    // queries of rows that saw nothing may hold anything: each wave clears them before it reads (D = 72: also row 0's first
    // columns behind the last row, which that one's read runs into)
    if (__builtin_expect(wave_any(none), 0)) {
#pragma unroll 1
      for (int i = 0; i < D / 8; ++i)
        if (none) *reinterpret_cast<bf16x8*>(Qs[buf] + lane * D + 8 * i) = bf16x8{};
      if (D % 16 != 0 && lane == 0 && none) *reinterpret_cast<bf16x8*>(Qs[buf] + BS * D) = bf16x8{};
    }
    if (u + 1 < end) stage(u + 1, buf ^ 1);
    if (busy) {
#pragma unroll
      for (int qb = 0; qb < BS / 32; ++qb) {
        f32x16 s[2] = {zero16(), zero16()};
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          const bf16x8 qf = fo.row8(Qs[buf], qb * 32, kk);
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) s[kb] = mfma32(kf[kb][kk], qf, s[kb]);
        }
        __builtin_amdgcn_s_setprio(0);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[kb][i] += fast_exp2(fmaf(s[kb][i], p.scale_log2, -__uint_as_float(lse2[qb])));
      }
    }
    buf ^= 1;
  }
  if (!busy) return;  // no barrier follows
  sum_rows(acc, sums[wave], lane);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the wave's own sums: no barrier)
  const int token = blk * 64 + lane;
  if (token < len) put_sum(p, seqs, sums[wave][lane], part, seqs.first[b] + blk, seq, token, lane);
}

// Sums of the parts, in order.
__global__ __launch_bounds__(256) void weigh_join_kernel(WeighParams p, WeighSeqs seqs) {
  const int id = blockIdx.x * 256 + threadIdx.x, range = id / 64, n = seqs.first[p.B];
  if (range >= n) return;
  int lo = 0, hi = p.B - 1;  // the last member whose first block is not behind this one
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (seqs.first[mid] <= range) {
      lo = mid;
    } else {
      hi = mid - 1;
    }
  }
  const int seq = seqs.seq[lo], token = id - seqs.first[lo] * 64;
  if (token >= max(0, min(p.lens[seq], p.W * p.L))) return;
  float x = 0.f;
  for (int s = 0; s < p.n_parts; ++s) x += p.part[(long long)s * n * 64 + id];
  float* out = p.weights + (long long)seq * p.W * p.L + token;
  *out = p.add ? *out + x : x;
}

namespace {

constexpr int kWaves = 4;

template <int D>
hipError_t launch_weigh_dim(const WeighParams& p, const WeighSeqs& seqs, hipStream_t stream) {
  const int blocks = seqs.first[p.B];
  long long grid = blocks;
  if (p.many) {
    grid = 0;
    for (int b = 0; b < p.B; ++b) grid += (seqs.first[b + 1] - seqs.first[b] + kWaves - 1) / kWaves;
  }
  grid *= p.n_parts;
  if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
  if (grid == 0) return hipSuccess;
  if (p.many) {
    hipLaunchKernelGGL((weigh_rows_kernel<D, kWaves, 2>), dim3((unsigned)grid), dim3(64 * kWaves), 0, stream, p, seqs);
  } else {
    hipLaunchKernelGGL((weigh_kernel<D, 4>), dim3((unsigned)grid), dim3(256), 0, stream, p, seqs);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.n_parts == 1) return e;
  hipLaunchKernelGGL(weigh_join_kernel, dim3((unsigned)((blocks + 3) / 4)), dim3(256), 0, stream, p, seqs);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_weigh(const WeighParams& p, const WeighSeqs& seqs, int D, hipStream_t stream) {
  return D == 64   ? launch_weigh_dim<64>(p, seqs, stream)
         : D == 72 ? launch_weigh_dim<72>(p, seqs, stream)
                   : launch_weigh_dim<128>(p, seqs, stream);
}

// The kernel of a call and the parts of its rows (over all key heads), so that there are workgroups enough for the card.
// Staging rows for several blocks pays from 65 rows of a key head on, where there is work for the card (12 heads over 14700
// tokens, D = 128, us: 64 rows 18.3 few | 42.5 many, 128 29.4 | 19.4, 600 82 | 41; 4 heads x 2000 rows over 300 tokens, D =
// 64, 13.9 | 22.7).  Its parts are those of the least time in rounds of the 512 workgroups that run at once at D = 128
// (three a CU at D = 64 and 72, priced as two), each of its steps and a beginning as long as three (always about 768 workgroups:
// the 1B stream step 386 us, so 367).
// No more parts than the workspace holds, and never more than kWeighBytes of them (by this count of rounds that costs 1.3%
// at most in 20000 drawn sizes of up to 2^18 blocks and 2^17 rows; without the limit parts of 750 MB came up).
WeighPlan weigh_plan(int Hkv, int R, long long blocks, size_t bytes) {
  const long long groups = (blocks + kWaves - 1) / kWaves, steps = (long long)Hkv * ((R + 63) / 64);
  const long long most = std::max(1LL, (long long)(std::min(bytes, kWeighBytes) / weigh_part_bytes(std::max(1LL, blocks))));
  if (R > 64 && groups * steps >= 1024) {
    long long best = 0;
    WeighPlan plan{true, 1};
    for (long long n = 1; n <= std::min({64LL, steps, most}); ++n) {
      const long long t = (groups * n + 511) / 512 * ((steps + n - 1) / n + 3);
      if (n > 1 && t >= best) continue;
      best = t;
      plan.parts = (int)n;
    }
    return plan;
  }
  const long long units = (long long)Hkv * ((R + 31) / 32);
  return {false, (int)std::max(1LL, std::min({units / 16, (1024 + blocks - 1) / std::max(1LL, blocks), most}))};
}

}  // namespace mw
