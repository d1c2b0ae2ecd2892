// Eviction from the paged cache by accumulated attention weight (gfx950): what weight each cached token gets from a
// call's rows, and the copy of a sequence's anchor, newest and heaviest tokens into pages of their own.
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

}  // namespace

// w_j = sum over rows r and key heads of exp(scale q_r k_j - LSE_r).  A workgroup takes one block of 64 cached tokens and
// one part of the pairs (key head, tile of 32 rows); a wave keeps the block's keys of a head in registers (S^T = K Q^T,
// rows of S^T are keys) and adds up its tiles' probabilities there, so that rows are summed across lanes once, at the
// end.  Sums are in 32 bits, in an order that the sizes alone decide; no atomics.
template <int D, int NW>
__global__ __launch_bounds__(64 * NW, 2) void weigh_kernel(WeighParams p, WeighSeqs seqs) {
  constexpr int KK = (D + 15) / 16;
  constexpr bool TAIL = D % 32 != 0;
  __shared__ float sums[NW][64];
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int part = blockIdx.x % p.n_parts, range = blockIdx.x / p.n_parts;
  int b = -1;  // the last member whose first block is not behind this one
  for (int i = 0; i < p.B; i += 64) {
    const int first = seqs.first[min(i + lane, p.B)];
    b += __builtin_popcountll(__builtin_amdgcn_ballot_w64(i + lane < p.B && first <= range));
  }
  b = __builtin_amdgcn_readfirstlane(b);
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
        if constexpr (TAIL) {  // columns 64..71 and zeros
          const u32x2 x = *reinterpret_cast<const u32x2*>(at + 64);
          kf[kb][KK - 1] = decode(h ? 0u : x[0], h ? 0u : x[1], scale);
        }
      }
    }
    const int row = rt * 32 + (lane & 31), rc = min(row, p.R - 1), t = rc / G;
    const bf16_t* qp = p.q + row_offset(p.sq, b, hk, G, rc);
    const float lse = p.lse[((long long)b * p.Hkv * G + hk * G + (rc - t * G)) * p.T + t];
    // rows behind the last one, and rows that saw nothing, weigh nothing
    const float lse2 = row < p.R && lse != -INFINITY ? lse * 1.4426950408889634f : INFINITY;
    f32x16 s[2] = {zero16(), zero16()};
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const int col = TAIL && kk == KK - 1 ? 64 : 32 * (kk / 2) + 16 * h + 8 * (kk & 1);
      const bf16x8 qf = *reinterpret_cast<const bf16x8*>(qp + col);  // (D = 72: K is zero where h = 1 repeats column 64)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) s[kb] = mfma32(kf[kb][kk], qf, s[kb]);
    }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[kb][i] += fast_exp2(fmaf(s[kb][i], p.scale_log2, -lse2));
  }
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = acc[kb][i];
    const float x = sum16_over32(v, lane);
    if (!(lane & 1)) sums[wave][kb * 32 + acc_row((lane & 31) >> 1, lane)] = x;
  }
  __syncthreads();
  if (tid >= 64) return;  // no barrier follows
  float x = 0.f;
#pragma unroll
  for (int i = 0; i < NW; ++i) x += sums[i][tid];
  const int token = blk * 64 + tid;
  if (token >= len) return;
  if (p.n_parts > 1) {
    p.part[((long long)part * seqs.first[p.B] + range) * 64 + tid] = x;
  } else {
    float* out = p.weights + (long long)seq * p.W * p.L + token;
    *out = p.add ? *out + x : x;
  }
}

// Sums of the parts, in order.
template <int D>
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

template <int D>
hipError_t launch_weigh_dim(const WeighParams& p, const WeighSeqs& seqs, hipStream_t stream) {
  const int blocks = seqs.first[p.B];
  const long long grid = (long long)blocks * p.n_parts;
  if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
  if (grid == 0) return hipSuccess;
  hipLaunchKernelGGL((weigh_kernel<D, 4>), dim3((unsigned)grid), dim3(256), 0, stream, p, seqs);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.n_parts == 1) return e;
  hipLaunchKernelGGL(weigh_join_kernel<D>, dim3((unsigned)((blocks + 3) / 4)), dim3(256), 0, stream, p, seqs);
  return hipGetLastError();
}

hipError_t launch_weigh(const WeighParams& p, const WeighSeqs& seqs, int D, hipStream_t stream) {
  return D == 64   ? launch_weigh_dim<64>(p, seqs, stream)
         : D == 72 ? launch_weigh_dim<72>(p, seqs, stream)
                   : launch_weigh_dim<128>(p, seqs, stream);
}

// Parts of the (key head, row tile) pairs, so that there are workgroups enough for the card, of a few tiles a wave.
int weigh_parts(int Hkv, int R, long long blocks) {
  const long long units = (long long)Hkv * ((R + 31) / 32);
  const long long most = std::max(1LL, units / 16);
  return (int)std::max(1LL, std::min(most, (1024 + blocks - 1) / std::max(1LL, blocks)));
}

}  // namespace mw
