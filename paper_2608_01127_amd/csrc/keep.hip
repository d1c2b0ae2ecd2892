// Eviction of a sequence's light tokens (gfx950): which tokens stay, and their copy into pages of their own.
#include "mw_device.h"
#include "mw_kernels.h"
#include "pages_codes.h"

namespace mw {

namespace {

constexpr int kThreads = 1024, kCached = 32768, kBins = 2048;

// Order of the weights as unsigned numbers; -0 is 0, NaN is the lightest.
__device__ __forceinline__ unsigned order_of(float w) {
  if (!(w == w)) return 0;
  const unsigned u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

}  // namespace

// One workgroup for each sequence.  Of its tokens [first, len - recent) the k heaviest stay, of equal ones those in
// front: the weight of the k-th is found by three counts of 11, 11 and 10 bits, from the top; then each wave walks its
// stretch of the tokens in order and lists what stays, with its page, at the place that the stretches in front leave.
__global__ __launch_bounds__(kThreads) void keep_select_kernel(PagePool c, KeepArgs a, const float* weights, int2* list,
                                                               float* kept) {
  __shared__ unsigned cache[kCached];
  __shared__ int bins[kBins];
  __shared__ int wave_sums[16], wave_gt[16], wave_eq[16];
  __shared__ int chosen, above;
  const int job = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int seq = a.seq[job], len = a.len[job], n = len - a.recent - a.first, k = a.keep - a.recent - a.first;
  const float* w = weights + (long long)seq * c.W * c.L;
  const int* row = c.table + (long long)seq * c.W;
  const int from = a.first / c.L * c.L;  // the anchor's whole pages stay where they are
  list += (long long)job * (a.keep - from);
  kept += (long long)job * (a.keep - from);
  const bool cached = n <= kCached;
  for (int i = tid; cached && i < n; i += kThreads) cache[i] = order_of(w[a.first + i]);
  auto key = [&](int i) { return cached ? cache[i] : order_of(w[a.first + i]); };
  unsigned limit = 0;  // the k-th heaviest, bit group by bit group
  int left = k;        // how many of those that agree with the groups so far stay
  for (int pass = 0; pass < 3 && k > 0; ++pass) {
    const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bits = pass == 2 ? 10 : 11;
    for (int i = tid; i < kBins; i += kThreads) bins[i] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) {
      const unsigned x = key(i);
      if (pass == 0 || (x >> (shift + bits)) == (limit >> (shift + bits)))
        atomicAdd(&bins[(x >> shift) & ((1u << bits) - 1)], 1);
    }
    __syncthreads();
    // the bin, from the top, that holds the left-th: a thread's two bins, then the sums over threads above
    const int hi = kBins - 1 - 2 * tid, two = bins[hi] + bins[hi - 1];
    int in = two;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(in, d);
      if (lane >= d) in += y;
    }
    if (lane == 63) wave_sums[wave] = in;
    __syncthreads();
    int front = in - two;
    for (int i = 0; i < wave; ++i) front += wave_sums[i];
    if (front < left && front + two >= left) {
      const bool second = front + bins[hi] < left;
      chosen = second ? hi - 1 : hi;
      above = second ? front + bins[hi] : front;
    }
    __syncthreads();
    limit |= (unsigned)chosen << shift;
    left -= above;
    __syncthreads();
  }
  __syncthreads();
  // this wave's stretch: how many are heavier than the limit, and equal to it
  const int per = (n + 15) / 16, i0 = min(n, wave * per), i1 = min(n, i0 + per);
  int gt = 0, eq = 0;
  for (int i = i0 + lane; i < i1; i += 64) {
    const unsigned x = key(i);
    gt += x > limit;
    eq += x == limit;
  }
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) {
    gt += __shfl_xor(gt, m);
    eq += __shfl_xor(eq, m);
  }
  if (lane == 0) {
    wave_gt[wave] = gt;
    wave_eq[wave] = eq;
  }
  __syncthreads();
  gt = eq = 0;
  for (int i = 0; i < wave; ++i) {
    gt += wave_gt[i];
    eq += wave_eq[i];
  }
  auto put = [&](int place, int token) {  // entry of the token at `place` of the new sequence
    list[place - from] = make_int2(row[token / c.L], token % c.L);
    kept[place - from] = w[token];
  };
  const unsigned long long below = (1ULL << lane) - 1;
  for (int i = i0; i < i1 && k > 0; i += 64) {
    const bool in = i + lane < i1;
    const unsigned x = in ? key(i + lane) : 0;
    const unsigned long long e = __builtin_amdgcn_ballot_w64(in && x == limit);
    const int mine = eq + __builtin_popcountll(e & below);
    const bool stays = in && (x > limit || (x == limit && mine < left));
    const unsigned long long s = __builtin_amdgcn_ballot_w64(stays);
    if (stays) put(a.first + gt + min(eq, left) + __builtin_popcountll(s & below), a.first + i + lane);
    // (gt + min(eq, left) tokens stay in front of this step)
    const unsigned long long g = __builtin_amdgcn_ballot_w64(in && x > limit);
    gt += __builtin_popcountll(g);
    eq += __builtin_popcountll(e);
  }
  for (int i = from + tid; i < a.first; i += kThreads) put(i, i);
  for (int i = tid; i < a.recent; i += kThreads) put(a.keep - a.recent + i, len - a.recent + i);
}

// The listed tokens into their pages: one workgroup for 64 of them of one head, K (blockIdx.y < H) or V.  Their block's
// scale is the least that holds them, so a code changes only where its own block's scale was finer.  The workgroups of
// K's first head also write the weights' row, the table and the length.
template <int D>
__global__ __launch_bounds__(256) void keep_gather_kernel(PagePool c, KeepRun a, float* weights, const int2* list,
                                                          const float* kept) {
  constexpr int PPR = D / 8, PIECES = 64 * PPR, ROUNDS = (PIECES + 255) / 256;
  const int run = blockIdx.z, tid = threadIdx.x, L = c.L;
  const int first = a.first[run], n_tok = a.n_tok[run];  // places [first, first + n_tok), first on a page's start
  const int at = first + (int)blockIdx.x * 64;
  float* w = weights + (long long)a.seq[run] * c.W * L;
  if (a.last[run] && blockIdx.x == 0 && blockIdx.y == 0) {
    if (tid == 0) c.lens[a.seq[run]] = a.keep;
    for (int i = a.keep + tid; i < a.len[run]; i += 256) w[i] = 0.f;  // places that are free again weigh nothing
  }
  if (at >= first + n_tok) return;
  const int n = min(64, first + n_tok - at);
  list += (long long)a.job[run] * a.stride + (at - a.from);
  kept += (long long)a.job[run] * a.stride + (at - a.from);
  const int dst_page = a.pages[a.page0[run] + (at - first) / L], off = at % L;
  if (blockIdx.y == 0) {
    if (tid < n) w[at + tid] = kept[tid];
    if (off == 0 && tid == 0) c.table[(long long)a.seq[run] * c.W + at / L] = dst_page;
  }
  const bool is_v = blockIdx.y >= (unsigned)c.H;
  const int h = is_v ? blockIdx.y - c.H : blockIdx.y, per = L / 64;
  uint8_t* pages = is_v ? c.v_pages : c.k_pages;
  float* scales = is_v ? c.v_scales : c.k_scales;
  float x[ROUNDS][8];
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int p = i * 256 + tid, r = p / PPR;
    if (r >= n) continue;
    const int2 from = list[r];
    const long long head = (long long)from.x * c.H + h;
    const u32x2 u = *reinterpret_cast<const u32x2*>(pages + (head * L + from.y) * D + (p - r * PPR) * 8);
    decode8(u, x[i]);
    const float scale = scales[head * per + from.y / 64];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[i][j] *= scale;
      amax = fmaxf(amax, fabsf(x[i][j]));  // (a NaN leaves it)
    }
  }
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) amax = fmaxf(amax, __shfl_xor(amax, m));
  __shared__ float wave_max[4];
  if ((tid & 63) == 0) wave_max[tid >> 6] = amax;
  __syncthreads();
  amax = fmaxf(fmaxf(wave_max[0], wave_max[1]), fmaxf(wave_max[2], wave_max[3]));
  const int e = block_exponent(amax);
  const float inv = pow2(-e);
  const long long head = (long long)dst_page * c.H + h;
  if (tid == 0) scales[head * per + off / 64] = pow2(e);
  uint8_t* dst = pages + (head * L + off) * D;
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int p = i * 256 + tid, r = p / PPR;
    if (r < n) *reinterpret_cast<u32x2*>(dst + r * D + (p - r * PPR) * 8) = encode8(x[i], inv);
  }
}

hipError_t launch_keep_select(const PagePool& c, const KeepArgs& a, const float* weights, int2* list, float* kept,
                              hipStream_t stream) {
  hipLaunchKernelGGL(keep_select_kernel, dim3(a.n_jobs), dim3(kThreads), 0, stream, c, a, weights, list, kept);
  return hipGetLastError();
}

hipError_t launch_keep_gather(const PagePool& c, const KeepRun& a, float* weights, const int2* list, const float* kept,
                              hipStream_t stream) {
  int blocks = 1;
  for (int j = 0; j < a.n_runs; ++j) blocks = std::max(blocks, (a.n_tok[j] + 63) / 64);
  const dim3 grid(blocks, 2 * c.H, a.n_runs);
  if (c.D == 64)
    hipLaunchKernelGGL(keep_gather_kernel<64>, grid, dim3(256), 0, stream, c, a, weights, list, kept);
  else if (c.D == 72)
    hipLaunchKernelGGL(keep_gather_kernel<72>, grid, dim3(256), 0, stream, c, a, weights, list, kept);
  else
    hipLaunchKernelGGL(keep_gather_kernel<128>, grid, dim3(256), 0, stream, c, a, weights, list, kept);
  return hipGetLastError();
}

}  // namespace mw
