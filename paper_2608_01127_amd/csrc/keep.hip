// Eviction of a sequence's light tokens (gfx950): which tokens stay, and their copy into pages of their own.
#include "mw_device.h"
#include "mw_kernels.h"
#include "pages_codes.h"

namespace mw {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kEach = 16, kBins = 256, kCopies = 32, kFew = 64;

// Order of the weights as unsigned numbers; -0 is 0, NaN is the lightest.
__device__ __forceinline__ unsigned order_of(float w) {
  if (!(w == w)) return 0;
  const unsigned u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

}  // namespace

// One workgroup for each sequence.  Of its tokens [first, len - recent) the k heaviest stay, of equal ones those in
// front: the weight of the k-th is found by four counts of 8 bits, from the top; with the numbers of heavier and equal ones in
// front of it, every token knows whether it stays and where.  A thread holds 16 tokens' weights in registers, every 1024th;
// more tokens than that are read again for each count.  Weights that lie close fall into few bins: each bin has a counter
// for every lane of a half wave, on a bank of its own.  Bound by its own latencies, one after another: 12 us for 2700 tokens,
// 18 for 12900 (walking them a wave a stretch, looking up pages on the way: 25; without the ranking of the last few 20).
__global__ __launch_bounds__(kThreads) void keep_select_kernel(PagePool c, KeepArgs a, const float* __restrict__ weights,
                                                               int2* __restrict__ list, float* __restrict__ kept) {
  __shared__ int bins[kBins * kCopies];
  __shared__ int counts[kBins];
  __shared__ int heavier[kEach * kWaves + 1], equal[kEach * kWaves + 1];
  __shared__ unsigned few[kFew];
  __shared__ int chosen, above, n_few;
  static_assert(kEach * kWaves == 256, "one wave adds up the counts, four a lane");
  const int job = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int seq = a.seq[job], len = a.len[job], n = len - a.recent - a.first, k = a.keep - a.recent - a.first;
  const float* w = weights + (long long)seq * c.W * c.L;
  const int* row = c.table + (long long)seq * c.W;
  const int from = a.first / c.L * c.L;  // the anchor's whole pages stay where they are
  list += (long long)job * (a.keep - from);
  kept += (long long)job * (a.keep - from);
  const int per = c.L / 64;
  auto put = [&](int place, int token, float weight) {  // entry of the token at `place` of the new sequence
    const int blk = token >> 6, at = per == 1 ? blk : (int)__umulhi((unsigned)blk, a.per_page_magic);
    list[place - from] = make_int2(row[at], token - at * c.L);
    kept[place - from] = weight;
  };
  for (int i = from + tid; i < a.first; i += kThreads) put(i, i, w[i]);
#pragma unroll 4
  for (int i = tid; i < a.recent; i += kThreads) put(a.keep - a.recent + i, len - a.recent + i, w[len - a.recent + i]);
  if (k == 0) return;

  constexpr int CHUNK = kEach * kThreads;
  const bool once = n <= CHUNK;
  float v[kEach];
  auto load = [&](int c0) {
#pragma unroll
    for (int j = 0; j < kEach; ++j) v[j] = w[a.first + min(c0 + j * kThreads + tid, n - 1)];
  };
  load(0);
  unsigned limit = 0;  // the k-th heaviest, bit group by bit group
  int left = k;        // how many of those that agree with the groups so far stay
  for (int shift = 24; shift >= 0; shift -= 8) {
#pragma unroll
    for (int i = 0; i < kBins * kCopies / kThreads; ++i) bins[i * kThreads + tid] = 0;
    __syncthreads();
    for (int c0 = 0; c0 < n; c0 += CHUNK) {
      if (!once) load(c0);
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        if (c0 + j * kThreads >= n) break;
        const unsigned x = order_of(v[j]);
        const bool agrees = shift == 24 || (x >> (shift + 8)) == (limit >> (shift + 8));
        if (agrees && c0 + j * kThreads + tid < n) atomicAdd(&bins[((x >> shift) & 255u) * kCopies + (lane & 31)], 1);
      }
    }
    __syncthreads();
    {  // four threads add up a bin's counters
      int sum = 0;
#pragma unroll
      for (int i = 0; i < kCopies / 4; ++i) sum += bins[(tid >> 2) * kCopies + ((i * 4 + tid + (tid >> 2)) & 31)];
      sum += __shfl_xor(sum, 1);
      sum += __shfl_xor(sum, 2);
      if ((tid & 3) == 0) counts[tid >> 2] = sum;
    }
    __syncthreads();
    if (wave == 0) {  // the bin, from the top, that holds the left-th: four bins a lane
      int own[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        own[i] = counts[kBins - 1 - 4 * lane - i];
        sum += own[i];
      }
      int front = sum;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(front, d);
        if (lane >= d) front += y;
      }
      front -= sum;
      if (front < left && front + sum >= left) {
        int bin = kBins - 1 - 4 * lane;
#pragma unroll
        for (int i = 0; i < 3; ++i)
          if (front + own[i] < left && bin == kBins - 1 - 4 * lane - i) {
            front += own[i];
            --bin;
          }
        chosen = bin;
        above = front;
      }
    }
    __syncthreads();
    limit |= (unsigned)chosen << shift;
    left -= above;
    if (counts[chosen] > kFew || shift == 0) continue;
    // few are left to choose from: each of them is ranked among them
    if (tid == 0) n_few = 0;
    __syncthreads();
    for (int c0 = 0; c0 < n; c0 += CHUNK) {
      if (!once) load(c0);
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        const unsigned x = order_of(v[j]);
        if (c0 + j * kThreads + tid < n && (x >> shift) == (limit >> shift)) few[atomicAdd(&n_few, 1)] = x;
      }
    }
    __syncthreads();
    if (wave == 0) {
      const int m = n_few;
      const unsigned x = few[lane < m ? lane : 0];
      int heavier_few = 0, equal_few = 0;
      for (int i = 0; i < m; ++i) {
        const unsigned y = __shfl(x, i);
        heavier_few += y > x;
        equal_few += y == x;
      }
      // the left-th (lanes of equal values agree)
      if (lane < m && heavier_few < left && heavier_few + equal_few >= left) {
        few[0] = x;
        above = heavier_few;
      }
    }
    __syncthreads();
    limit = few[0];
    left -= above;
    break;
  }

  int gt0 = 0, eq0 = 0;  // heavier and equal tokens of the chunks in front
  const unsigned long long below = (1ULL << lane) - 1;
  for (int c0 = 0; c0 < n; c0 += CHUNK) {
    if (!once) load(c0);
    unsigned long long gt[kEach], eq[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const bool in = c0 + j * kThreads + tid < n;
      const unsigned x = order_of(v[j]);
      gt[j] = __builtin_amdgcn_ballot_w64(in && x > limit);
      eq[j] = __builtin_amdgcn_ballot_w64(in && x == limit);
      if (lane == 0) {
        heavier[j * kWaves + wave] = __builtin_popcountll(gt[j]);
        equal[j * kWaves + wave] = __builtin_popcountll(eq[j]);
      }
    }
    __syncthreads();
    if (wave < 2) {  // numbers in front of each wave's 64 tokens
      int* x = wave == 0 ? heavier : equal;
      int own[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        own[i] = x[4 * lane + i];
        sum += own[i];
      }
      int front = sum;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(front, d);
        if (lane >= d) front += y;
      }
      if (lane == 63) x[kEach * kWaves] = front;
      front -= sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[4 * lane + i] = front;
        front += own[i];
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int before = eq0 + equal[j * kWaves + wave] + __builtin_popcountll(eq[j] & below);
      const bool stays = (gt[j] >> lane & 1) || ((eq[j] >> lane & 1) && before < left);
      if (stays)
        put(a.first + gt0 + heavier[j * kWaves + wave] + __builtin_popcountll(gt[j] & below) + min(before, left),
            a.first + c0 + j * kThreads + tid, v[j]);
    }
    gt0 += heavier[kEach * kWaves];
    eq0 += equal[kEach * kWaves];
    __syncthreads();
  }
}

// The listed tokens into their pages: one workgroup for 64 of them of one head, K (blockIdx.y < H) or V.  Their block's
// scale is the least that holds them, so a code changes only where its own block's scale was finer.  The workgroups of
// K's first head also write the weights' row, the table and the length.  Bound by HBM: 4 x 7664 tokens of 16 heads, D = 128,
// 251 MB read and written: 52 us, 4.8 TB/s (in 8-byte pieces 66).
template <int D>
__global__ __launch_bounds__(256) void keep_gather_kernel(PagePool c, KeepRun a, float* weights, const int2* list,
                                                          const float* kept) {
  constexpr int CODES = D % 16 == 0 ? 16 : 8;  // of a thread's piece
  constexpr int PPR = D / CODES, PIECES = 64 * PPR, ROUNDS = (PIECES + 255) / 256;
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
  float x[ROUNDS][CODES];
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int p = i * 256 + tid, r = p / PPR;
    if (r >= n) continue;
    const int2 from = list[r];
    const long long head = (long long)from.x * c.H + h;
    const uint8_t* src = pages + (head * L + from.y) * D + (p - r * PPR) * CODES;
    const float scale = scales[head * per + from.y / 64];
    if constexpr (CODES == 16) {
      const u32x4 u = *reinterpret_cast<const u32x4*>(src);
      decode8(u32x2{u[0], u[1]}, x[i]);
      decode8(u32x2{u[2], u[3]}, x[i] + 8);
    } else {
      decode8(*reinterpret_cast<const u32x2*>(src), x[i]);
    }
#pragma unroll
    for (int j = 0; j < CODES; ++j) {
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
    if (r >= n) continue;
    uint8_t* to = dst + r * D + (p - r * PPR) * CODES;
    if constexpr (CODES == 16) {
      const u32x2 a = encode8(x[i], inv), b = encode8(x[i] + 8, inv);
      *reinterpret_cast<u32x4*>(to) = u32x4{a[0], a[1], b[0], b[1]};
    } else {
      *reinterpret_cast<u32x2*>(to) = encode8(x[i], inv);
    }
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
