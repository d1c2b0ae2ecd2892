// Plan of the packed attention (gfx950): which workgroup does what, from the sequences' places in device memory, so
// that a batch is planned without the host's knowing its lengths.
#include <algorithm>

#include "mw_device.h"
#include "mw_kernels.h"

namespace mw {

namespace {

struct PlanArgs {
  const int* cu_q;
  const int* cu_k;
  int* plan;
  long long scratch;  // word of the plan where the lists' scratch begins
  int N, G, Hkv, L, total_q, total_k;
  PackedList list[3];
};

// Sequence s; places that are out of order or out of range give empty or shorter sequences, never a row outside.
struct Sequence {
  int q0, nq, k0, nk;
  __device__ __forceinline__ Sequence(const PlanArgs& a, int s) {
    q0 = min(max(a.cu_q[s], 0), a.total_q);
    nq = min(max(a.cu_q[s + 1], q0), a.total_q) - q0;
    k0 = min(max(a.cu_k[s], 0), a.total_k);
    nk = min(max(a.cu_k[s + 1], k0), a.total_k) - k0;
  }
};

__device__ __forceinline__ int tiles_of(const PackedList& l, const Sequence& s, int G) {
  return ((l.keys ? s.nk : s.nq * G) + l.tile - 1) / l.tile;
}

// Steps [beg, end) of a tile: the keys its last row sees; the rows from the first one that sees its first key.
__device__ __forceinline__ void steps_of(const PackedList& l, const Sequence& s, int tile, int G, int L, int& beg, int& end) {
  beg = end = 0;
  if (l.keys) {
    const int token = max(0, tile * l.tile / L * L - (s.nk - s.nq));
    if (token >= s.nq) return;
    beg = token * G / l.step;
    end = (s.nq * G + l.step - 1) / l.step;
  } else {
    const int place = (min((tile + 1) * l.tile, s.nq * G) - 1) / G + s.nk - s.nq;
    if (place < 0) return;
    end = (min(s.nk, (place / L + 1) * L) + l.step - 1) / l.step;
  }
}

constexpr int kThreads = 1024, kBins = 1024, kCUs = 256;

// Workgroups that tiles are shared out to, two a CU: one that has more than an even share of the steps is cut.  (256, 768,
// 1024: one token of 8 sequences 34.7, 42.5, 43.5 for 33.9 us; the text batch of 8192 tokens, forward and backward, 467, 401,
// 383 for 368 us.)
constexpr int kSlots = 512;

// Sum over the workgroup and everything in front of this thread (exclusive).
__device__ __forceinline__ int block_scan(int x, int* wave_sums, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int in = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(in, d);
    if (lane >= d) in += y;
  }
  __syncthreads();
  if (lane == 63) wave_sums[wave] = in;
  __syncthreads();
  int front = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    const int v = wave_sums[w];
    if (w < wave) front += v;
    total += v;
  }
  return front + in - x;
}

__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

// What an item costs beside its steps, in steps (6: two sequences of 1500 and 1400 tokens, 8 heads, D = 128, forward and
// backward 95.8 for 91.1 us; 9 and 12 between them, 24 as 16).
constexpr int kBegin = 16;

// Length of the items that fewer tiles than kSlots are cut into, from `lo` steps (an even share) to `hi` (no cut).  With no
// more items than places, the longest one decides; with more, two of the first places + 1 items meet in one place.  Each wave
// prices one length from lo to the shortest that leaves no more items than places.
// (Always lo: one token of 8 sequences of up to 15840 keys 42.7 for 34.3 us.  Always the other end, of kSlots places: 8 heads
// of 3471, 2406 and 1997 tokens, D = 64, forward and backward 182 for 147; 4 heads on 1 of 3091, 2664 and 1849, D = 72, 113
// for 105.)
__device__ __forceinline__ int few_tiles_target(const int* tile_steps, int n_tiles, int places, int lo, int hi,
                                                unsigned long long all_steps, int* trial) {
  constexpr int NW = kThreads / 64, PER = kSlots / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, least = lo;
  int n[PER], len[PER], parts[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) n[i] = 64 * i + lane < n_tiles ? tile_steps[64 * i + lane] : -1;
  auto cut = [&](int target) {  // items
    int all = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      parts[i] = n[i] < 0 ? 0 : max(1, (n[i] + target - 1) / target);
      all += parts[i];
    }
    return wave_sum(all);
  };
  int a = lo, b = hi;
  while (a < b) {
    const int mid = a + (int)((long long)(b - a) * wave / NW);
    const int items = cut(mid);
    if (lane == 0) trial[wave] = items;
    __syncthreads();
    int w = 0;
    while (w < NW && trial[w] > places) ++w;
    const int from = a, span = b - a;
    if (w > 0) a = from + (int)((long long)span * (w - 1) / NW) + 1;
    if (w < NW) b = from + (int)((long long)span * w / NW);
    __syncthreads();
  }
  const int target = least + (int)((long long)(b - least) * wave / (NW - 1)), items = cut(target);
  long long cost = target + kBegin;
  if (items > places) {
    // x: the (places + 1)-th longest item
    int x = 0, y = target;
#pragma unroll
    for (int i = 0; i < PER; ++i) len[i] = parts[i] == 0 ? 0 : (n[i] + parts[i] - 1) / parts[i];
    while (x < y) {
      const int mid = x + (y - x) / 2;
      int more = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) more += len[i] > mid ? parts[i] : 0;
      if (wave_sum(more) > places) {
        x = mid + 1;
      } else {
        y = mid;
      }
    }
    cost = max(cost, 2 * ((long long)x + kBegin));
    cost = max(cost, (long long)(all_steps + (long long)items * kBegin) / places);
  }
  if (lane == 0) trial[wave] = (int)min(cost, 0x7fffffffLL);
  __syncthreads();
  int best = 0;
  for (int w = 1; w < NW; ++w)
    if (trial[w] <= trial[best]) best = w;
  return least + (int)((long long)(b - least) * best / (NW - 1));
}

}  // namespace

// One workgroup for each list.  Tiles are numbered sequence after sequence; with all steps known, a tile longer than a
// workgroup's share of them is cut into items of about equal length; the items are put in order of their length, longest
// first, by counting (items of a bin in any order: the order decides when a workgroup runs, not what it computes).
// A chain of short phases in one launch: 16 us for seven sequences of 19200 tokens in all, 16 to 20 with the backward's lists,
// 25 for one token of eight sequences, whose few tiles are priced.  A batch is planned once for all layers.
__global__ __launch_bounds__(kThreads) void packed_plan_kernel(PlanArgs a) {
  __shared__ int wave_sums[kThreads / 64];
  __shared__ int bins[kBins];
  __shared__ unsigned long long all_steps;
  __shared__ int longest, n_slots, n_joins;
  __shared__ int tile_steps[kSlots], trial[kThreads / 64];
  const PackedList l = a.list[blockIdx.x];
  const int tid = threadIdx.x;
  int* head = a.plan + l.at;
  PackedItem* items = reinterpret_cast<PackedItem*>(head + 8);
  PackedJoin* joins = reinterpret_cast<PackedJoin*>(items + l.max_items);
  int* first = a.plan + a.scratch + (long long)blockIdx.x * (a.N + 1);  // first tile of each sequence
  int n_tiles = 0;
  for (int s0 = 0; s0 < a.N; s0 += kThreads) {
    const int s = s0 + tid;
    const int n = s < a.N ? tiles_of(l, Sequence(a, s), a.G) : 0;
    int total;
    // (sequences that overlap, which is no valid input, could have more tiles than there is room for)
    const long long at = (long long)n_tiles + block_scan(min(n, l.max_tiles), wave_sums, total);
    if (s < a.N) first[s] = (int)min(at, (long long)l.max_tiles);
    n_tiles = (int)min((long long)n_tiles + max(total, 0), (long long)l.max_tiles);
  }
  if (tid == 0) {
    first[a.N] = n_tiles;
    all_steps = 0;
    longest = n_slots = n_joins = 0;
  }
  bins[tid] = 0;
  __syncthreads();
  // the sequence of a tile: the last one whose first tile is not behind it
  auto find = [&](int t) {
    int lo = 0, hi = a.N - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (first[mid] <= t) {
        lo = mid;
      } else {
        hi = mid - 1;
      }
    }
    return lo;
  };
  int beg, end;
  {
    unsigned long long sum = 0;
    int most = 0;
    for (int t = tid; t < n_tiles; t += kThreads) {
      const int s = find(t);
      steps_of(l, Sequence(a, s), t - first[s], a.G, a.L, beg, end);
      if (t < kSlots) tile_steps[t] = end - beg;
      sum += end - beg;
      most = max(most, end - beg);
    }
    atomicAdd(&all_steps, sum);
    atomicMax(&longest, most);
  }
  __syncthreads();
  const unsigned long long mean = (all_steps + l.share - 1) / l.share;
  // (twice the mean: the text batch 469 for 387 us)
  int target = (int)min(max(mean, (unsigned long long)l.min_steps), 0x7fffffffULL);
  if (n_tiles < l.share && target < longest)
    target = few_tiles_target(tile_steps, n_tiles, l.places, target, longest, all_steps, trial);
  const int top = min(target, longest);
  auto bin_of = [&](int steps, int parts) { return kBins - 1 - (int)((long long)(steps / parts) * (kBins - 1) / max(top, 1)); };
  for (int t = tid; t < n_tiles; t += kThreads) {
    const int s = find(t);
    steps_of(l, Sequence(a, s), t - first[s], a.G, a.L, beg, end);
    const int parts = max(1, (end - beg + target - 1) / target);
    atomicAdd(&bins[bin_of(end - beg, parts)], parts);
  }
  __syncthreads();
  int all_items;
  const int mine = block_scan(bins[tid], wave_sums, all_items);
  __syncthreads();
  bins[tid] = mine;
  __syncthreads();
  // The first round meets empty CUs, the second the same ones in the same order: turned round, it gives the CU of the
  // longest item the shortest of it (16 heads of 4717 tokens, D = 72, forward and backward 181.5 -> 176.7 us, the 1B clips 1876
  // -> 1860).
  const int round = max(1, kCUs / a.Hkv), n_two = min(2 * round, min(all_items, l.max_items));
  auto place = [&](int x) { return x < round || x >= n_two ? x : round + n_two - 1 - x; };
  for (int t0 = 0; t0 < n_tiles; t0 += kThreads) {
    const int t = t0 + tid;
    if (t < n_tiles) {
      const int s = find(t);
      const Sequence q(a, s);
      const int tile = t - first[s];
      steps_of(l, q, tile, a.G, a.L, beg, end);
      const int n = end - beg, parts = max(1, (n + target - 1) / target);
      const int at = atomicAdd(&bins[bin_of(n, parts)], parts);
      const int slot = parts > 1 ? atomicAdd(&n_slots, parts) : -1;
      if (parts > 1) {
        const int j = atomicAdd(&n_joins, 1);
        if (j < l.max_joins) joins[j] = {q.q0, q.nq, q.k0, q.nk, tile, slot, parts, 0};
      }
      for (int i = 0; i < parts; ++i)
        if (at + i < l.max_items)
          items[place(at + i)] = {q.q0, q.nq, q.k0, q.nk, tile, beg + (int)((long long)n * i / parts),
                           beg + (int)((long long)n * (i + 1) / parts), parts > 1 ? slot + i : -1};
    }
    __syncthreads();  // (earlier tiles take the earlier places of a bin: neighbours stay near each other)
  }
  if (tid == 0) {
    head[0] = min(all_items, l.max_items);
    head[1] = min(n_joins, l.max_joins);
    head[2] = n_slots;
  }
}

namespace {

// Keys (or rows) that an item of a cut tile walks at least.
constexpr int kLeast = 512;

// units: rows (or keys) of all sequences; walked: keys (or rows) that a tile's steps run over at most.
void finish_list(PackedList& l, PackedShape& s, long long units, long long walked, int per_cu) {
  // (the backward's two lists run in one grid: with the forward's share each, 12 heads of 3531 tokens, D = 128, forward and
  // backward 156 for 149 us; with half of it the text batch 411 for 348)
  const int slots = s.n_lists == 0 ? kSlots : kSlots * 3 / 4;
  l.share = std::max(1, slots / s.Hkv);
  l.places = std::max(1, kCUs * per_cu * slots / kSlots / s.Hkv);
  l.max_tiles = (int)std::min<long long>(units / l.tile + s.N, 0x3fffffff);
  // parts = ceil(steps / target), target >= all steps / share: fewer than one for each tile and `share` more; of cut
  // tiles, which have more steps than target, at most twice steps / target
  l.max_items = l.max_tiles + l.share;
  const long long steps = (walked + l.step - 1) / l.step;
  if (walked <= 2 * kLeast) l.min_steps = (int)steps;  // what a cut would save, the join's launch costs
  const long long parts = (steps + l.min_steps - 1) / l.min_steps;
  l.max_slots = parts > 1 ? (int)std::min<long long>(2 * l.share, parts * l.max_tiles) : 0;
  l.max_joins = parts > 1 ? std::min(l.share, l.max_tiles) : 0;
  l.at = s.words;
  s.words += l.words();
  s.n_lists += 1;
}

// Tiles of 64 up to this many of them over all heads, us as (128 | 64): forward, D = 128, 8 heads x 2900 27.3 | 25.1, 16 heads
// on 4 x 1800 21.1 | 18.6, x 19200 402 | 480; D = 64, 16 on 4 x 4000 58.1 | 50.0; forward and backward, dQ and the forward in
// 64, dK/dV as (128 | 64): D = 128, 8 x 2900 97.7 | 90.1, 12 x 3960 197 | 192; D = 64, 12 x 4000 173 | 163, 24 on 8 x 8192 368
// | 384; D = 72, 16 x 4717, all three, 198 | 186.
int packed_small(int D, bool keys) { return D == 128 ? 768 : (D == 72 ? 1400 : (keys ? 768 : 1536)); }

}  // namespace

PackedShape packed_shape(int N, int H, int Hkv, int D, int L, int total_q, int total_k, bool backward) {
  PackedShape s{};
  s.N = N;
  s.G = H / Hkv;
  s.Hkv = Hkv;
  s.D = D;
  s.L = L;
  s.total_q = total_q;
  s.total_k = total_k;
  const long long rows = (long long)total_q * s.G;
  const auto kind = [&](bool keys, long long units) {
    return (units / 64 + N) * Hkv <= packed_small(D, keys) ? PackedTile::pairs : PackedTile::wide;
  };
  const auto add = [&](PackedList& l, bool keys, long long units, long long walked, int per_cu) {
    l.keys = keys;
    l.kind = kind(keys, units);
    l.tile = l.kind == PackedTile::pairs ? 64 : 128;
    l.step = keys ? packed_dkv_step(D, l.kind) : 64;
    l.min_steps = kLeast / l.step;
    finish_list(l, s, units, walked, per_cu);
  };
  add(s.fwd, false, rows, total_k, packed_fwd_per_cu(D, kind(false, rows)));
  if (backward) {
    const int per_cu = packed_bwd_per_cu(D, kind(false, rows), kind(true, total_k));
    add(s.dq, false, rows, total_k, per_cu);
    add(s.dkv, true, total_k, rows, per_cu);
  }
  s.words += (long long)s.n_lists * (N + 1);
  return s;
}

hipError_t launch_packed_plan(const PackedShape& s, const int* cu_q, const int* cu_k, int* plan, hipStream_t stream) {
  PlanArgs a{cu_q, cu_k, plan, s.words - (long long)s.n_lists * (s.N + 1), s.N, s.G, s.Hkv, s.L, s.total_q, s.total_k,
             {s.fwd, s.dq, s.dkv}};
  hipLaunchKernelGGL(packed_plan_kernel, dim3(s.n_lists), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

size_t packed_part_bytes(const PackedShape& s) {
  return (size_t)s.fwd.max_slots * s.Hkv * s.fwd.tile * (s.D + 2) * sizeof(float);
}

}  // namespace mw
