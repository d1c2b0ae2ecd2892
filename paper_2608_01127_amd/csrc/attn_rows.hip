// Cross attention and cached attention over 8-bit pages: launchers of the kernels in
// attn_rows.h.  Compiled once per head dimension (MW_ROWS_HEAD_DIM = 64, 72 or 128) and kind
// (MW_ROWS_PAGED); the plan of a call lives in the D = 128 cross unit.
#include <algorithm>
#include <cmath>

#include "attn_rows.h"

namespace mw {

#define MW_CAT_(a, b) a##b
#define MW_CAT(a, b) MW_CAT_(a, b)
constexpr int kD = MW_ROWS_HEAD_DIM;

namespace {

template <bool PAGES, class Ranges>
hipError_t join_ranges(const RowsParams& p, const Ranges& ranges, hipStream_t stream) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.n_splits == 1) return e;
  const long long threads = (long long)p.B * p.Hkv * p.R * (kD / 4);
  hipLaunchKernelGGL((attn_rows_join_kernel<kD, PAGES>), dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream, p,
                     ranges);
  return hipGetLastError();
}

template <bool PAGED, int NW, int BN, int KG, int WPS>
hipError_t launch_tile(RowsParams p, const RowsSeqs<PAGED>& seqs, const RowsPlan& plan, hipStream_t stream) {
  constexpr int BM = 32 * NW / KG;
  p.n_rtiles = (p.R + BM - 1) / BM;
  p.n_splits = plan.n_splits;
  const long long grid = (long long)p.B * p.Hkv * p.n_rtiles * p.n_splits;
  if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
  hipLaunchKernelGGL((attn_rows_kernel<kD, PAGED, NW, BN, KG, WPS>), dim3((unsigned)grid), dim3(64 * NW), 0, stream, p,
                     seqs);
  return join_ranges<false>(p, 0, stream);
}

#ifdef MW_ROWS_PAGED
// Four waves; up to 32 rows (RB = 1) two stages a wave leave room for two workgroups a CU, whose prologues and ends
// overlap (with four stages and one workgroup: one token of 8 sequences over up to 15840 tokens 27.3 us for 25.2, in two
// rounds 34.8 for 27.5).  RB = 2 is compiled for one: at D = 128 it takes 443 registers and 135 KB of LDS for the join.
template <int RB>
hipError_t launch_pages(RowsParams p, const PageRanges& ranges, const RowsPlan& plan, hipStream_t stream) {
  p.n_splits = plan.n_splits;
  const long long grid = (long long)ranges.first[p.B] * p.Hkv;
  if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
  hipLaunchKernelGGL((attn_pages_kernel<kD, RB, 4, 2>), dim3((unsigned)grid), dim3(256), 0, stream, p, ranges, plan.chunk);
  return join_ranges<true>(p, ranges, stream);
}
#endif

template <bool PAGED>
hipError_t launch_rows(const RowsParams& p, const RowsSeqs<PAGED>& seqs, const RowsPlan& plan, hipStream_t stream) {
  if (plan.bm == 64) return launch_tile<PAGED, 4, 32, 2, 2>(p, seqs, plan, stream);
  // (bf16 keys at D = 72: three waves a SIMD spill five registers, 24 bytes a lane)
  return launch_tile<PAGED, 4, 64, 1, kD == 128 || (kD == 72 && PAGED) ? 2 : 3>(p, seqs, plan, stream);
}

}  // namespace

#ifdef MW_ROWS_PAGED
hipError_t MW_CAT(launch_paged_, MW_ROWS_HEAD_DIM)(const RowsParams& p, const int* seqs, const int* blocks,
                                                   const RowsPlan& plan, hipStream_t stream) {
  if (plan.chunk > 0) {
    PageRanges r{};
    std::copy(seqs, seqs + p.B, r.seq);
    for (int i = 0; i < p.B; ++i) r.first[i + 1] = r.first[i] + std::max(1, (blocks[i] + plan.chunk - 1) / plan.chunk);
    return p.R <= 32 ? launch_pages<1>(p, r, plan, stream) : launch_pages<2>(p, r, plan, stream);
  }
  RowsSeqs<true> s{};
  std::copy(seqs, seqs + p.B, s.seq);
  return launch_rows<true>(p, s, plan, stream);
}
#else
hipError_t MW_CAT(launch_cross_, MW_ROWS_HEAD_DIM)(const RowsParams& p, const RowsPlan& plan, hipStream_t stream) {
  return launch_rows<false>(p, RowsSeqs<false>{}, plan, stream);
}

#if MW_ROWS_HEAD_DIM == 128
size_t rows_part_bytes(int D, int BHkv, int R, int n_splits) {
  return n_splits <= 1 ? 0 : (size_t)n_splits * BHkv * R * (D + 2) * sizeof(float);
}

// attn_pages_kernel's ranges, of `chunk` blocks.  Up to three workgroups a CU without a cut, a call takes about as long as
// the workgroups of the busiest CU (L of them) take to stream their ranges, one after another or side by side, each
// beside its range as long as nine blocks: one token of 8 sequences of up to 248 blocks (4 key heads), us for chunks of
// 8 | 16 | 24 | 32 blocks (L = 3, 2, 2, 1) 31.3 | 27.5 | 30.9 | 25.3; 64 rows of 16 heads over 248 (L = 2, 1, 1, 1)
// 38.7 | 29.2 | 34.0 | 38.7.  With more workgroups the CUs' shares of all blocks even out (a workgroup counts for two
// blocks, eight with more than 32 rows) but for a third of the longest range, until that one streams alone; a cut then
// costs a join, as long as eight blocks, and its partials' transfer, and is made where a tenth is to be had.  One token,
// 16 heads, D = 128: a member of 248 blocks and 63 of 2, uncut 93 us, in ranges of 8 blocks 32; 64 members of 248, uncut
// 680 us, in ranges of 124 down to 4 blocks 688 to 824.  Of 13420 shapes (1 to 256 members, 1 to 64 rows, up to 500
// blocks, equal or ragged) the plans taken are on average 4.4% off the fastest chunk timed, the 99th percentile 29%, the
// worst 67%; with no cut from 1024 workgroups on the worst took 5.4 times as long.
RowsPlan pages_plan(int D, int R, const int* blocks, int n_seqs, int Hkv, size_t ws_bytes) {
  RowsPlan plan{0, 1, 1};
  int longest = 1;
  long long total = 0;
  for (int i = 0; i < n_seqs; ++i) {
    longest = std::max(longest, blocks[i]);
    total += (long long)blocks[i] * Hkv;
  }
  plan.chunk = longest;
  auto count = [&](int chunk) {
    int n = 0;
    for (int i = 0; i < n_seqs; ++i) n += (int)((unsigned)(blocks[i] + chunk - 1) / (unsigned)chunk);
    return (long long)n * Hkv;
  };
  // every member has room for as many partials as the longest one, 1 GiB of them at most
  const size_t partial = rows_part_bytes(D, n_seqs * Hkv, R, 2) / 2, most = std::min(ws_bytes, (size_t)1 << 30) / partial;
  const long long uncut = (count(longest) + 255) / 256;
  const bool many = uncut > 3;
  auto price = [&](int chunk) {
    const long long n = count(chunk);
    if (!many) return (double)((n + 255) / 256) * (chunk + 9);
    const double mb = (double)n * R * (D + 2) * 4e-6;
    const double share = (total + (R <= 32 ? 2.0 : 8.0) * n) / 256;
    return std::max((double)chunk, share + 0.3 * chunk) + 9 + (chunk < longest ? 8 + 0.5 * mb : 0.0);
  };
  double best = (many ? 0.9 : 1.0) * price(longest);
  auto offer = [&](int chunk) {
    const double t = price(chunk);
    if (t >= best) return;
    best = t;
    plan.chunk = chunk;
  };
  bool fits = true;
  int hi = longest;
  for (long long L = uncut; L <= (many ? uncut + 3 : 4); ++L) {
    int lo = 4;  // the smallest chunk of at most 256 L workgroups
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (count(mid) <= 256 * L) {
        hi = mid;
      } else {
        lo = mid + 1;
      }
    }
    if (lo > longest) break;
    hi = lo;
    if ((size_t)((longest + lo - 1) / lo) <= most) {
      offer(lo);
    } else {
      fits = false;
    }
  }
  if (!fits && plan.chunk == longest && most > 1) offer(std::max(4, (int)((longest + most - 1) / most)));
  plan.n_splits = (longest + plan.chunk - 1) / plan.chunk;
  return plan;
}

// attn_rows_kernel's tile (64 rows in two key groups, or 128) and key ranges, by a price for each pair.  A workgroup's
// steps take `lone` us each where it has a CU for itself and `shared` us of the CU where others keep it busy too (L on
// the busiest CU, `occ` of them resident); a round of resident workgroups begins with `round` us; ranges cost the join
// a launch, time for each range, and their fp32 partials a transfer.  The constants are a least-squares fit to
// 2600 (bf16 keys) and 3100 (pages) shapes of 1 to 64 key heads, up to 60000 rows and 16000 keys, each timed with both
// tiles and 1 to 64 ranges: the plans taken are on average 1.4% and 1.3% (at the 90th percentile 6% and 5%) off the fastest.
// (Tiles of 32 and 256 rows, timed in another such run, would have gained 0.1%.)
struct TilePrice {
  double start, round, lone, shared, join, per_mb, per_range;
  int occ;
};
const TilePrice& tile_price(int D, bool paged, int bm) {
  static const TilePrice bf16[3][2] = {
      {{4.38, 2.45, 0.52, 0.365, 1.72, 0.363, 0.088, 4}, {6.04, 0.53, 0.76, 0.57, 1.92, 0.333, 0.081, 3}},   // D = 64
      {{4.56, 2.77, 0.62, 0.413, 1.72, 0.308, 0.089, 3}, {7.32, 0.0, 0.48, 0.87, 2.05, 0.226, 0.073, 3}},    // 72
      {{5.78, 2.36, 0.70, 0.721, 1.71, 0.281, 0.074, 2}, {6.46, 1.03, 1.14, 0.91, 1.85, 0.343, 0.071, 2}}};  // 128
  static const TilePrice pages[3][2] = {
      {{8.71, 0.0, 0.73, 0.436, 1.67, 0.456, 0.070, 4}, {8.88, 0.0, 0.98, 0.636, 2.40, 0.307, 0.070, 3}},
      {{9.63, 0.0, 0.91, 0.583, 1.01, 0.602, 0.065, 3}, {9.44, 0.0, 1.16, 0.81, 2.02, 0.357, 0.069, 2}},
      {{10.05, 0.0, 1.04, 0.729, 1.42, 0.435, 0.062, 2}, {9.77, 0.0, 1.39, 1.01, 2.88, 0.319, 0.055, 2}}};
  return (paged ? pages : bf16)[D == 64 ? 0 : (D == 72 ? 1 : 2)][bm == 64 ? 0 : 1];
}

RowsPlan rows_plan(int D, bool paged, int BHkv, int R, long long keys, size_t ws_bytes) {
  RowsPlan plan{64, 1, 0};
  double best = 1e300;
  const long long steps = std::max(1LL, (keys + 63) / 64);
  for (const int bm : {64, 128}) {
    const TilePrice& c = tile_price(D, paged, bm);
    const long long tiles = (long long)BHkv * ((R + bm - 1) / bm);
    for (long long ns = 1; ns <= std::min(64LL, steps); ++ns) {
      const size_t part = rows_part_bytes(D, BHkv, R, (int)ns);
      if (part > ws_bytes || (ns > 1 && tiles * ns > 8192)) break;
      const double L = (double)((tiles * ns + 255) / 256), k = std::min(L, (double)c.occ);
      const double t = c.start + std::ceil(L / k) * c.round + L / k * ((steps + ns - 1) / ns) * std::max(c.lone, k * c.shared) +
                       (ns > 1 ? c.join + c.per_mb * part * 1e-6 + c.per_range * ns : 0.0);
      if (t < best) {
        best = t;
        plan.bm = bm;
        plan.n_splits = (int)ns;
      }
    }
  }
  return plan;
}
#endif
#endif

}  // namespace mw
