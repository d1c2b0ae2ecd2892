// Cross attention and cached attention over 8-bit pages: launchers of the kernels in
// attn_rows.h.  Compiled once per head dimension (MW_ROWS_HEAD_DIM = 64, 72 or 128) and kind
// (MW_ROWS_PAGED); the plan of a call lives in the D = 128 cross unit.
#include <algorithm>

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
// Four waves; two stages a wave leave room for two workgroups a CU, whose prologues and ends overlap (with four stages
// and one workgroup: one token of 8 sequences over up to 15840 tokens 28.2 us for 26.2, in two rounds 39 for 31).
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
  if constexpr (!PAGED) {
    if (plan.bm == 32) return launch_tile<PAGED, 4, 32, 4, 2>(p, seqs, plan, stream);
  }
  if (plan.bm == 64) return launch_tile<PAGED, 4, 32, 2, 2>(p, seqs, plan, stream);
  if (plan.bm == 128) return launch_tile<PAGED, 4, 64, 1, kD == 128 || (kD == 72 && PAGED) ? 2 : 3>(p, seqs, plan, stream);
  return launch_tile<PAGED, 8, 64, 1, 1>(p, seqs, plan, stream);
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

// attn_pages_kernel's ranges, of `chunk` blocks.  A call takes about as long as the workgroups of the busiest CU (L of
// them) take to stream their ranges, one after another or side by side, each beside its range as long as nine blocks:
// one token of 8 sequences of up to 248 blocks (4 key heads), us for chunks of 8 | 16 | 24 | 32 blocks (L = 3, 2, 2, 1)
// 31.0 | 27.1 | 31.1 | 26.2; 64 rows of 16 heads over 248 (L = 2, 1, 1, 1) 37.7 | 28.5 | 33.3 | 38.1.
RowsPlan pages_plan(int D, int R, const int* blocks, int n_seqs, int Hkv, size_t ws_bytes) {
  RowsPlan plan{0, 1, 1};
  long long longest = 1;
  for (int i = 0; i < n_seqs; ++i) longest = std::max<long long>(longest, blocks[i]);
  plan.chunk = (int)longest;
  if ((long long)n_seqs * Hkv >= 1024) return plan;  // four workgroups a CU without a cut
  auto count = [&](long long chunk) {
    long long n = 0;
    for (int i = 0; i < n_seqs; ++i) n += (blocks[i] + chunk - 1) / chunk;
    return n * Hkv;
  };
  double best = (double)((count(longest) + 255) / 256) * (longest + 9);
  for (int L = 1; L <= 4; ++L) {
    long long lo = 4, hi = longest;  // the smallest chunk of at most 256 L workgroups
    while (lo < hi) {
      const long long mid = (lo + hi) / 2;
      if (count(mid) <= 256LL * L) {
        hi = mid;
      } else {
        lo = mid + 1;
      }
    }
    const long long ns = (longest + lo - 1) / lo;
    const double cost = (double)((count(lo) + 255) / 256) * (lo + 9);
    if (lo > longest || cost >= best || rows_part_bytes(D, n_seqs * Hkv, R, (int)ns) > ws_bytes) continue;
    best = cost;
    plan.chunk = (int)lo;
  }
  plan.n_splits = (int)((longest + plan.chunk - 1) / plan.chunk);
  return plan;
}

RowsPlan rows_plan(int D, int BHkv, int R, long long keys, size_t ws_bytes) {
  RowsPlan plan{128, 1, 0};
  auto fits = [&](long long ns) { return rows_part_bytes(D, BHkv, R, (int)ns) <= ws_bytes; };
  if (R <= 32) {
    plan.bm = 32;
  } else if (R <= 64 || (long long)BHkv * ((R + 127) / 128) < 256) {
    plan.bm = 64;
  }
  const long long wgs = (long long)BHkv * ((R + plan.bm - 1) / plan.bm);
  const long long steps = (keys + 127) / 128;
  long long ns = std::min({(512 + wgs - 1) / wgs, std::max(1LL, steps / 2), 64LL});
  while (ns > 1 && !fits(ns)) --ns;
  plan.n_splits = (int)std::max(1LL, ns);
  return plan;
}
#endif
#endif

}  // namespace mw
