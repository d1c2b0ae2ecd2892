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

hipError_t join_ranges(const RowsParams& p, hipStream_t stream) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.n_splits == 1) return e;
  const long long threads = (long long)p.B * p.Hkv * p.R * (kD / 4);
  hipLaunchKernelGGL(attn_rows_join_kernel<kD>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream, p);
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
  return join_ranges(p, stream);
}

#ifdef MW_ROWS_PAGED
// Four waves; units in flight a wave beside the one it works on: 3.
template <int RB>
hipError_t launch_pages(RowsParams p, const RowsSeqs<true>& seqs, const RowsPlan& plan, hipStream_t stream) {
  p.n_splits = plan.n_splits;
  const long long grid = (long long)p.B * p.Hkv * p.n_splits;
  if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
  hipLaunchKernelGGL((attn_pages_kernel<kD, RB, 4, 4>), dim3((unsigned)grid), dim3(256), 0, stream, p, seqs, plan.chunk);
  return join_ranges(p, stream);
}
#endif

template <bool PAGED>
hipError_t launch_rows(const RowsParams& p, const RowsSeqs<PAGED>& seqs, const RowsPlan& plan, hipStream_t stream) {
  if constexpr (PAGED) {
    if (plan.chunk > 0) return p.R <= 32 ? launch_pages<1>(p, seqs, plan, stream) : launch_pages<2>(p, seqs, plan, stream);
  } else {
    if (plan.bm == 32) return launch_tile<PAGED, 4, 32, 4, 2>(p, seqs, plan, stream);
  }
  if (plan.bm == 64) return launch_tile<PAGED, 4, 32, 2, 2>(p, seqs, plan, stream);
  if (plan.bm == 128) return launch_tile<PAGED, 4, 64, 1, kD == 128 || (kD == 72 && PAGED) ? 2 : 3>(p, seqs, plan, stream);
  return launch_tile<PAGED, 8, 64, 1, 1>(p, seqs, plan, stream);
}

}  // namespace

#ifdef MW_ROWS_PAGED
hipError_t MW_CAT(launch_paged_, MW_ROWS_HEAD_DIM)(const RowsParams& p, const int* seqs, const RowsPlan& plan,
                                                   hipStream_t stream) {
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

RowsPlan rows_plan(int D, bool paged, int BHkv, int R, long long keys, long long all_blocks, size_t ws_bytes) {
  RowsPlan plan{128, 1, 0};
  auto fits = [&](long long ns) { return rows_part_bytes(D, BHkv, R, (int)ns) <= ws_bytes; };
  if (paged && R <= 64) {
    // attn_pages_kernel: ranges of equally many blocks, about one workgroup a CU, at least four blocks each
    plan.bm = R <= 32 ? 32 : 64;
    const long long longest = std::max(1LL, (keys + 63) / 64);
    long long chunk = std::max(4LL, (all_blocks + 255) / 256);
    while ((longest + chunk - 1) / chunk > 1 && !fits((longest + chunk - 1) / chunk)) chunk = chunk * 2;
    plan.chunk = (int)chunk;
    plan.n_splits = (int)((longest + chunk - 1) / chunk);
    return plan;
  }
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
