// C ABI of the cross attention (declared in include/mw.h): argument checks and kernel launches.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "mw.h"
#include "mw_host.h"
#include "mw_kernels.h"

using namespace mw;

namespace {

int check_cross(const char* fn, int B, int H, int Hkv, int T, int M, int D) {
  if (B < 1 || H < 1 || Hkv < 1 || T < 1 || M < 1)
    return fail(MW_EINVAL, "%s: B, H, Hkv, T and M must be >= 1 (got %d, %d, %d, %d, %d)", fn, B, H, Hkv, T, M);
  if (H % Hkv) return fail(MW_EINVAL, "%s: %d query heads are no multiple of %d key heads", fn, H, Hkv);
  if (D != 64 && D != 72 && D != 128)
    return fail(MW_EUNSUPPORTED, "%s: head dimension %d is not supported (64, 72 or 128)", fn, D);
  if ((long long)T * (H / Hkv) > kMaxT || M > kMaxT)
    return fail(MW_EUNSUPPORTED, "%s: T * H / Hkv or M exceeds %d", fn, kMaxT);
  if ((long long)B * H > (1LL << 24)) return fail(MW_EUNSUPPORTED, "%s: B*H too large", fn);
  return MW_OK;
}

size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace

extern "C" {

size_t mw_cross_attn_workspace_size(int B, int H, int Hkv, int T, int M, int D) {
  if (check_cross("mw_cross_attn_workspace_size", B, H, Hkv, T, M, D)) return 0;
  const int R = T * (H / Hkv);
  return rows_part_bytes(D, B * Hkv, R, rows_plan(D, false, B * Hkv, R, M, (size_t)-1).n_splits);
}

int mw_cross_attn_fwd(const void* q, const void* k, const void* v, const int32_t* kv_len, void* o, float* lse,
                      const mw_strides* strides, int B, int H, int Hkv, int T, int M, int D, float scale, void* workspace,
                      size_t workspace_bytes, mw_stream_t stream) {
  const char* fn = "mw_cross_attn_fwd";
  int st = check_ptrs(fn, {{"q", q}, {"k", k}, {"v", v}, {"o", o}});
  if (!st) st = check_cross(fn, B, H, Hkv, T, M, D);
  if (st) return st;
  if (!good_scale(scale)) return fail(MW_EINVAL, "%s: scale must be finite and > 0", fn);
  if (!aligned16(kv_len) || !aligned16(lse) || !aligned16(workspace))
    return fail(MW_EALIGN, "%s: kv_len, lse or workspace is not 16-byte aligned", fn);
  Strides sv[4];
  const char* names[4] = {"q", "k", "v", "o"};
  for (int i = 0; i < 4; ++i) {
    const bool key = i == 1 || i == 2;
    sv[i] = contiguous(key ? Hkv : H, key ? M : T, D);
    if (strides == nullptr) continue;
    st = check_view(fn, names[i], strides[i], B, key ? Hkv : H, key ? M : T, D, i == 3);
    if (st) return st;
    sv[i] = to_internal(strides[i]);
  }
  RowsParams p{};
  p.q = static_cast<const uint16_t*>(q);
  p.k = static_cast<const uint16_t*>(k);
  p.v = static_cast<const uint16_t*>(v);
  p.o = static_cast<uint16_t*>(o);
  p.lse = lse;
  p.sq = sv[0];
  p.sk = sv[1];
  p.sv = sv[2];
  p.so = sv[3];
  p.B = B;
  p.Hkv = Hkv;
  p.G = H / Hkv;
  p.T = T;
  p.R = T * p.G;
  p.M = M;
  p.kv_len = kv_len;
  p.mode = ROWS_SEE_ALL;
  p.qlen = 1;
  p.scale_log2 = scale * kLog2e;
  p.part = static_cast<float*>(workspace);
  const RowsPlan plan = rows_plan(D, false, B * Hkv, p.R, M, workspace != nullptr ? workspace_bytes : 0);
  hipStream_t hs = static_cast<hipStream_t>(stream);
  return hip_status(fn, D == 64   ? launch_cross_64(p, plan, hs)
                        : D == 72 ? launch_cross_72(p, plan, hs)
                                  : launch_cross_128(p, plan, hs));
}

// Workspace of the backward: row terms (two fp32 a row), the fp32 dK and dV of the slices, the fp32 dQ of the
// key ranges.
struct CrossBwdLayout {
  CrossBwdPlan plan;
  size_t rows, part, part_q;  // bytes of one row term, of the slices and of the ranges
  CrossBwdLayout(int B, int H, int Hkv, int T, int M, int D) {
    const int R = T * (H / Hkv);
    plan = cross_bwd_plan(D, B * Hkv, R, M);
    rows = round256((size_t)B * H * T * sizeof(float));
    part = plan.n_slices > 1 ? round256((size_t)plan.n_slices * 2 * B * Hkv * M * D * sizeof(float)) : 0;
    part_q = plan.n_ranges > 1 ? round256((size_t)plan.n_ranges * B * H * T * D * sizeof(float)) : 0;
  }
  size_t bytes() const { return 2 * rows + part + part_q; }
};

size_t mw_cross_attn_bwd_workspace_size(int B, int H, int Hkv, int T, int M, int D) {
  if (check_cross("mw_cross_attn_bwd_workspace_size", B, H, Hkv, T, M, D)) return 0;
  return CrossBwdLayout(B, H, Hkv, T, M, D).bytes();
}

int mw_cross_attn_bwd(const void* q, const void* k, const void* v, const int32_t* kv_len, const void* o, const void* d_o,
                      const float* lse, void* dq, void* dk, void* dv, void* workspace, size_t workspace_bytes,
                      const mw_strides* strides, int B, int H, int Hkv, int T, int M, int D, float scale,
                      mw_stream_t stream) {
  const char* fn = "mw_cross_attn_bwd";
  int st = check_ptrs(fn, {{"q", q}, {"k", k}, {"v", v}, {"o", o}, {"d_o", d_o}, {"lse", lse}, {"dq", dq}, {"dk", dk},
                           {"dv", dv}, {"workspace", workspace}});
  if (!st) st = check_cross(fn, B, H, Hkv, T, M, D);
  if (st) return st;
  if (!good_scale(scale)) return fail(MW_EINVAL, "%s: scale must be finite and > 0", fn);
  if (!aligned16(kv_len)) return fail(MW_EALIGN, "%s: kv_len is not 16-byte aligned", fn);
  const CrossBwdLayout lay(B, H, Hkv, T, M, D);
  const size_t need = lay.bytes();
  if (workspace_bytes < need)
    return fail(MW_EINVAL, "%s: workspace of %zu bytes is smaller than the %zu bytes needed", fn, workspace_bytes, need);
  Strides sv[8];
  const char* names[8] = {"q", "k", "v", "o", "d_o", "dq", "dk", "dv"};
  for (int i = 0; i < 8; ++i) {
    const bool key = i == 1 || i == 2 || i >= 6;
    sv[i] = contiguous(key ? Hkv : H, key ? M : T, D);
    if (strides == nullptr) continue;
    st = check_view(fn, names[i], strides[i], B, key ? Hkv : H, key ? M : T, D, i >= 5);
    if (st) return st;
    sv[i] = to_internal(strides[i]);
  }
  CrossBwdParams p{};
  p.q = static_cast<const uint16_t*>(q);
  p.k = static_cast<const uint16_t*>(k);
  p.v = static_cast<const uint16_t*>(v);
  p.o = static_cast<const uint16_t*>(o);
  p.d_o = static_cast<const uint16_t*>(d_o);
  p.lse = lse;
  p.kv_len = kv_len;
  p.dq = static_cast<uint16_t*>(dq);
  p.dk = static_cast<uint16_t*>(dk);
  p.dv = static_cast<uint16_t*>(dv);
  char* ws = static_cast<char*>(workspace);
  p.delta = reinterpret_cast<float*>(ws);
  p.lse2 = reinterpret_cast<float*>(ws + lay.rows);
  p.part = reinterpret_cast<float*>(ws + 2 * lay.rows);
  p.part_q = reinterpret_cast<float*>(ws + 2 * lay.rows + lay.part);
  p.sq = sv[0];
  p.sk = sv[1];
  p.sv = sv[2];
  p.so = sv[3];
  p.sdo = sv[4];
  p.sdq = sv[5];
  p.sdk = sv[6];
  p.sdv = sv[7];
  p.B = B;
  p.Hkv = Hkv;
  p.G = H / Hkv;
  p.T = T;
  p.R = T * p.G;
  p.M = M;
  p.key_waves = lay.plan.key_waves;
  p.n_slices = lay.plan.n_slices;
  p.n_ranges = lay.plan.n_ranges;
  p.scale = scale;
  p.scale_log2 = scale * kLog2e;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  return hip_status(fn, D == 64   ? launch_cross_bwd_64(p, hs)
                        : D == 72 ? launch_cross_bwd_72(p, hs)
                                  : launch_cross_bwd_128(p, hs));
}

}  // extern "C"
