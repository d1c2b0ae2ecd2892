// C ABI of the attention of packed sequences (declared in include/mw.h): argument checks and kernel launches.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "mw.h"
#include "mw_host.h"
#include "mw_kernels.h"

using namespace mw;

namespace {

int check_sizes(const char* fn, int N, int total_q, int total_k, int H, int Hkv, int D, int chunk_len) {
  if (N < 1 || total_q < 1 || total_k < 1 || H < 1 || Hkv < 1 || chunk_len < 1)
    return fail(MW_EINVAL, "%s: N, total_q, total_k, H, Hkv and chunk_len must be >= 1 (got %d, %d, %d, %d, %d, %d)", fn, N,
                total_q, total_k, H, Hkv, chunk_len);
  if (H % Hkv) return fail(MW_EINVAL, "%s: %d query heads are no multiple of %d key heads", fn, H, Hkv);
  if (D != 64 && D != 72 && D != 128)
    return fail(MW_EUNSUPPORTED, "%s: head dimension %d is not supported (64, 72 or 128)", fn, D);
  if (N > (1 << 16) || H > (1 << 14) || (long long)total_q * (H / Hkv) > kMaxT || total_k > kMaxT)
    return fail(MW_EUNSUPPORTED, "%s: N, H, total_q * H / Hkv or total_k is too large", fn);
  return MW_OK;
}

PackedShape shape_of(int N, int total_q, int total_k, int H, int Hkv, int D, int chunk_len, bool backward) {
  return packed_shape(N, H, Hkv, D, std::min(chunk_len, kMaxT), total_q, total_k, backward);
}

PackedShape shape_of(const mw_packed* p) {
  return shape_of(p->N, p->total_q, p->total_k, p->H, p->Hkv, p->D, p->chunk_len, p->backward != 0);
}

size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

int check_packed(const char* fn, const mw_packed* p) {
  if (p == nullptr) return fail(MW_EINVAL, "%s: the packed batch is NULL", fn);
  if (p->plan == nullptr || p->cu_q == nullptr || p->cu_k == nullptr)
    return fail(MW_EINVAL, "%s: the packed batch is not initialised", fn);
  return check_sizes(fn, p->N, p->total_q, p->total_k, p->H, p->Hkv, p->D, p->chunk_len);
}

// Views [total, heads, D] as strides {-, h, t}: of queries, or of keys.
int check_views(const char* fn, const mw_packed* p, const mw_strides* strides, int n, const char* const* names,
                const bool* key, int first_output, Strides* out) {
  for (int i = 0; i < n; ++i) {
    const int heads = key[i] ? p->Hkv : p->H, total = key[i] ? p->total_k : p->total_q;
    out[i] = {0, p->D, (long long)heads * p->D};
    if (strides == nullptr) continue;
    const mw_strides s = {0, strides[i].h, strides[i].t};
    const int st = check_view(fn, names[i], s, 1, heads, total, p->D, i >= first_output);
    if (st) return st;
    out[i] = to_internal(s);
  }
  return MW_OK;
}

// Workspace of the backward: row terms (two fp32 a row), the fp32 parts of cut tiles.
struct BwdLayout {
  size_t rows, part_q, part_k;
  explicit BwdLayout(const PackedShape& s) {
    rows = round256((size_t)s.total_q * s.G * s.Hkv * sizeof(float));
    part_q = round256((size_t)s.dq.max_slots * s.Hkv * s.dq.tile * s.D * sizeof(float));
    part_k = round256((size_t)s.dkv.max_slots * s.Hkv * 2 * s.dkv.tile * s.D * sizeof(float));
  }
  size_t bytes() const { return 2 * rows + part_q + part_k; }
};

}  // namespace

extern "C" {

size_t mw_packed_plan_bytes(int N, int total_q, int total_k, int H, int Hkv, int D, int chunk_len, int backward) {
  if (check_sizes("mw_packed_plan_bytes", N, total_q, total_k, H, Hkv, D, chunk_len)) return 0;
  return sizeof(int32_t) * (size_t)shape_of(N, total_q, total_k, H, Hkv, D, chunk_len, backward != 0).words;
}

int mw_packed_init(mw_packed* p, const int32_t* cu_q, const int32_t* cu_k, int32_t* plan, size_t plan_bytes, int N,
                   int total_q, int total_k, int H, int Hkv, int D, int chunk_len, int backward, mw_stream_t stream) {
  const char* fn = "mw_packed_init";
  if (p == nullptr) return fail(MW_EINVAL, "%s: the packed batch is NULL", fn);
  if (cu_q == nullptr || cu_k == nullptr) return fail(MW_EINVAL, "%s: cu_q or cu_k is NULL", fn);
  int st = check_ptrs(fn, {{"plan", plan}});
  if (st) return st;
  if (reinterpret_cast<uintptr_t>(cu_q) % 4 || reinterpret_cast<uintptr_t>(cu_k) % 4)
    return fail(MW_EALIGN, "%s: cu_q or cu_k is not 4-byte aligned", fn);
  st = check_sizes(fn, N, total_q, total_k, H, Hkv, D, chunk_len);
  if (st) return st;
  const PackedShape s = shape_of(N, total_q, total_k, H, Hkv, D, chunk_len, backward != 0);
  const size_t need = sizeof(int32_t) * (size_t)s.words;
  if (plan_bytes < need) return fail(MW_EINVAL, "%s: plan of %zu bytes is smaller than the %zu needed", fn, plan_bytes, need);
  const hipError_t e = launch_packed_plan(s, cu_q, cu_k, plan, static_cast<hipStream_t>(stream));
  if (e == hipSuccess) *p = {cu_q, cu_k, plan, N, total_q, total_k, H, Hkv, D, chunk_len, backward != 0};
  return hip_status(fn, e);
}

size_t mw_packed_attn_workspace_size(const mw_packed* p) {
  if (check_packed("mw_packed_attn_workspace_size", p)) return 0;
  return packed_part_bytes(shape_of(p));
}

int mw_packed_attn_fwd(const void* q, const void* k, const void* v, const mw_packed* p, void* o, float* lse, float scale,
                       void* workspace, size_t workspace_bytes, const mw_strides* strides, mw_stream_t stream) {
  const char* fn = "mw_packed_attn_fwd";
  int st = check_packed(fn, p);
  if (!st) st = check_ptrs(fn, {{"q", q}, {"k", k}, {"v", v}, {"o", o}, {"lse", lse}});
  if (st) return st;
  if (!good_scale(scale)) return fail(MW_EINVAL, "%s: scale must be finite and > 0", fn);
  if (!aligned16(workspace)) return fail(MW_EALIGN, "%s: workspace is not 16-byte aligned", fn);
  const PackedShape s = shape_of(p);
  const size_t need = packed_part_bytes(s);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need))
    return fail(MW_EINVAL, "%s: workspace of %zu bytes is smaller than the %zu bytes needed", fn,
                workspace == nullptr ? (size_t)0 : workspace_bytes, need);
  Strides sv[4];
  const char* const names[4] = {"q", "k", "v", "o"};
  const bool key[4] = {false, true, true, false};
  st = check_views(fn, p, strides, 4, names, key, 3, sv);
  if (st) return st;
  PackedParams a{};
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.o = static_cast<uint16_t*>(o);
  a.lse = lse;
  a.sq = sv[0];
  a.sk = sv[1];
  a.sv = sv[2];
  a.so = sv[3];
  a.Hkv = p->Hkv;
  a.G = s.G;
  a.L = s.L;
  a.total_q = p->total_q;
  a.list = p->plan + s.fwd.at;
  a.joins = reinterpret_cast<const PackedJoin*>(a.list + 8 + 8LL * s.fwd.max_items);
  a.part = need > 0 ? static_cast<float*>(workspace) : nullptr;
  a.max_slots = s.fwd.max_slots;
  a.scale_log2 = scale * kLog2e;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  return hip_status(fn, p->D == 64   ? launch_packed_fwd_64(a, s.fwd, hs)
                        : p->D == 72 ? launch_packed_fwd_72(a, s.fwd, hs)
                                     : launch_packed_fwd_128(a, s.fwd, hs));
}

size_t mw_packed_attn_bwd_workspace_size(const mw_packed* p) {
  const char* fn = "mw_packed_attn_bwd_workspace_size";
  if (check_packed(fn, p)) return 0;
  if (!p->backward) {
    fail(MW_EINVAL, "%s: the batch was planned without its backward", fn);
    return 0;
  }
  return BwdLayout(shape_of(p)).bytes();
}

int mw_packed_attn_bwd(const void* q, const void* k, const void* v, const void* o, const void* d_o, const float* lse,
                       const mw_packed* p, void* dq, void* dk, void* dv, float scale, void* workspace,
                       size_t workspace_bytes, const mw_strides* strides, mw_stream_t stream) {
  const char* fn = "mw_packed_attn_bwd";
  int st = check_packed(fn, p);
  if (!st) st = check_ptrs(fn, {{"q", q}, {"k", k}, {"v", v}, {"o", o}, {"d_o", d_o}, {"lse", lse}, {"dq", dq}, {"dk", dk},
                                {"dv", dv}, {"workspace", workspace}});
  if (st) return st;
  if (!p->backward) return fail(MW_EINVAL, "%s: the batch was planned without its backward", fn);
  if (!good_scale(scale)) return fail(MW_EINVAL, "%s: scale must be finite and > 0", fn);
  const PackedShape s = shape_of(p);
  const BwdLayout lay(s);
  if (workspace_bytes < lay.bytes())
    return fail(MW_EINVAL, "%s: workspace of %zu bytes is smaller than the %zu bytes needed", fn, workspace_bytes, lay.bytes());
  Strides sv[8];
  const char* const names[8] = {"q", "k", "v", "o", "d_o", "dq", "dk", "dv"};
  const bool key[8] = {false, true, true, false, false, false, true, true};
  st = check_views(fn, p, strides, 8, names, key, 5, sv);
  if (st) return st;
  PackedBwdParams a{};
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.o = static_cast<const uint16_t*>(o);
  a.d_o = static_cast<const uint16_t*>(d_o);
  a.lse = lse;
  a.dq = static_cast<uint16_t*>(dq);
  a.dk = static_cast<uint16_t*>(dk);
  a.dv = static_cast<uint16_t*>(dv);
  char* ws = static_cast<char*>(workspace);
  a.delta = reinterpret_cast<float*>(ws);
  a.lse2 = reinterpret_cast<float*>(ws + lay.rows);
  a.part_q = reinterpret_cast<float*>(ws + 2 * lay.rows);
  a.part_k = reinterpret_cast<float*>(ws + 2 * lay.rows + lay.part_q);
  a.sq = sv[0];
  a.sk = sv[1];
  a.sv = sv[2];
  a.so = sv[3];
  a.sdo = sv[4];
  a.sdq = sv[5];
  a.sdk = sv[6];
  a.sdv = sv[7];
  a.Hkv = p->Hkv;
  a.G = s.G;
  a.L = s.L;
  a.total_q = p->total_q;
  const auto near = [&](const Strides& x) {
    return 2.0 * ((double)(s.dkv.step / s.G + 2) * x.t + (double)s.G * x.h + p->D) < 4294967296.0;
  };
  a.near = near(a.sq) && near(a.sdo);
  a.magic = (unsigned)(((1ULL << 32) + s.G - 1) / s.G);  // (2^32 wraps to 0 at 1, which is not used)
  a.list_q = p->plan + s.dq.at;
  a.list_k = p->plan + s.dkv.at;
  a.joins_q = reinterpret_cast<const PackedJoin*>(a.list_q + 8 + 8LL * s.dq.max_items);
  a.joins_k = reinterpret_cast<const PackedJoin*>(a.list_k + 8 + 8LL * s.dkv.max_items);
  a.scale = scale;
  a.scale_log2 = scale * kLog2e;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  return hip_status(fn, p->D == 64   ? launch_packed_bwd_64(a, s, hs)
                        : p->D == 72 ? launch_packed_bwd_72(a, s, hs)
                                     : launch_packed_bwd_128(a, s, hs));
}

}  // extern "C"
