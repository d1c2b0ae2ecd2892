// C ABI of the rotary positions (declared in include/mw.h): bands, argument checks and the kernel launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "mw.h"
#include "mw_host.h"
#include "mw_kernels.h"

using namespace mw;

static_assert(kRopePairs == MW_MAX_ROPE_PAIRS, "the kernel's arguments hold the pairs of every band");

extern "C" {

int mw_rope_bands_init(mw_rope_bands* out, const mw_rope_band* bands, int n_bands, int halves, float gain) {
  const char* fn = "mw_rope_bands_init";
  if (out == nullptr || bands == nullptr) return fail(MW_EINVAL, "%s: a pointer is NULL", fn);
  if (n_bands < 1 || n_bands > MW_MAX_ROPE_BANDS)
    return fail(MW_EINVAL, "%s: %d bands (1 to %d)", fn, n_bands, MW_MAX_ROPE_BANDS);
  if (halves != 0 && halves != 1) return fail(MW_EINVAL, "%s: halves must be 0 or 1", fn);
  if (!std::isfinite(gain) || gain == 0.f) return fail(MW_EINVAL, "%s: gain must be finite and not 0", fn);
  mw_rope_bands r;
  std::memset(&r, 0, sizeof(r));
  r.n_bands = n_bands;
  r.halves = halves;
  r.gain = gain;
  for (int i = 0; i < n_bands; ++i) {
    const mw_rope_band& b = bands[i];
    if (b.dim_offset < 0 || b.dim_offset % 2 || b.dim_count < 2 || b.dim_count % 2 || b.dim_offset > 128 || b.dim_count > 128 ||
        b.dim_offset + b.dim_count > 128)
      return fail(MW_EINVAL, "%s: band %d: dimensions [%d, %d + %d) must be even and within a head of 128", fn, i, b.dim_offset,
                  b.dim_offset, b.dim_count);
    for (int j = 0; j < i; ++j)
      if (b.dim_offset < bands[j].dim_offset + bands[j].dim_count && bands[j].dim_offset < b.dim_offset + b.dim_count)
        return fail(MW_EINVAL, "%s: bands %d and %d share dimensions", fn, j, i);
    if (!(b.theta > 0) || !std::isfinite(b.theta)) return fail(MW_EINVAL, "%s: band %d: theta must be finite and > 0", fn, i);
    if (b.axis < 0 || b.axis >= MW_MAX_ROPE_BANDS) return fail(MW_EINVAL, "%s: band %d: axis %d", fn, i, b.axis);
    if (!(b.factor > 0) || !std::isfinite(b.factor)) return fail(MW_EINVAL, "%s: band %d: factor must be finite and > 0", fn, i);
    const bool ramp = b.turns_hi > b.turns_lo;
    if (!std::isfinite(b.turns_lo) || !std::isfinite(b.turns_hi) || b.turns_hi < b.turns_lo ||
        (ramp && !(b.trained_len > 0 && std::isfinite(b.trained_len))))
      return fail(MW_EINVAL, "%s: band %d: a ramp needs finite turns_lo <= turns_hi and trained_len > 0", fn, i);
    r.dim_offset[i] = b.dim_offset;
    r.dim_count[i] = b.dim_count;
    r.n_axes = std::max(r.n_axes, b.axis + 1);
    for (int p = 0; p < b.dim_count / 2; ++p) {
      double turns = std::pow(b.theta, -2.0 * p / b.dim_count) / (2.0 * M_PI);  // of one position
      double keep = 0.0;
      if (ramp) keep = std::min(1.0, std::max(0.0, (b.trained_len * turns - b.turns_lo) / (b.turns_hi - b.turns_lo)));
      if (b.factor != 1.0) turns *= keep + (1.0 - keep) / b.factor;
      r.freq[r.n_pairs] = turns;
      r.axis[r.n_pairs] = (uint8_t)b.axis;
      r.n_pairs += 1;
    }
  }
  *out = r;
  return ok();
}

int mw_rope_apply(const void* q, const void* k, void* q_out, void* k_out, const mw_rope_bands* bands, const void* positions,
                  int pos_bytes, const mw_strides* pos_strides, int64_t first, int inverse, const mw_strides* strides, int B,
                  int H, int Hkv, int T, int D, mw_stream_t stream) {
  const char* fn = "mw_rope_apply";
  int st = check_ptrs(fn, {{"q", q}, {"q_out", q_out}});
  if (st) return st;
  if ((k == nullptr) != (k_out == nullptr)) return fail(MW_EINVAL, "%s: only one of k and k_out is NULL", fn);
  if (!aligned16(k) || !aligned16(k_out)) return fail(MW_EALIGN, "%s: k or k_out is not 16-byte aligned", fn);
  if (bands == nullptr || bands->n_bands < 1 || bands->n_bands > MW_MAX_ROPE_BANDS || bands->n_pairs < 1 ||
      bands->n_pairs > MW_MAX_ROPE_PAIRS)
    return fail(MW_EINVAL, "%s: bands is NULL or not initialised", fn);
  if (B < 1 || H < 1 || T < 1 || Hkv < (k != nullptr ? 1 : 0))
    return fail(MW_EINVAL, "%s: B, H, T and Hkv (with k) must be >= 1 (got %d, %d, %d, %d)", fn, B, H, T, Hkv);
  if (D != 64 && D != 72 && D != 128)
    return fail(MW_EUNSUPPORTED, "%s: head dimension %d is not supported (64, 72 or 128)", fn, D);
  if (T > kMaxT || (long long)B * T > 0x3fffffff || H > (1 << 14) || Hkv > (1 << 14))
    return fail(MW_EUNSUPPORTED, "%s: B * T, T, H or Hkv is too large", fn);
  if (inverse != 0 && inverse != 1) return fail(MW_EINVAL, "%s: inverse must be 0 or 1", fn);
  if (positions != nullptr) {
    if (pos_bytes != 4 && pos_bytes != 8) return fail(MW_EINVAL, "%s: positions of %d bytes (4 or 8)", fn, pos_bytes);
    if (reinterpret_cast<uintptr_t>(positions) % pos_bytes) return fail(MW_EALIGN, "%s: positions are not aligned", fn);
    if (pos_strides == nullptr) return fail(MW_EINVAL, "%s: pos_strides is NULL", fn);
    if (pos_strides->b < 0 || pos_strides->h < 0 || pos_strides->t < 0)
      return fail(MW_EINVAL, "%s: strides of the positions must be >= 0", fn);
  } else if (bands->n_axes > 1) {
    return fail(MW_EINVAL, "%s: bands of several axes need positions", fn);
  }
  RopeArgs a{};
  int n_pairs = 0;
  bool in[128] = {};
  for (int i = 0; i < bands->n_bands; ++i) {
    const int o = bands->dim_offset[i], n = bands->dim_count[i];
    if (o < 0 || n < 2 || o % 2 || n % 2 || o + n > D)
      return fail(MW_EINVAL, "%s: band %d is not within the head of %d", fn, i, D);
    n_pairs += n / 2;
    std::fill(in + o, in + o + n, true);
  }
  if (n_pairs != bands->n_pairs) return fail(MW_EINVAL, "%s: bands is not initialised", fn);
  const bool with_k = k != nullptr;
  Strides sv[4];
  const char* names[4] = {"q", "k", "q_out", "k_out"};
  for (int i = 0; i < 4; ++i) {
    const int heads = i % 2 ? Hkv : H;
    sv[i] = contiguous(heads, T, D);
    if (strides == nullptr || (i % 2 && !with_k)) continue;
    st = check_view(fn, names[i], strides[i], B, heads, T, D, i >= 2);
    if (st) return st;
    sv[i] = to_internal(strides[i]);
  }
  const auto same = [](const Strides& x, const Strides& y) { return x.b == y.b && x.h == y.h && x.t == y.t; };
  if ((q == q_out && !same(sv[0], sv[2])) || (with_k && k == k_out && !same(sv[1], sv[3])))
    return fail(MW_EINVAL, "%s: an output in its input's place must have its strides", fn);
  const bool in_place = q == q_out && (!with_k || k == k_out);
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.q_out = static_cast<uint16_t*>(q_out);
  a.k_out = static_cast<uint16_t*>(k_out);
  a.sq = sv[0];
  a.sk = sv[1];
  a.sqo = sv[2];
  a.sko = sv[3];
  a.B = B;
  a.heads_q.n = H;
  a.heads_k.n = with_k ? Hkv : 0;
  a.T = T;
  a.pos = positions;
  a.pos64 = pos_bytes == 8;
  if (positions != nullptr) {
    a.pos_axis = pos_strides->h;
    a.pos_b = pos_strides->b;
    a.pos_t = pos_strides->t;
  }
  a.first = first;
  a.gain = bands->gain;
  a.gain_sin = inverse ? -bands->gain : bands->gain;
  a.n_pairs = n_pairs;
  std::copy(bands->freq, bands->freq + n_pairs, a.freq);
  std::copy(bands->axis, bands->axis + n_pairs, a.axis);
  int width = 8;
  if (bands->halves) {
    // the widest pieces that both halves of every band, and what is between the bands, consist of
    for (int i = 0; i < bands->n_bands; ++i)
      while (bands->dim_offset[i] % width || bands->dim_count[i] / 2 % width) width /= 2;
    int pair = 0;
    for (int i = 0; i < bands->n_bands; ++i)
      for (int p = 0; p < bands->dim_count[i] / 2; p += width) {
        a.at_a[a.units] = (uint8_t)(bands->dim_offset[i] + p);
        a.at_b[a.units] = (uint8_t)(bands->dim_offset[i] + bands->dim_count[i] / 2 + p);
        a.pair[a.units++] = (uint8_t)pair;
        pair += width;
      }
    for (int d = 0; d < D && !in_place; d += width)
      if (!in[d]) {
        a.at_a[a.units] = (uint8_t)d;
        a.at_b[a.units++] = kRopeAlone;
      }
  } else {
    a.units = D / 8;
    std::fill(a.pair, a.pair + sizeof(a.pair), (uint8_t)kRopeAlone);
    int pair = 0;
    for (int i = 0; i < bands->n_bands; ++i)
      for (int p = 0; p < bands->dim_count[i] / 2; ++p) a.pair[bands->dim_offset[i] / 2 + p] = (uint8_t)pair++;
  }
  return hip_status(fn, launch_rope(a, bands->halves != 0, width, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
