// Rotary positions of queries and keys (gfx950): y_a = g (x_a cos t - x_b sin t), y_b = g (x_b cos t + x_a sin t) for the
// pairs (a, b) of up to four bands of the head, t the token's position on the band's axis times the pair's frequency.
//
// Bound by HBM: every element is read and written once.  A workgroup takes a few tokens of all heads of both tensors, so
// that an angle is worked out once for all of them: the turns pos * f / 2 pi in 64 bits, of which the fraction is exact
// for any position, then sine and cosine of it in 32 bits.  19200 tokens of 24 heads of q and k, D = 128, three bands, 236 MB:
// 50.5 us, 4.7 TB/s, of 5.15 that a copy of 1 GiB reaches.  Eight tokens take 5 us, a launch.
#include "mw_device.h"
#include "mw_kernels.h"

namespace mw {

namespace {

// Elements of a thread's accesses: V = 2, 4 or 8 as 32-, 64- or 128-bit words, V = 1 singly.
template <int V>
struct Piece {
  __bf16 x[V];
};
template <>
struct alignas(4) Piece<2> {
  __bf16 x[2];
};
template <>
struct alignas(8) Piece<4> {
  __bf16 x[4];
};
template <>
struct alignas(16) Piece<8> {
  __bf16 x[8];
};

__device__ __forceinline__ long long position(const RopeArgs& a, int axis, int b, int t) {
  if (a.pos == nullptr) return a.first + t;
  const long long i = axis * a.pos_axis + b * a.pos_b + t * a.pos_t;
  return a.pos64 ? static_cast<const long long*>(a.pos)[i] : static_cast<const int*>(a.pos)[i];
}

}  // namespace

// HALVES: a thread's piece is V elements of a band's first half and the V they pair with, or V elements outside the
// bands; else eight consecutive elements, which are four pairs.
template <bool HALVES, int V>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  __shared__ float2 turn[kRopeTableMax];  // [tokens][pairs]
  const int tid = threadIdx.x, n_tokens = a.B * a.T, t0 = blockIdx.x * a.tokens, n = min(a.tokens, n_tokens - t0);
  const int heads = a.H + a.Hkv, rows = n * heads, per_pass = 256 / a.units;
  const int unit = tid % a.units, row0 = tid / a.units;
  const bool busy = row0 < per_pass;
  constexpr int ROWS = 4;  // rows in flight
  struct Row {
    Piece<V> x, y;
    __bf16* out;
    int token;
  } r[ROWS];
  const int at_a = HALVES ? a.at_a[unit] : 8 * unit, at_b = HALVES ? a.at_b[unit] : 0;
  const bool paired = HALVES && at_b != kRopeAlone;
  const int pair0 = HALVES ? a.pair[unit] : 4 * unit;
  int pairs[V / 2 + 1];  // (interleaved) of this piece
  if constexpr (!HALVES) {
#pragma unroll
    for (int j = 0; j < V / 2; ++j) pairs[j] = a.pair[pair0 + j];
  }
  auto load = [&](int i0) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const int row = min(i0 + i * per_pass, rows - 1);
      r[i].token = row / heads;
      const int h = row - r[i].token * heads, token = t0 + r[i].token, b = token / a.T, t = token - b * a.T;
      const bool is_k = h >= a.H;
      const Strides& si = is_k ? a.sk : a.sq;
      const Strides& so = is_k ? a.sko : a.sqo;
      const long long hh = is_k ? h - a.H : h;
      const __bf16* in = reinterpret_cast<const __bf16*>(is_k ? a.k : a.q) + b * si.b + hh * si.h + t * si.t;
      r[i].out = reinterpret_cast<__bf16*>(is_k ? a.k_out : a.q_out) + b * so.b + hh * so.h + t * so.t;
      r[i].x = *reinterpret_cast<const Piece<V>*>(in + at_a);
      if (paired) r[i].y = *reinterpret_cast<const Piece<V>*>(in + at_b);
    }
  };
  if (busy) load(row0);  // the first rows are on their way while the angles are worked out
  for (int i = tid; i < n * a.n_pairs; i += 256) {
    const int token = i / a.n_pairs, j = i - token * a.n_pairs, b = (t0 + token) / a.T, t = t0 + token - b * a.T;
    const double turns = (double)position(a, a.axis[j], b, t) * a.freq[j];
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    turn[i] = make_float2(c * a.gain, s * a.gain_sin);
  }
  __syncthreads();
  if (!busy) return;
  for (int i0 = row0; i0 < rows; i0 += ROWS * per_pass) {
    if (i0 != row0) load(i0);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      if (i0 + i * per_pass >= rows) break;
      if constexpr (HALVES) {
        if (paired) {
          const float2* cs = turn + r[i].token * a.n_pairs + pair0;
          Piece<V> u, w;
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const float x = (float)r[i].x.x[j], y = (float)r[i].y.x[j];
            u.x[j] = to_bf16(x * cs[j].x - y * cs[j].y);
            w.x[j] = to_bf16(y * cs[j].x + x * cs[j].y);
          }
          *reinterpret_cast<Piece<V>*>(r[i].out + at_a) = u;
          *reinterpret_cast<Piece<V>*>(r[i].out + at_b) = w;
        } else {
          *reinterpret_cast<Piece<V>*>(r[i].out + at_a) = r[i].x;
        }
      } else {
        Piece<V> u = r[i].x;
#pragma unroll
        for (int j = 0; j < V / 2; ++j) {
          if (pairs[j] == kRopeAlone) continue;
          const float2 cs = turn[r[i].token * a.n_pairs + pairs[j]];
          const float x = (float)u.x[2 * j], y = (float)u.x[2 * j + 1];
          u.x[2 * j] = to_bf16(x * cs.x - y * cs.y);
          u.x[2 * j + 1] = to_bf16(y * cs.x + x * cs.y);
        }
        *reinterpret_cast<Piece<V>*>(r[i].out + at_a) = u;
      }
    }
  }
}

hipError_t launch_rope(RopeArgs a, bool halves, int width, hipStream_t stream) {
  // as many tokens as give each thread its rows in flight, up to what the table of angles holds
  const long long n_tokens = (long long)a.B * a.T;
  const int pieces = (a.H + a.Hkv) * a.units, most = std::min(16, kRopeTableMax / std::max(1, a.n_pairs));
  a.tokens = std::max(1, std::min(most, 1024 / pieces));
  while (a.tokens > 1 && n_tokens / a.tokens < 1024) --a.tokens;
  const long long grid = (n_tokens + a.tokens - 1) / a.tokens;
  if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
  const dim3 g((unsigned)grid), w(256);
  if (!halves)
    hipLaunchKernelGGL((rope_kernel<false, 8>), g, w, 0, stream, a);
  else if (width == 8)
    hipLaunchKernelGGL((rope_kernel<true, 8>), g, w, 0, stream, a);
  else if (width == 4)
    hipLaunchKernelGGL((rope_kernel<true, 4>), g, w, 0, stream, a);
  else if (width == 2)
    hipLaunchKernelGGL((rope_kernel<true, 2>), g, w, 0, stream, a);
  else
    hipLaunchKernelGGL((rope_kernel<true, 1>), g, w, 0, stream, a);
  return hipGetLastError();
}

}  // namespace mw
