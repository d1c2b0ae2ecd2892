// Rotary positions of queries and keys (gfx950): y_a = g (x_a cos t - x_b sin t), y_b = g (x_b cos t + x_a sin t) for the
// pairs (a, b) of up to four bands of the head, t the token's position on the band's axis times the pair's frequency.
//
// Bound by HBM: every element is read and written once.  A workgroup takes a few tokens of many heads of both tensors, so
// that an angle is worked out once for all of them: the turns pos * f / 2 pi in 64 bits, their fraction (that step is exact),
// then sine and cosine of it in 32 bits.  The turns are off by a few 2^-53 of themselves (exponent, power, 2 pi, position,
// product), so the angle by |pos| 2^-50 at most (theta >= 1), more than the 2^-22 of 32 bits from |pos| = 2^28 on.
// 19200 tokens of 24 heads of q and k, D = 128, three bands, 236 MB: 44 to 48 us, 4.9 to 5.3 TB/s (a copy of 1 GiB: 5.15;
// 50.5 us with a row's token and head found by divisions, whose instructions kept the vector units busy all the time).
// Eight tokens take 5 us, a launch.
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

__device__ __forceinline__ unsigned quotient(unsigned x, int d, unsigned magic) { return d == 1 ? x : __umulhi(x, magic); }

// A workgroup's rows of q or of k: n_fast * n_slow of (token, head), or (head, token), in steps of so many bytes.
struct Side {
  const char* in;
  char* out;
  int n_fast, n_slow, pitch, rows;
  unsigned magic, in_fast, in_slow, out_fast, out_slow;
  __device__ __forceinline__ Side(const uint16_t* x, uint16_t* y, const Strides& sx, const Strides& sy, const RopeArgs& a,
                                  const RopeArgs::Heads& h, int b, int group, int t0, int n) {
    const int heads = max(0, min(h.per_group, h.n - group * h.per_group)), h0 = max(0, min(group * h.per_group, h.n - 1));
    in = reinterpret_cast<const char*>(x + b * sx.b + h0 * sx.h + t0 * sx.t);
    out = reinterpret_cast<char*>(y + b * sy.b + h0 * sy.h + t0 * sy.t);
    pitch = a.by_head ? a.tokens : h.per_group;
    magic = a.by_head ? a.tokens_magic : h.magic;
    n_fast = a.by_head ? n : heads;
    n_slow = a.by_head ? heads : n;
    rows = heads > 0 ? pitch * n_slow : 0;
    const unsigned ix = 2 * (unsigned)sx.t, ih = 2 * (unsigned)sx.h, ox = 2 * (unsigned)sy.t, oh = 2 * (unsigned)sy.h;
    in_fast = a.by_head ? ix : ih;
    in_slow = a.by_head ? ih : ix;
    out_fast = a.by_head ? ox : oh;
    out_slow = a.by_head ? oh : ox;
  }
};

}  // namespace

// HALVES: a thread's piece is V elements of a band's first half and the V they pair with, or V elements outside the
// bands; else eight consecutive elements, which are four pairs.
template <bool HALVES, int V>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  __shared__ float2 turn[kRopeTableMax];  // [tokens][pairs]
  const int tid = threadIdx.x, block = blockIdx.x / a.groups, group = blockIdx.x - block * a.groups;
  const int b = block / a.blocks, t0 = (block - b * a.blocks) * a.tokens, n = min(a.tokens, a.T - t0);
  const int per_pass = 256 / a.units, unit = tid % a.units, row0 = tid / a.units;
  const bool busy = row0 < per_pass;
  const int at_a = 2 * (HALVES ? a.at_a[unit] : 8 * unit), at_b = HALVES ? 2 * a.at_b[unit] : 0;  // (bytes)
  const bool paired = HALVES && at_b != 2 * kRopeAlone;
  const int pair0 = HALVES ? a.pair[unit] : 4 * unit;
  int pairs[V / 2 + 1];  // (interleaved) of this piece
  if constexpr (!HALVES) {
#pragma unroll
    for (int j = 0; j < V / 2; ++j) pairs[j] = a.pair[pair0 + j];
  }
  const Side q(a.q, a.q_out, a.sq, a.sqo, a, a.heads_q, b, group, t0, n);
  const Side k(a.k, a.k_out, a.sk, a.sko, a, a.heads_k, b, group, t0, n);
  const int rows = q.rows + k.rows;
  constexpr int ROWS = 4;  // rows in flight
  Piece<V> xs[ROWS], ys[ROWS];
  char* out[ROWS];
  int tokens[ROWS];  // -1: no row (the first one is read in its place)
  auto load = [&](int i0) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const int row = i0 + i * per_pass;
      const bool is_k = row >= q.rows && row < rows;
      const unsigned x = row < rows ? row - (is_k ? q.rows : 0) : 0, pitch = is_k ? k.pitch : q.pitch;
      const unsigned slow = pitch == 1 ? x : __umulhi(x, is_k ? k.magic : q.magic), fast = x - slow * pitch;
      const bool in = fast < (unsigned)(is_k ? k.n_fast : q.n_fast) && row < rows;
      tokens[i] = in ? (int)(a.by_head ? fast : slow) : -1;
      const unsigned f = in ? fast : 0, w = in ? slow : 0;
      out[i] = (is_k ? k.out : q.out) + (f * (is_k ? k.out_fast : q.out_fast) + w * (is_k ? k.out_slow : q.out_slow));
      const char* from = (is_k ? k.in : q.in) + (f * (is_k ? k.in_fast : q.in_fast) + w * (is_k ? k.in_slow : q.in_slow));
      xs[i] = *reinterpret_cast<const Piece<V>*>(from + at_a);
      if (paired) ys[i] = *reinterpret_cast<const Piece<V>*>(from + at_b);
    }
  };
  auto rotate = [&] {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      if (tokens[i] < 0) continue;
      const float2* cs = turn + tokens[i] * a.n_pairs;
      char* to = out[i];
      if constexpr (HALVES) {
        if (paired) {
          Piece<V> u, w;
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const float x = (float)xs[i].x[j], y = (float)ys[i].x[j];
            const float2 t = cs[pair0 + j];
            u.x[j] = to_bf16(x * t.x - y * t.y);
            w.x[j] = to_bf16(y * t.x + x * t.y);
          }
          *reinterpret_cast<Piece<V>*>(to + at_a) = u;
          *reinterpret_cast<Piece<V>*>(to + at_b) = w;
        } else {
          *reinterpret_cast<Piece<V>*>(to + at_a) = xs[i];
        }
      } else {
        Piece<V> u = xs[i];
#pragma unroll
        for (int j = 0; j < V / 2; ++j) {
          if (pairs[j] == kRopeAlone) continue;
          const float2 t = cs[pairs[j]];
          const float x = (float)u.x[2 * j], y = (float)u.x[2 * j + 1];
          u.x[2 * j] = to_bf16(x * t.x - y * t.y);
          u.x[2 * j + 1] = to_bf16(y * t.x + x * t.y);
        }
        *reinterpret_cast<Piece<V>*>(to + at_a) = u;
      }
    }
  };
  if (busy) load(row0);  // the first rows are on their way while the angles are worked out
  for (int i = tid; i < n * a.n_pairs; i += 256) {
    const int token = quotient(i, a.n_pairs, a.pairs_magic), j = i - token * a.n_pairs, t = t0 + token;
    long long pos = a.first + t;
    if (a.pos != nullptr) {
      const long long at = a.axis[j] * a.pos_axis + b * a.pos_b + t * a.pos_t;
      pos = a.pos64 ? static_cast<const long long*>(a.pos)[at] : static_cast<const int*>(a.pos)[at];
    }
    const double turns = (double)pos * a.freq[j];
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    turn[i] = make_float2(c * a.gain, s * a.gain_sin);
  }
  __syncthreads();
  if (!busy) return;
  for (int i0 = row0; i0 < rows; i0 += ROWS * per_pass) {
    if (i0 != row0) load(i0);
    rotate();
  }
}

hipError_t launch_rope(RopeArgs a, bool halves, int width, hipStream_t stream) {
  const auto magic = [](int d) { return d == 1 ? 0u : (unsigned)(((1ULL << 32) + d - 1) / d); };
  const int heads = a.heads_q.n + a.heads_k.n, most = std::min({16, a.T, kRopeTableMax / a.n_pairs});
  // A workgroup takes all heads of as many tokens as give each thread its rows in flight.  Where the tokens of a head lie next
  // to each other and rows share cache lines, 16 tokens of as many heads as give a thread 16 pieces: 3 x 4562 tokens, 60
  // heads, D = 72, 85 -> 53 us (rows that are whole lines lose by it: 19200 tokens, 24 heads, D = 128, 51 -> 55).
  a.by_head = a.sq.t < a.sq.h && a.T > 1 && a.sq.t % 64 != 0;
  a.tokens = a.by_head ? most : std::max(1, std::min(most, 1024 / (heads * a.units)));
  a.groups = a.by_head ? std::max(1, heads * a.tokens * a.units / 4096) : 1;
  const auto grid = [&] { return (long long)a.B * ((a.T + a.tokens - 1) / a.tokens) * a.groups; };
  while (a.tokens > 1 && grid() < 1024) --a.tokens;
  // a workgroup's offsets pass no 32 bits (those between 16 tokens never do)
  const auto far = [&](const Strides& s, int n) {
    return std::max(0, (n + a.groups - 1) / a.groups - 1) * s.h + 16 * s.t >= 1LL << 30;
  };
  if (far(a.sq, a.heads_q.n) || far(a.sqo, a.heads_q.n) || far(a.sk, a.heads_k.n) || far(a.sko, a.heads_k.n))
    a.groups = std::max(a.heads_q.n, a.heads_k.n);
  for (RopeArgs::Heads* h : {&a.heads_q, &a.heads_k}) {
    h->per_group = std::max(1, (h->n + a.groups - 1) / a.groups);
    h->magic = magic(h->per_group);
  }
  a.tokens_magic = magic(a.tokens);
  a.pairs_magic = magic(a.n_pairs);
  a.blocks = (a.T + a.tokens - 1) / a.tokens;
  if (grid() > 0x7fffffffLL) return hipErrorInvalidValue;
  const dim3 g((unsigned)grid()), w(256);
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
