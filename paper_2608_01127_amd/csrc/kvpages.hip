// Pages of the 8-bit cache with a scale for each 64 tokens and head (gfx950): commit of new
// tokens, copies, and the device side of the page tables.  All of it moves bytes: wide loads and
// stores, and one launch for an operation, whose decisions (pages, places) the host has made and
// passes in the kernel's arguments.
#include "mw_device.h"
#include "mw_kernels.h"

namespace mw {

namespace {

constexpr int kBlock = 64;  // tokens that share a scale

// The scale of a block: 2^e with the least e such that amax <= 448 * 2^e, clamped to [-100, 100].
// A power of two makes the division by it, the product with it and a later change of it exact
// (up to e4m3's subnormals), and costs e4m3, which is a floating-point format, no precision.
__device__ __forceinline__ int block_exponent(float amax) {
  const unsigned u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);  // 448 = 1.75 * 2^8
  return min(max(e, -100), 100);
}
__device__ __forceinline__ float pow2(int e) { return e < -126 ? 0.f : __uint_as_float((unsigned)(e + 127) << 23); }

// +-448 at most; NaN stays NaN.
__device__ __forceinline__ float clamp448(float x) { return x == x ? fminf(fmaxf(x, -448.f), 448.f) : x; }

__device__ __forceinline__ u32x2 encode8(const float (&x)[8], float mul) {
  float y[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) y[j] = clamp448(x[j] * mul);
  u32x2 r;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w], y[4 * w + 1], 0, false);
    r[w] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w + 2], y[4 * w + 3], lo, true);
  }
  return r;
}

}  // namespace

// Commit: one workgroup for a block of 64 tokens of one head, K (blockIdx.y < H) or V.  The block's
// new tokens are read once into registers; with the largest magnitude its scale is known and the
// codes are written.  Tokens that the block holds already keep their codes unless the scale grows
// (then code * 2^(e_old - e) is rounded again) or the page is a copy of a shared one (blocks in
// front of the new tokens are then copied too).  Rows behind the last token are not touched.
// Bound by HBM: 15840 tokens of 16 heads, D = 128 (130 MB in, 65 MB out): 48 us, 4.1 TB/s.
template <int D>
__global__ __launch_bounds__(256) void pages_append_kernel(PagePool c, const uint16_t* __restrict__ kn,
                                                           const uint16_t* __restrict__ vn, Strides sk, Strides sv,
                                                           AppendArgs a) {
  constexpr int PPR = D / 8, PIECES = kBlock * PPR, ROUNDS = (PIECES + 255) / 256;
  const int job = blockIdx.z, tid = threadIdx.x;
  const int pos0 = a.pos[job], n_tok = a.n_tok[job], L = c.L;
  const int page_pos = pos0 / L * L;  // first token of the first page
  const bool cow = a.cow[job] >= 0;
  if (blockIdx.x == 0 && blockIdx.y == 0) {  // the table and the length
    const int n_pages = (pos0 + n_tok - 1) / L - pos0 / L + 1;
    int* row = c.table + (long long)a.seq[job] * c.W + pos0 / L;
    for (int i = tid; i < n_pages; i += 256) row[i] = a.pages[a.page0[job] + i];
    if (tid == 0) c.lens[a.seq[job]] = a.len[job];
  }
  const int at = (cow ? page_pos : pos0 / kBlock * kBlock) + (int)blockIdx.x * kBlock;  // first token of this block
  if (at >= pos0 + n_tok) return;
  const bool is_v = blockIdx.y >= (unsigned)c.H;
  const int h = is_v ? blockIdx.y - c.H : blockIdx.y;
  const int w = at / L - pos0 / L, off = at - at / L * L;
  const int n_old = min(max(pos0 - at, 0), kBlock), n_end = min(pos0 + n_tok - at, kBlock);
  const long long dst_head = (long long)a.pages[a.page0[job] + w] * c.H + h;
  const long long src_head = cow && w == 0 ? (long long)a.cow[job] * c.H + h : dst_head;
  uint8_t* pages = is_v ? c.v_pages : c.k_pages;
  float* scales = is_v ? c.v_scales : c.k_scales;
  const int per = L / kBlock;
  uint8_t* dst = pages + (dst_head * L + off) * D;
  const uint8_t* src = pages + (src_head * L + off) * D;
  float* dst_scale = scales + dst_head * per + off / kBlock;
  const float old_scale = n_old > 0 ? scales[src_head * per + off / kBlock] : 0.f;
  const bool moved = src != dst;
  const Strides s = is_v ? sv : sk;
  const uint16_t* x = (is_v ? vn : kn) + a.row[job] * s.b + h * s.h + (a.tok[job] + (long long)(at - pos0)) * s.t;

  bf16x8 val[ROUNDS];
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int p = i * 256 + tid, row = p / PPR;
    if (row >= n_old && row < n_end) {
      val[i] = *reinterpret_cast<const bf16x8*>(x + row * s.t + (p - row * PPR) * 8);
#pragma unroll
      for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fabsf((float)val[i][j]));  // (a NaN leaves it)
    }
  }
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) amax = fmaxf(amax, __shfl_xor(amax, m));
  __shared__ float wave_max[4];
  if ((tid & 63) == 0) wave_max[tid >> 6] = amax;
  __syncthreads();
  amax = fmaxf(fmaxf(wave_max[0], wave_max[1]), fmaxf(wave_max[2], wave_max[3]));
  const int e_old = n_old > 0 ? (int)(__float_as_uint(old_scale) >> 23) - 127 : -127;
  const int e = n_end > n_old ? max(e_old, block_exponent(amax)) : e_old;
  const float inv = pow2(-e), shift = pow2(e_old - e);
  const bool again = e > e_old;
  if (tid == 0) *dst_scale = pow2(e);
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int p = i * 256 + tid, row = p / PPR, o = row * D + (p - row * PPR) * 8;
    if (row < n_old) {
      if (!moved && !again) continue;
      u32x2 u = *reinterpret_cast<const u32x2*>(src + o);
      if (again) {
        float y[8];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)u[j], false);
          const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)u[j], true);
          y[4 * j] = lo[0];
          y[4 * j + 1] = lo[1];
          y[4 * j + 2] = hi[0];
          y[4 * j + 3] = hi[1];
        }
        u = encode8(y, shift);
      }
      *reinterpret_cast<u32x2*>(dst + o) = u;
    } else if (row < n_end) {
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = (float)val[i][j];
      *reinterpret_cast<u32x2*>(dst + o) = encode8(y, inv);
    }
  }
}

hipError_t launch_pages_append(const PagePool& c, const uint16_t* k, const uint16_t* v, Strides sk, Strides sv,
                               const AppendArgs& a, hipStream_t stream) {
  int blocks = 1;
  for (int j = 0; j < a.n_jobs; ++j) {
    const int from = a.cow[j] >= 0 ? a.pos[j] / c.L * c.L : a.pos[j] / kBlock * kBlock;
    const int n = (a.pos[j] + a.n_tok[j] - from + kBlock - 1) / kBlock;
    blocks = n > blocks ? n : blocks;
  }
  const dim3 grid(blocks, 2 * c.H, a.n_jobs);
  if (c.D == 64)
    hipLaunchKernelGGL(pages_append_kernel<64>, grid, dim3(256), 0, stream, c, k, v, sk, sv, a);
  else if (c.D == 72)
    hipLaunchKernelGGL(pages_append_kernel<72>, grid, dim3(256), 0, stream, c, k, v, sk, sv, a);
  else
    hipLaunchKernelGGL(pages_append_kernel<128>, grid, dim3(256), 0, stream, c, k, v, sk, sv, a);
  return hipGetLastError();
}

// Copy of whole pages: workgroups of 16 KB pieces, pair by pair; the last gridDim.x - n_copy of
// them write the table.  14700 tokens of 12 heads, D = 128 (45 MB each way): 16 us.
__global__ __launch_bounds__(256) void pages_copy_kernel(PagePool c, PairArgs a, int per_pair, int n_copy, int seq, int w0,
                                                         int len, int n_seqs) {
  const int id = blockIdx.x, tid = threadIdx.x;
  if (id < n_copy) {
    const int pair = id / (2 * per_pair), r = id - pair * 2 * per_pair;
    const bool is_v = r >= per_pair;
    const long long piece = is_v ? r - per_pair : r;
    const long long bytes = (long long)c.H * c.L * c.D;
    uint8_t* pages = is_v ? c.v_pages : c.k_pages;
    const u32x4* src = reinterpret_cast<const u32x4*>(pages + a.src[pair] * bytes);
    u32x4* dst = reinterpret_cast<u32x4*>(pages + a.dst[pair] * bytes);
    const long long n16 = bytes / 16;
    u32x4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long long j = piece * 1024 + i * 256 + tid;
      if (j < n16) x[i] = __builtin_nontemporal_load(src + j);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long long j = piece * 1024 + i * 256 + tid;
      if (j < n16) dst[j] = x[i];
    }
    if (piece == 0) {
      float* scales = is_v ? c.v_scales : c.k_scales;
      const int n = c.H * (c.L / kBlock);
      for (int i = tid; i < n; i += 256) scales[(long long)a.dst[pair] * n + i] = scales[(long long)a.src[pair] * n + i];
    }
    return;
  }
  if (seq >= 0) {  // the copies are entries w0.. of row `seq`
    int* row = c.table + (long long)seq * c.W + w0;
    for (int i = tid; i < a.n; i += 256) row[i] = a.dst[i];
    if (tid == 0) c.lens[seq] = len;
    return;
  }
  // the pages have moved: every live entry that names a source names its copy from now on
  const int s = id - n_copy;
  if (s >= n_seqs) return;
  const int used = (c.lens[s] + c.L - 1) / c.L;
  int* row = c.table + (long long)s * c.W;
  for (int i = tid; i < used; i += 256) {
    const int page = row[i];
    int lo = 0, hi = a.n;  // the first source >= page
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (a.src[mid] < page) {
        lo = mid + 1;
      } else {
        hi = mid;
      }
    }
    if (lo < a.n && a.src[lo] == page) row[i] = a.dst[lo];
  }
}

hipError_t launch_pages_copy(const PagePool& c, const PairArgs& a, int seq, int w0, int len, int n_seqs,
                             hipStream_t stream) {
  const long long bytes = (long long)c.H * c.L * c.D;
  const long long per_pair = (bytes + 16383) / 16384;
  const long long n_copy = 2 * per_pair * a.n, grid = n_copy + (seq >= 0 ? 1 : n_seqs);
  if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
  hipLaunchKernelGGL(pages_copy_kernel, dim3((unsigned)grid), dim3(256), 0, stream, c, a, (int)per_pair, (int)n_copy, seq,
                     w0, len, n_seqs);
  return hipGetLastError();
}

__global__ __launch_bounds__(256) void pages_fork_kernel(PagePool c, int src, int dst, int n, int len) {
  const int* from = c.table + (long long)src * c.W;
  int* to = c.table + (long long)dst * c.W;
  for (int i = threadIdx.x; i < n; i += 256) to[i] = from[i];
  if (threadIdx.x == 0) c.lens[dst] = len;
}
hipError_t launch_pages_fork(const PagePool& c, int src, int dst, int n, int len, hipStream_t stream) {
  hipLaunchKernelGGL(pages_fork_kernel, dim3(1), dim3(256), 0, stream, c, src, dst, n, len);
  return hipGetLastError();
}

__global__ __launch_bounds__(256) void pages_clear_kernel(PagePool c, SeqArgs a) {
  if ((int)threadIdx.x < a.n) c.lens[a.seq[threadIdx.x]] = 0;
}
hipError_t launch_pages_clear(const PagePool& c, const SeqArgs& a, hipStream_t stream) {
  static_assert(kMaxSeqs <= 256, "one workgroup");
  hipLaunchKernelGGL(pages_clear_kernel, dim3(1), dim3(256), 0, stream, c, a);
  return hipGetLastError();
}

// One workgroup moves the row's tail forward, 256 entries at a time: each round is read whole before
// it is written, and a later round reads only behind what the earlier ones wrote.
__global__ __launch_bounds__(256) void pages_evict_kernel(PagePool c, int seq, int first, int n, int used, int len) {
  int* row = c.table + (long long)seq * c.W;
  for (int i0 = first; i0 + n < used; i0 += 256) {
    const int i = i0 + threadIdx.x;
    const int page = i + n < used ? row[i + n] : 0;
    __syncthreads();
    if (i + n < used) row[i] = page;
    __syncthreads();
  }
  if (threadIdx.x == 0) c.lens[seq] = len;
}
hipError_t launch_pages_evict(const PagePool& c, int seq, int first, int n, int used, int len, hipStream_t stream) {
  hipLaunchKernelGGL(pages_evict_kernel, dim3(1), dim3(256), 0, stream, c, seq, first, n, used, len);
  return hipGetLastError();
}

}  // namespace mw
