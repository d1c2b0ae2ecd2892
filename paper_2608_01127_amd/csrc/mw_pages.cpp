// C ABI of the paged 8-bit cache and of the attention over it (declared in include/mw.h): argument
// checks, page bookkeeping on the host and kernel launches.
//
// Host side of a cache: who owns which page.  Kept in the caller's host block (int32 words):
//   [magic, lowest, n_free, 0] [refs: P] [moved: P] [lens: N] [table: N * W]
// refs[p] counts the table entries that name page p (0: free); lowest is a bound below every free
// page, so that pages are taken lowest first by a scan that starts there; moved is scratch of a
// compaction.  The device's table and lengths are written by the kernels of the operations, in the
// order of the stream.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>

#include "mw.h"
#include "mw_host.h"
#include "mw_kernels.h"

using namespace mw;

static_assert(kMaxSeqs == MW_MAX_SEQS, "the kernels' arguments hold the sequences of a call");

namespace {

struct Book {
  int32_t* head;
  int32_t* refs;
  int32_t* moved;
  int32_t* lens;
  int32_t* table;
};

int32_t magic_of(int P, int N, int W) {
  return (int32_t)(0x6d770000u ^ ((uint32_t)P * 2654435761u) ^ ((uint32_t)N * 40503u) ^ ((uint32_t)W * 69069u));
}

Book book(const mw_kvpages* c) {
  Book b;
  b.head = c->host;
  b.refs = c->host + 4;
  b.moved = b.refs + c->P;
  b.lens = b.moved + c->P;
  b.table = b.lens + c->N;
  return b;
}

int32_t* row_of(const mw_kvpages* c, const Book& b, int seq) { return b.table + (long long)seq * c->W; }
int pages_of(const mw_kvpages* c, int len) { return (len + c->L - 1) / c->L; }

int check_sizes(const char* fn, int P, int H, int L, int D, int N, int W) {
  if (P < 1 || H < 1 || L < 1 || N < 1 || W < 1)
    return fail(MW_EINVAL, "%s: P, H, L, N and W must be >= 1 (got %d, %d, %d, %d, %d)", fn, P, H, L, N, W);
  if (D != 64 && D != 72 && D != 128)
    return fail(MW_EUNSUPPORTED, "%s: head dimension %d is not supported (64, 72 or 128)", fn, D);
  if (L % MW_PAGE_BLOCK) return fail(MW_EINVAL, "%s: L = %d is not a multiple of %d", fn, L, MW_PAGE_BLOCK);
  // (L up to 2^16: block numbers below 2^18 are then divided exactly by the high word of a product)
  if (P > (1 << 24) || N > (1 << 16) || L > (1 << 16) || H > (1 << 14) || (long long)W * L > kMaxT || (long long)N * W > (1LL << 28) ||
      (long long)H * L * D > (1LL << 30) || (long long)P * H * (L / MW_PAGE_BLOCK) > 0x7fffffffLL)
    return fail(MW_EUNSUPPORTED, "%s: P, N, H, L, W * L, N * W, H * L * D or P * H * L is too large", fn);
  return MW_OK;
}

int check_pages(const char* fn, const mw_kvpages* c) {
  if (c == nullptr) return fail(MW_EINVAL, "%s: cache is NULL", fn);
  if (c->host == nullptr || c->k_pages == nullptr || c->v_pages == nullptr || c->k_scales == nullptr ||
      c->v_scales == nullptr || c->table == nullptr || c->lens == nullptr || c->P < 1 || c->N < 1 || c->W < 1 ||
      c->host[0] != magic_of(c->P, c->N, c->W))
    return fail(MW_EINVAL, "%s: cache descriptor is not initialised or is corrupt", fn);
  return check_sizes(fn, c->P, c->H, c->L, c->D, c->N, c->W);
}

int check_seq(const char* fn, const mw_kvpages* c, int seq) {
  if (seq < 0 || seq >= c->N) return fail(MW_EINVAL, "%s: sequence %d is not in [0, %d)", fn, seq, c->N);
  return MW_OK;
}

int check_seqs(const char* fn, const mw_kvpages* c, const int32_t* seqs, int n, bool distinct) {
  if (seqs == nullptr) return fail(MW_EINVAL, "%s: seqs is NULL", fn);
  if (n < 1) return fail(MW_EINVAL, "%s: n_seqs must be >= 1", fn);
  if (n > MW_MAX_SEQS) return fail(MW_EUNSUPPORTED, "%s: %d sequences exceed %d", fn, n, MW_MAX_SEQS);
  for (int i = 0; i < n; ++i) {
    const int st = check_seq(fn, c, seqs[i]);
    if (st) return st;
    for (int j = 0; distinct && j < i; ++j)
      if (seqs[j] == seqs[i]) return fail(MW_EINVAL, "%s: sequence %d is listed twice", fn, seqs[i]);
  }
  return MW_OK;
}

// A recorded operation would run again with the pages and places of its first time, which the books no longer match.
int check_not_captured(const char* fn, mw_stream_t stream) {
  hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(static_cast<hipStream_t>(stream), &status) != hipSuccess) {
    (void)hipGetLastError();  // (the launch reports it)
    return MW_OK;
  }
  if (status != hipStreamCaptureStatusNone)
    return fail(MW_EINVAL, "%s: the stream is being captured into a graph; the call changes host state", fn);
  return MW_OK;
}

PagePool pool_of(const mw_kvpages* c) {
  return {static_cast<uint8_t*>(c->k_pages), static_cast<uint8_t*>(c->v_pages), c->k_scales, c->v_scales, c->table,
          c->lens, c->H, c->L, c->D, c->W};
}

// The lowest free page (there is one: the callers have counted).
int take(const mw_kvpages* c, const Book& b) {
  int p = b.head[1];
  while (p < c->P - 1 && b.refs[p] != 0) ++p;
  b.refs[p] = 1;
  b.head[1] = p + 1;
  b.head[2] -= 1;
  return p;
}

void release(const Book& b, int page) {
  if (--b.refs[page] == 0) {
    b.head[1] = std::min(b.head[1], page);
    b.head[2] += 1;
  }
}

}  // namespace

extern "C" {

size_t mw_kvpages_host_bytes(int P, int N, int W) {
  if (P < 1 || N < 1 || W < 1 || P > (1 << 24) || N > (1 << 16) || (long long)N * W > (1LL << 28)) return 0;
  return sizeof(int32_t) * (4 + 2 * (size_t)P + N + (size_t)N * W);
}

int mw_kvpages_init(mw_kvpages* c, void* k_pages, void* v_pages, float* k_scales, float* v_scales, int32_t* table,
                    int32_t* lens, int32_t* host, size_t host_bytes, int P, int H, int L, int D, int N, int W) {
  const char* fn = "mw_kvpages_init";
  if (c == nullptr) return fail(MW_EINVAL, "%s: cache is NULL", fn);
  if (host == nullptr) return fail(MW_EINVAL, "%s: host is NULL", fn);
  int st = check_ptrs(fn, {{"k_pages", k_pages}, {"v_pages", v_pages}, {"k_scales", k_scales}, {"v_scales", v_scales},
                           {"table", table}, {"lens", lens}});
  if (st) return st;
  st = check_sizes(fn, P, H, L, D, N, W);
  if (st) return st;
  const size_t need = mw_kvpages_host_bytes(P, N, W);
  if (host_bytes < need)
    return fail(MW_EINVAL, "%s: host block of %zu bytes is smaller than the %zu needed", fn, host_bytes, need);
  std::memset(host, 0, need);
  host[0] = magic_of(P, N, W);
  host[2] = P;
  *c = {k_pages, v_pages, k_scales, v_scales, table, lens, host, P, H, L, D, N, W};
  return ok();
}

int mw_kvpages_len(const mw_kvpages* c, int seq) {
  const char* fn = "mw_kvpages_len";
  int st = check_pages(fn, c);
  if (!st) st = check_seq(fn, c, seq);
  return st ? st : book(c).lens[seq];
}

int mw_kvpages_n_free(const mw_kvpages* c) {
  const int st = check_pages("mw_kvpages_n_free", c);
  return st ? st : book(c).head[2];
}

int mw_kvpages_page_of(const mw_kvpages* c, int seq, int index) {
  const char* fn = "mw_kvpages_page_of";
  int st = check_pages(fn, c);
  if (!st) st = check_seq(fn, c, seq);
  if (st) return st;
  const Book b = book(c);
  if (index < 0 || index >= pages_of(c, b.lens[seq]))
    return fail(MW_EINVAL, "%s: sequence %d has no page %d", fn, seq, index);
  return row_of(c, b, seq)[index];
}

int mw_kvpages_append(mw_kvpages* c, const int32_t* seqs, int n_seqs, const void* k, const void* v,
                      const mw_strides* strides, int n_tokens, mw_stream_t stream) {
  const char* fn = "mw_kvpages_append";
  int st = check_pages(fn, c);
  if (!st) st = check_seqs(fn, c, seqs, n_seqs, true);
  if (!st) st = check_ptrs(fn, {{"k", k}, {"v", v}});
  if (!st) st = check_not_captured(fn, stream);
  if (st) return st;
  if (n_tokens < 1) return fail(MW_EINVAL, "%s: n_tokens must be >= 1", fn);
  if (n_tokens > kMaxT) return fail(MW_EUNSUPPORTED, "%s: too many tokens", fn);
  Strides sv[2] = {contiguous(c->H, n_tokens, c->D), contiguous(c->H, n_tokens, c->D)};
  for (int i = 0; strides != nullptr && i < 2; ++i) {
    st = check_view(fn, i ? "v" : "k", strides[i], n_seqs, c->H, n_tokens, c->D, false);
    if (st) return st;
    sv[i] = to_internal(strides[i]);
  }
  const Book b = book(c);
  const int L = c->L;
  long long need = 0;
  for (int i = 0; i < n_seqs; ++i) {
    const int len = b.lens[seqs[i]];
    if ((long long)len + n_tokens > (long long)c->W * L)
      return fail(MW_EFULL, "%s: sequence %d of %d tokens and %d more exceed its row of %d pages", fn, seqs[i], len,
                  n_tokens, c->W);
    const bool shared = len % L != 0 && b.refs[row_of(c, b, seqs[i])[len / L]] > 1;
    need += pages_of(c, len + n_tokens) - pages_of(c, len) + (shared ? 1 : 0);
  }
  if (need > b.head[2])
    return fail(MW_EFULL, "%s: %lld pages are needed and %d are free", fn, need, b.head[2]);
  // A page shared at the start of the call is copied by every listed sequence (not written by the
  // last of them while the others read it), and no reference to it is dropped before all pages
  // are taken.
  int32_t old_page[MW_MAX_SEQS];
  for (int i = 0; i < n_seqs; ++i) {
    const int len = b.lens[seqs[i]];
    const int page = len % L != 0 ? row_of(c, b, seqs[i])[len / L] : -1;
    old_page[i] = page >= 0 && b.refs[page] > 1 ? page : -1;
  }
  AppendArgs a;
  a.n_jobs = 0;
  int n_pages = 0;
  hipError_t e = hipSuccess;
  auto flush = [&]() {
    if (e == hipSuccess && a.n_jobs > 0)
      e = launch_pages_append(pool_of(c), static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v), sv[0], sv[1], a,
                              static_cast<hipStream_t>(stream));
    a.n_jobs = 0;
    n_pages = 0;
  };
  for (int i = 0; i < n_seqs; ++i) {
    const int seq = seqs[i], len = b.lens[seq];
    int32_t* row = row_of(c, b, seq);
    for (int tok = 0; tok < n_tokens;) {  // runs of whole pages of at most the arguments' room
      if (a.n_jobs == kAppendJobs || n_pages == kAppendPages) flush();
      const int j = a.n_jobs++;
      const int pos = len + tok, room = kAppendPages - n_pages;
      const int n = (int)std::min<long long>(n_tokens - tok, (long long)(pos / L + room) * L - pos);
      a.seq[j] = seq;
      a.row[j] = i;
      a.pos[j] = pos;
      a.tok[j] = tok;
      a.n_tok[j] = n;
      a.page0[j] = n_pages;
      a.cow[j] = tok == 0 ? old_page[i] : -1;
      a.len[j] = len + n_tokens;
      for (int w = pos / L; w <= (pos + n - 1) / L; ++w) {
        if (w * L >= pos || a.cow[j] >= 0) row[w] = take(c, b);  // else the page holds older tokens, unshared
        a.pages[n_pages++] = row[w];
      }
      tok += n;
    }
  }
  flush();
  for (int i = 0; i < n_seqs; ++i) {
    const int len = b.lens[seqs[i]];
    int32_t* row = row_of(c, b, seqs[i]);
    if (e == hipSuccess) {
      b.lens[seqs[i]] = len + n_tokens;
      if (old_page[i] >= 0) release(b, old_page[i]);
      continue;
    }
    for (int w = old_page[i] >= 0 ? len / L : pages_of(c, len); w < pages_of(c, len + n_tokens); ++w) release(b, row[w]);
    if (old_page[i] >= 0) row[len / L] = old_page[i];
  }
  return hip_status(fn, e);
}

static int check_empty_pair(const char* fn, const mw_kvpages* c, int src, int dst, mw_stream_t stream) {
  int st = check_pages(fn, c);
  if (!st) st = check_seq(fn, c, src);
  if (!st) st = check_seq(fn, c, dst);
  if (!st) st = check_not_captured(fn, stream);
  if (st) return st;
  if (src == dst) return fail(MW_EINVAL, "%s: source and destination are both sequence %d", fn, src);
  if (book(c).lens[dst] != 0)
    return fail(MW_EINVAL, "%s: sequence %d holds %d tokens; free it first", fn, dst, book(c).lens[dst]);
  return MW_OK;
}

int mw_kvpages_fork(mw_kvpages* c, int src, int dst, mw_stream_t stream) {
  const char* fn = "mw_kvpages_fork";
  const int st = check_empty_pair(fn, c, src, dst, stream);
  if (st) return st;
  const Book b = book(c);
  const int len = b.lens[src], n = pages_of(c, len);
  if (n == 0) return ok();
  const hipError_t e = launch_pages_fork(pool_of(c), src, dst, n, len, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_status(fn, e);
  int32_t *from = row_of(c, b, src), *to = row_of(c, b, dst);
  for (int w = 0; w < n; ++w) {
    to[w] = from[w];
    b.refs[to[w]] += 1;
  }
  b.lens[dst] = len;
  return ok();
}

int mw_kvpages_copy(mw_kvpages* c, int src, int dst, mw_stream_t stream) {
  const char* fn = "mw_kvpages_copy";
  const int st = check_empty_pair(fn, c, src, dst, stream);
  if (st) return st;
  const Book b = book(c);
  const int len = b.lens[src], n = pages_of(c, len);
  if (n == 0) return ok();
  if (n > b.head[2]) return fail(MW_EFULL, "%s: %d pages are needed and %d are free", fn, n, b.head[2]);
  int32_t *from = row_of(c, b, src), *to = row_of(c, b, dst);
  PairArgs a;
  hipError_t e = hipSuccess;
  for (int w0 = 0; w0 < n; w0 += kPagePairs) {
    a.n = std::min(kPagePairs, n - w0);
    for (int i = 0; i < a.n; ++i) {
      to[w0 + i] = take(c, b);
      a.src[i] = from[w0 + i];
      a.dst[i] = to[w0 + i];
    }
    if (e == hipSuccess) e = launch_pages_copy(pool_of(c), a, dst, w0, len, 0, static_cast<hipStream_t>(stream));
  }
  if (e == hipSuccess) {
    b.lens[dst] = len;
  } else {
    for (int w = 0; w < n; ++w) release(b, to[w]);
  }
  return hip_status(fn, e);
}

int mw_kvpages_free(mw_kvpages* c, const int32_t* seqs, int n_seqs, mw_stream_t stream) {
  const char* fn = "mw_kvpages_free";
  int st = check_pages(fn, c);
  if (!st) st = check_seqs(fn, c, seqs, n_seqs, true);
  if (!st) st = check_not_captured(fn, stream);
  if (st) return st;
  const Book b = book(c);
  SeqArgs a;
  a.n = n_seqs;
  std::copy(seqs, seqs + n_seqs, a.seq);
  const hipError_t e = launch_pages_clear(pool_of(c), a, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_status(fn, e);
  for (int i = 0; i < n_seqs; ++i) {
    const int32_t* row = row_of(c, b, seqs[i]);
    for (int w = 0; w < pages_of(c, b.lens[seqs[i]]); ++w) release(b, row[w]);
    b.lens[seqs[i]] = 0;
  }
  return ok();
}

int mw_kvpages_evict(mw_kvpages* c, int seq, int first_page, int n_pages, mw_stream_t stream) {
  const char* fn = "mw_kvpages_evict";
  int st = check_pages(fn, c);
  if (!st) st = check_seq(fn, c, seq);
  if (!st) st = check_not_captured(fn, stream);
  if (st) return st;
  const Book b = book(c);
  const int len = b.lens[seq], used = pages_of(c, len);
  if (first_page < 0 || n_pages < 0) return fail(MW_EINVAL, "%s: first_page and n_pages must be >= 0", fn);
  if ((long long)first_page + n_pages > len / c->L)
    return fail(MW_EEMPTY, "%s: pages [%d, %lld) are not all full: sequence %d has %d full pages", fn, first_page,
                (long long)first_page + n_pages, seq, len / c->L);
  if (n_pages == 0) return ok();
  const int left = len - n_pages * c->L;
  const hipError_t e =
      launch_pages_evict(pool_of(c), seq, first_page, n_pages, used, left, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_status(fn, e);
  int32_t* row = row_of(c, b, seq);
  for (int w = first_page; w < first_page + n_pages; ++w) release(b, row[w]);
  for (int w = first_page + n_pages; w < used; ++w) row[w - n_pages] = row[w];
  b.lens[seq] = left;
  return ok();
}

int mw_kvpages_compact(mw_kvpages* c, mw_stream_t stream) {
  const char* fn = "mw_kvpages_compact";
  int st = check_pages(fn, c);
  if (!st) st = check_not_captured(fn, stream);
  if (st) return st;
  const Book b = book(c);
  const int live = c->P - b.head[2];
  // pages at or above `live` move, in ascending order, to the free ones below it, lowest first
  PairArgs a;
  a.n = 0;
  int moves = 0, dst = 0;
  hipError_t e = hipSuccess;
  auto flush = [&]() {
    if (a.n > 0) e = launch_pages_copy(pool_of(c), a, -1, 0, 0, c->N, static_cast<hipStream_t>(stream));
    for (int i = 0; i < a.n && e == hipSuccess; ++i) {
      b.moved[a.src[i]] = a.dst[i];
      std::swap(b.refs[a.src[i]], b.refs[a.dst[i]]);
      ++moves;
    }
    a.n = 0;
  };
  for (int src = live; src < c->P && e == hipSuccess; ++src) {
    if (b.refs[src] == 0) continue;
    while (b.refs[dst] != 0) ++dst;
    a.src[a.n] = src;
    a.dst[a.n++] = dst++;
    if (a.n == kPagePairs) flush();
  }
  if (e == hipSuccess) flush();
  for (int s = 0; s < c->N && moves > 0; ++s) {
    int32_t* row = row_of(c, b, s);
    for (int w = 0; w < pages_of(c, b.lens[s]); ++w)
      if (row[w] >= live && b.refs[row[w]] == 0) row[w] = b.moved[row[w]];
  }
  if (e != hipSuccess) {
    b.head[1] = 0;
    return hip_status(fn, e);
  }
  b.head[1] = live;
  ok();
  return moves;
}

// ---------------------------------------------------------------------------
// Eviction by accumulated attention weight.
// ---------------------------------------------------------------------------

static int check_weigh(const char* fn, const mw_kvpages* c, const int32_t* seqs, int n_seqs, int H, int T) {
  int st = check_pages(fn, c);
  if (!st) st = check_seqs(fn, c, seqs, n_seqs, true);
  if (st) return st;
  if (H < 1 || H % c->H) return fail(MW_EINVAL, "%s: %d query heads are no multiple of the cache's %d", fn, H, c->H);
  if (H > (1 << 14)) return fail(MW_EUNSUPPORTED, "%s: H too large", fn);
  if (T < 1) return fail(MW_EINVAL, "%s: T must be >= 1", fn);
  if ((long long)T * (H / c->H) > kMaxT) return fail(MW_EUNSUPPORTED, "%s: too many tokens", fn);
  if ((long long)T * H > (1LL << 30)) return fail(MW_EUNSUPPORTED, "%s: T * H is too large", fn);
  return MW_OK;
}

static int weigh_blocks(const mw_kvpages* c, const int32_t* seqs, int n_seqs, WeighSeqs* out) {
  const Book b = book(c);
  long long n = 0;
  for (int i = 0; i < n_seqs; ++i) {
    if (out != nullptr) {
      out->seq[i] = seqs[i];
      out->first[i] = (int)n;
    }
    n += (b.lens[seqs[i]] + MW_PAGE_BLOCK - 1) / MW_PAGE_BLOCK;
  }
  if (out != nullptr) out->first[n_seqs] = (int)n;
  return (int)n;  // at most 256 * 2^24 / 64
}

size_t mw_kvpages_weigh_workspace_size(const mw_kvpages* c, const int32_t* seqs, int n_seqs, int H, int T) {
  if (check_weigh("mw_kvpages_weigh_workspace_size", c, seqs, n_seqs, H, T)) return 0;
  const int n = weigh_blocks(c, seqs, n_seqs, nullptr), parts = weigh_plan(c->H, T * (H / c->H), n, kWeighBytes).parts;
  return parts > 1 ? parts * weigh_part_bytes(n) : 0;
}

int mw_kvpages_weigh(const mw_kvpages* c, const int32_t* seqs, int n_seqs, const void* q, const float* lse, int H, int T,
                     float* weights, int add, float scale, void* workspace, size_t workspace_bytes, const mw_strides* strides,
                     mw_stream_t stream) {
  const char* fn = "mw_kvpages_weigh";
  int st = check_weigh(fn, c, seqs, n_seqs, H, T);
  if (!st) st = check_ptrs(fn, {{"q", q}, {"lse", lse}, {"weights", weights}});
  if (!st) st = check_not_captured(fn, stream);
  if (st) return st;
  if (!aligned16(workspace)) return fail(MW_EALIGN, "%s: workspace is not 16-byte aligned", fn);
  if (add != 0 && add != 1) return fail(MW_EINVAL, "%s: add must be 0 or 1", fn);
  if (!good_scale(scale)) return fail(MW_EINVAL, "%s: scale must be finite and > 0", fn);
  Strides sq = contiguous(H, T, c->D);
  if (strides != nullptr) {
    st = check_view(fn, "q", strides[0], n_seqs, H, T, c->D, false);
    if (st) return st;
    sq = to_internal(strides[0]);
  }
  WeighSeqs s{};
  const int blocks = weigh_blocks(c, seqs, n_seqs, &s);
  WeighParams p{};
  const WeighPlan plan = weigh_plan(c->H, T * (H / c->H), blocks, workspace == nullptr ? 0 : workspace_bytes);
  p.many = plan.many;
  p.n_parts = plan.parts;
  p.q = static_cast<const uint16_t*>(q);
  p.lse = lse;
  const PagePool pool = pool_of(c);
  p.k_pages = pool.k_pages;
  p.k_scales = pool.k_scales;
  p.table = pool.table;
  p.lens = pool.lens;
  p.weights = weights;
  p.part = static_cast<float*>(workspace);
  p.sq = sq;
  p.B = n_seqs;
  p.Hkv = c->H;
  p.G = H / c->H;
  p.T = T;
  p.R = T * p.G;
  p.L = c->L;
  p.W = c->W;
  p.per_page = c->L / MW_PAGE_BLOCK;
  p.add = add != 0;
  p.near = 2.0 * (66.0 * sq.t + (double)p.G * sq.h + c->D) < 4294967296.0;
  p.magic = (unsigned)(((1ULL << 32) + p.G - 1) / p.G);  // (2^32 wraps to 0 at 1, which is not used)
  p.scale_log2 = scale * kLog2e;
  return hip_status(fn, launch_weigh(p, s, c->D, static_cast<hipStream_t>(stream)));
}

// Bytes of the list of places that stay.
static size_t places_bytes(int n_seqs, int n) { return ((size_t)n_seqs * n * sizeof(int2) + 15) / 16 * 16; }

static int check_keep(const char* fn, const mw_kvpages* c, const int32_t* seqs, int n_seqs, int n_keep, int first) {
  int st = check_pages(fn, c);
  if (!st) st = check_seqs(fn, c, seqs, n_seqs, true);
  if (st) return st;
  if (n_keep < 1 || first < 0 || first > n_keep)
    return fail(MW_EINVAL, "%s: n_keep must be >= 1 and first in [0, n_keep] (got %d, %d)", fn, n_keep, first);
  if ((long long)n_keep > (long long)c->W * c->L)
    return fail(MW_EINVAL, "%s: n_keep of %d exceeds a row of %d pages", fn, n_keep, c->W);
  return MW_OK;
}

size_t mw_kvpages_evict_weighted_workspace_size(const mw_kvpages* c, const int32_t* seqs, int n_seqs, int n_keep, int first) {
  if (check_keep("mw_kvpages_evict_weighted_workspace_size", c, seqs, n_seqs, n_keep, first)) return 0;
  const size_t places = (size_t)n_seqs * (n_keep - first / c->L * c->L);
  return std::max<size_t>(16, places_bytes(n_seqs, n_keep - first / c->L * c->L) + places * sizeof(float));
}

int mw_kvpages_evict_weighted(mw_kvpages* c, const int32_t* seqs, int n_seqs, float* weights, int n_keep, int first,
                              int recent, void* workspace, size_t workspace_bytes, mw_stream_t stream) {
  const char* fn = "mw_kvpages_evict_weighted";
  int st = check_keep(fn, c, seqs, n_seqs, n_keep, first);
  if (!st) st = check_ptrs(fn, {{"weights", weights}, {"workspace", workspace}});
  if (!st) st = check_not_captured(fn, stream);
  if (st) return st;
  if (recent < 0 || recent > n_keep - first)
    return fail(MW_EINVAL, "%s: recent = %d is not in [0, n_keep - first]", fn, recent);
  const size_t bytes = mw_kvpages_evict_weighted_workspace_size(c, seqs, n_seqs, n_keep, first);
  if (workspace_bytes < bytes)
    return fail(MW_EINVAL, "%s: workspace of %zu bytes is smaller than the %zu needed", fn, workspace_bytes, bytes);
  const Book b = book(c);
  const int L = c->L, w0 = first / L, w1 = pages_of(c, n_keep), from = w0 * L;
  KeepArgs a{};
  a.keep = n_keep;
  a.first = first;
  a.recent = recent;
  const int per_page = L / MW_PAGE_BLOCK;
  a.per_page_magic = (unsigned)(((1ULL << 32) + per_page - 1) / per_page);  // (2^32 wraps to 0 at 1, which is not used)
  for (int i = 0; i < n_seqs; ++i) {
    if (b.lens[seqs[i]] <= n_keep) continue;  // nothing to drop
    a.seq[a.n_jobs] = seqs[i];
    a.len[a.n_jobs++] = b.lens[seqs[i]];
  }
  if (a.n_jobs == 0) return ok();
  const long long need = (long long)a.n_jobs * (w1 - w0);
  if (need > b.head[2]) return fail(MW_EFULL, "%s: %lld pages are needed and %d are free", fn, need, b.head[2]);
  int2* list = static_cast<int2*>(workspace);
  float* kept = reinterpret_cast<float*>(static_cast<char*>(workspace) + places_bytes(n_seqs, n_keep - from));
  hipStream_t hs = static_cast<hipStream_t>(stream);
  const PagePool pool = pool_of(c);
  hipError_t e = launch_keep_select(pool, a, weights, list, kept, hs);
  if (e != hipSuccess) return hip_status(fn, e);
  // New pages are taken before old ones are given back: no sequence's copy may land on what another one still reads.
  // They are noted in `moved`, which only a compaction uses, until every launch has succeeded.
  KeepRun r;
  r.keep = n_keep;
  r.from = from;
  r.stride = n_keep - from;
  r.n_runs = 0;
  int n_pages = 0;
  auto flush = [&]() {
    if (e == hipSuccess && r.n_runs > 0) e = launch_keep_gather(pool, r, weights, list, kept, hs);
    r.n_runs = 0;
    n_pages = 0;
  };
  int taken = 0;
  for (int j = 0; j < a.n_jobs; ++j) {
    int w = w0;
    do {
      if (r.n_runs == kKeepRuns || n_pages == kKeepPages) flush();
      const int i = r.n_runs++, n = std::min(w1 - w, kKeepPages - n_pages);
      r.seq[i] = a.seq[j];
      r.job[i] = j;
      r.len[i] = a.len[j];
      r.first[i] = w * L;
      r.n_tok[i] = std::min(n_keep, (w + n) * L) - w * L;
      r.page0[i] = n_pages;
      r.last[i] = w + n == w1;
      for (int x = 0; x < n; ++x) {
        const int page = take(c, b);
        b.moved[taken++] = page;
        r.pages[n_pages++] = page;
      }
      w += n;
    } while (w < w1);
  }
  flush();
  if (e != hipSuccess) {
    for (int i = 0; i < taken; ++i) release(b, b.moved[i]);
    return hip_status(fn, e);
  }
  for (int j = 0, at = 0; j < a.n_jobs; ++j) {
    int32_t* row = row_of(c, b, a.seq[j]);
    for (int w = w0; w < pages_of(c, a.len[j]); ++w) release(b, row[w]);
    for (int w = w0; w < w1; ++w) row[w] = b.moved[at++];
    b.lens[a.seq[j]] = n_keep;
  }
  return ok();
}

// ---------------------------------------------------------------------------
// Attention over the pages.
// ---------------------------------------------------------------------------

static int check_paged_call(const char* fn, const mw_kvpages* c, const int32_t* seqs, int n_seqs, int H, int n_queued,
                            int q_len) {
  int st = check_pages(fn, c);
  if (!st) st = check_seqs(fn, c, seqs, n_seqs, false);
  if (st) return st;
  if (H < 1 || H % c->H) return fail(MW_EINVAL, "%s: %d query heads are no multiple of the cache's %d", fn, H, c->H);
  if (H > (1 << 14)) return fail(MW_EUNSUPPORTED, "%s: H too large", fn);
  if (n_queued < 1 || q_len < 1) return fail(MW_EINVAL, "%s: n_queued and q_len must be >= 1", fn);
  if (n_queued > MW_MAX_QUEUED) return fail(MW_EUNSUPPORTED, "%s: n_queued %d exceeds %d", fn, n_queued, MW_MAX_QUEUED);
  if ((long long)n_queued * q_len * (H / c->H) > kMaxT) return fail(MW_EUNSUPPORTED, "%s: too many tokens", fn);
  return MW_OK;
}

// blocks: room for MW_MAX_SEQS; the blocks of 64 cached tokens of each sequence.
static RowsPlan paged_plan(const mw_kvpages* c, const int32_t* seqs, int n_seqs, int H, int tokens, size_t ws_bytes,
                           int* blocks) {
  const Book b = book(c);
  const int R = tokens * (H / c->H);
  int longest = 0;
  for (int i = 0; i < n_seqs; ++i) {
    longest = std::max(longest, b.lens[seqs[i]]);
    blocks[i] = (b.lens[seqs[i]] + MW_PAGE_BLOCK - 1) / MW_PAGE_BLOCK;
  }
  if (R <= kPagesRows) return pages_plan(c->D, R, blocks, n_seqs, c->H, ws_bytes);
  return rows_plan(c->D, true, n_seqs * c->H, R, (long long)longest + tokens, ws_bytes);
}

size_t mw_chunk_attn_paged_workspace_size(const mw_kvpages* c, const int32_t* seqs, int n_seqs, int H, int n_queued,
                                          int q_len) {
  if (check_paged_call("mw_chunk_attn_paged_workspace_size", c, seqs, n_seqs, H, n_queued, q_len)) return 0;
  const int tokens = n_queued * q_len;
  int blocks[MW_MAX_SEQS];
  const RowsPlan plan = paged_plan(c, seqs, n_seqs, H, tokens, (size_t)-1, blocks);
  return rows_part_bytes(c->D, n_seqs * c->H, tokens * (H / c->H), plan.n_splits);
}

int mw_chunk_attn_paged(const void* q, const void* k_new, const void* v_new, int n_queued, int q_len, const mw_kvpages* c,
                        const int32_t* seqs, int n_seqs, int H, int flags, void* o, float* lse, float scale,
                        void* workspace, size_t workspace_bytes, const mw_strides* strides, mw_stream_t stream) {
  const char* fn = "mw_chunk_attn_paged";
  int st = check_paged_call(fn, c, seqs, n_seqs, H, n_queued, q_len);
  if (!st) st = check_ptrs(fn, {{"q", q}, {"o", o}});
  if (st) return st;
  if ((k_new == nullptr) != (v_new == nullptr)) return fail(MW_EINVAL, "%s: only one of k_new and v_new is NULL", fn);
  if (!aligned16(k_new) || !aligned16(v_new)) return fail(MW_EALIGN, "%s: k_new or v_new is not 16-byte aligned", fn);
  if (!aligned16(lse)) return fail(MW_EALIGN, "%s: lse is not 16-byte aligned", fn);
  if (!aligned16(workspace)) return fail(MW_EALIGN, "%s: workspace is not 16-byte aligned", fn);
  if (flags != MW_QUEUED_CAUSAL && flags != MW_QUEUED_ISOLATED) return fail(MW_EINVAL, "%s: unknown flags %d", fn, flags);
  if (!good_scale(scale)) return fail(MW_EINVAL, "%s: scale must be finite and > 0", fn);
  const int T = n_queued * q_len, D = c->D;
  Strides sv[4];
  const char* names[4] = {"q", "k_new", "v_new", "o"};
  for (int i = 0; i < 4; ++i) {
    const int heads = i == 1 || i == 2 ? c->H : H;
    sv[i] = contiguous(heads, T, D);
    if (strides == nullptr || ((i == 1 || i == 2) && k_new == nullptr)) continue;
    st = check_view(fn, names[i], strides[i], n_seqs, heads, T, D, i == 3);
    if (st) return st;
    sv[i] = to_internal(strides[i]);
  }
  RowsParams p{};
  p.q = static_cast<const uint16_t*>(q);
  p.k = static_cast<const uint16_t*>(k_new);
  p.v = static_cast<const uint16_t*>(v_new);
  p.o = static_cast<uint16_t*>(o);
  p.lse = lse;
  p.sq = sv[0];
  p.sk = sv[1];
  p.sv = sv[2];
  p.so = sv[3];
  p.B = n_seqs;
  p.Hkv = c->H;
  p.G = H / c->H;
  p.T = T;
  p.R = T * p.G;
  p.M = k_new != nullptr ? T : 0;
  p.mode = k_new == nullptr ? ROWS_SEE_ALL : (flags == MW_QUEUED_CAUSAL ? ROWS_SEE_EARLIER : ROWS_SEE_OWN);
  p.qlen = q_len;
  p.scale_log2 = scale * kLog2e;
  const PagePool pool = pool_of(c);
  p.k_pages = pool.k_pages;
  p.v_pages = pool.v_pages;
  p.k_scales = pool.k_scales;
  p.v_scales = pool.v_scales;
  p.table = pool.table;
  p.lens = pool.lens;
  p.L = c->L;
  p.W = c->W;
  p.per_page = c->L / MW_PAGE_BLOCK;
  p.per_page_magic = (unsigned)(((1ULL << 32) + p.per_page - 1) / p.per_page);  // (2^32 wraps to 0 at 1, which is not used)
  p.part = static_cast<float*>(workspace);
  int blocks[MW_MAX_SEQS];
  const RowsPlan plan = paged_plan(c, seqs, n_seqs, H, T, workspace != nullptr ? workspace_bytes : 0, blocks);
  hipStream_t hs = static_cast<hipStream_t>(stream);
  return hip_status(fn, D == 64   ? launch_paged_64(p, seqs, blocks, plan, hs)
                        : D == 72 ? launch_paged_72(p, seqs, blocks, plan, hs)
                                  : launch_paged_128(p, seqs, blocks, plan, hs));
}

}  // extern "C"
