// k_kv.hip -- the paged cache's bookkeeping: block tables and slot maps from
// request lengths, and the store of new keys and values to their slots.
#include "cf_internal.h"

namespace cf {
namespace {

constexpr int kMapThreads = 256;
constexpr int kMapTokens = 2048;  // tokens of a workgroup

struct MapArgs {
  const int32_t *ctx, *nw, *freep, *head;
  int32_t *table;
  int32_t *q_start, *kv_len, *pos, *head_out, *status;
  int64_t *slot;
  int32_t n_seq, page_log2, max_pages, n_free, n_tok;
};

// Sum over the threads before this one; total gets the sum over all of them.
__device__ __forceinline__ int64_t scan_before(int64_t x, int64_t *wave_sum, int64_t &total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int64_t incl = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up(incl, o);
    if (lane >= o) incl += y;
  }
  __syncthreads();
  if (lane == 63) wave_sum[w] = incl;
  __syncthreads();
  int64_t before = incl - x;
  total = 0;
#pragma unroll
  for (int i = 0; i < kMapThreads / 64; i++) {
    if (i < w) before += wave_sum[i];
    total += wave_sum[i];
  }
  return before;
}

// One workgroup per 2048 packed tokens.  Each workgroup scans all the lengths
// itself (they are few next to the tokens, and in L2), so one launch does the
// whole step; workgroup 0 writes the per-request outputs.  A thread owns a run
// of consecutive requests: their new tokens are summed first, then, with each
// request's first token known, the pages it needs.  The requests that own some
// of the workgroup's tokens go to a list in LDS, and each token finds its own
// there by bisection.  A new page's first token enters the page in the table.
// Bound by the latency of its loads and scans: 64 requests 3.3 us, 256 whole prompts
// (428,070 tokens) 9.5 us.
__global__ __launch_bounds__(kMapThreads) void k_kv_map(MapArgs a) {
  __shared__ int64_t wave_sum[kMapThreads / 64];
  __shared__ int32_t l_req[kMapTokens], l_first[kMapTokens], l_page[kMapTokens];
  __shared__ int32_t l_head;
  const int tid = threadIdx.x;
  const int64_t t0 = (int64_t)blockIdx.x * kMapTokens, t1 = min(t0 + kMapTokens, (int64_t)a.n_tok);
  const int64_t P = 1ll << a.page_log2;
  const int64_t row_tokens = min((int64_t)a.max_pages << a.page_log2, (int64_t)INT32_MAX);
  const int per = (a.n_seq + kMapThreads - 1) / kMapThreads;
  const int r0 = min(tid * per, a.n_seq), r1 = min(r0 + per, a.n_seq);
  const int64_t head = max(a.head[0], 0);

  int64_t tok = 0, total;
  for (int r = r0; r < r1; r++) tok += max(a.nw[r], 0);
  const int64_t tok0 = scan_before(tok, wave_sum, total);
  const int64_t all_tok = total;

  // pages needed; high half: requests with tokens in [t0, t1)
  int64_t need = 0;
  int64_t t = tok0;
  auto one = [&](int r, int64_t first, int64_t &nd, int64_t &have, bool &bad) {
    const int64_t c = a.ctx[r], m = a.nw[r];
    bad = c < 0 || m < 0 || c + m > row_tokens || first + m > a.n_tok;  // row_tokens <= INT32_MAX
    have = bad ? 0 : (c + P - 1) >> a.page_log2;
    nd = bad ? 0 : ((c + m + P - 1) >> a.page_log2) - have;
  };
  for (int r = r0; r < r1; r++) {
    int64_t nd, have;
    bool bad;
    one(r, t, nd, have, bad);
    const int64_t m = max(a.nw[r], 0);
    need += nd + ((m > 0 && t < t1 && t + m > t0) ? 1ll << 40 : 0);
    t += m;
  }
  const int64_t s = scan_before(need, wave_sum, total);
  int64_t page_at = head + (s & ((1ll << 40) - 1));
  int at = (int)(s >> 40);
  const int n_list = (int)(total >> 40);
  if (tid == 0) l_head = (int32_t)head;
  __syncthreads();
  int64_t taken = head;
  t = tok0;
  for (int r = r0; r < r1; r++) {
    int64_t nd, have;
    bool bad;
    one(r, t, nd, have, bad);
    const int64_t m = max(a.nw[r], 0);
    const bool none = nd > 0 && page_at + nd > a.n_free;
    if (nd > 0 && !none) taken = page_at + nd;
    if (m > 0 && t < t1 && t + m > t0) {
      l_req[at] = r;
      l_first[at] = (int32_t)(t - t0);  // may be before the workgroup's first token
      l_page[at] = (bad || none) ? -1 : (int32_t)min(page_at, (int64_t)INT32_MAX);
      at++;
    }
    if (blockIdx.x == 0) {
      a.q_start[r] = (int32_t)min(t, (int64_t)INT32_MAX);
      a.status[r] = bad ? CF_KV_TOO_LONG : none ? CF_KV_NO_PAGE : 0;
      a.kv_len[r] = (bad || none) ? 0 : a.ctx[r] + a.nw[r];
    }
    page_at += nd;
    t += m;
  }
  if (blockIdx.x == 0) {
    if (taken > head) atomicMax(&l_head, (int32_t)taken);
    __syncthreads();
    if (tid == 0) {
      a.head_out[0] = l_head;
      a.q_start[a.n_seq] = (int32_t)min(all_tok, (int64_t)INT32_MAX);
    }
  }
  __syncthreads();

  for (int64_t i = t0 + tid; i < t1; i += kMapThreads) {
    const int rel = (int)(i - t0);
    int64_t slot = -1;
    int32_t pos = 0;
    if (i < all_tok && n_list > 0) {
      int lo = 0, hi = n_list;  // the last listed request that starts at or before the token
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (l_first[mid] <= rel) lo = mid; else hi = mid;
      }
      const int r = l_req[lo], p0 = l_page[lo];
      const int64_t c = a.ctx[r];
      const int64_t ps = c + rel - l_first[lo];
      pos = (int32_t)max(min(ps, (int64_t)INT32_MAX), (int64_t)INT32_MIN);
      if (p0 >= 0) {
        const int64_t col = ps >> a.page_log2, have = (c + P - 1) >> a.page_log2;
        int32_t page;
        if (col < have) {
          page = a.table[(int64_t)r * a.max_pages + col];
        } else {
          page = a.freep[p0 + (col - have)];
          if ((ps & (P - 1)) == 0) a.table[(int64_t)r * a.max_pages + col] = page;
        }
        slot = page < 0 ? -1 : ((int64_t)page << a.page_log2) + (ps & (P - 1));
      }
    }
    a.slot[i] = slot;
    a.pos[i] = pos;
  }
}

struct WriteArgs {
  const uint4 *k, *v;
  uint4 *kc, *vc;
  int64_t k_tok, k_head, v_tok, v_head;  // 16-byte chunks
  const int64_t *slot;
  int64_t n_slots;
  int32_t n_tok, Hkv, chunks, page_log2;  // chunks: 16-byte pieces of one head's row
};

// One thread per 16-byte piece of the keys (blockIdx.y 0) or values (1): a copy,
// bound by memory.  Tokens of a page are neighbours in their head's block, so a
// prompt's rows are written in whole lines: 52,808 tokens of 8 x 128 in 74 us, 5.8
// TB/s read and written; 256 tokens 2.8 us.
__global__ __launch_bounds__(256) void k_kv_write(WriteArgs a) {
  const bool is_v = blockIdx.y != 0;
  const uint4 *src = is_v ? a.v : a.k;
  uint4 *dst = is_v ? a.vc : a.kc;
  const int64_t s_tok = is_v ? a.v_tok : a.k_tok, s_head = is_v ? a.v_head : a.k_head;
  const int per_tok = a.Hkv * a.chunks;
  const int64_t n = (int64_t)a.n_tok * per_tok;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t t = i / per_tok;
    const int rest = (int)(i - t * per_tok), h = rest / a.chunks, c = rest - h * a.chunks;
    const int64_t slot = a.slot[t];
    if (slot < 0 || slot >= a.n_slots) continue;
    const int64_t page = slot >> a.page_log2, off = slot & ((1ll << a.page_log2) - 1);
    dst[(((page * a.Hkv + h) << a.page_log2) + off) * a.chunks + c] = src[t * s_tok + h * s_head + c];
  }
}

}  // namespace

// Page sizes of the cache: powers of two, 16 to 256.
bool page_ok(int page) { return page >= 16 && page <= 256 && (page & (page - 1)) == 0; }

cf_status check_cache(const cf_kv_cache *c) {
  if (!c) return set_error(CF_EINVAL, "cache is NULL");
  if (c->n_pages < 0 || c->n_kv_heads < 1 || c->n_kv_heads > 65535)
    return set_error(CF_EINVAL, "cache: n_pages %d, n_kv_heads %d", c->n_pages, c->n_kv_heads);
  if (!page_ok(c->page)) return set_error(CF_EINVAL, "page %d is not a power of two in 16..256", c->page);
  if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8)
    return set_error(CF_EINVAL, "head_dim %d is not a multiple of 8 in 8..256", c->head_dim);
  if (c->dtype != CF_BF16 && c->dtype != CF_F16) return set_error(CF_EINVAL, "dtype %d", c->dtype);
  if (c->n_pages > 0 && (!c->k_dev || !c->v_dev)) return set_error(CF_EINVAL, "NULL cache");
  if (((uintptr_t)c->k_dev | (uintptr_t)c->v_dev) & 15) return set_error(CF_EINVAL, "cache is not 16-byte aligned");
  return CF_OK;
}

}  // namespace cf

extern "C" cf_status cf_kv_map(int32_t n_seq, const int32_t *ctx_len_dev, const int32_t *new_len_dev, int32_t page,
                               int32_t *table_dev, int32_t max_pages, const int32_t *free_dev, int32_t n_free,
                               const int32_t *head_dev, int32_t n_tok, int32_t *q_start_dev, int32_t *kv_len_dev,
                               int64_t *slot_dev, int32_t *pos_dev, int32_t *head_out_dev, int32_t *status_dev,
                               void *stream) {
  using namespace cf;
  if (n_seq < 1 || max_pages < 1 || n_free < 0 || n_tok < 0)
    return set_error(CF_EINVAL, "n_seq %d, max_pages %d, n_free %d, n_tok %d", n_seq, max_pages, n_free, n_tok);
  if (!page_ok(page)) return set_error(CF_EINVAL, "page %d is not a power of two in 16..256", page);
  if (!ctx_len_dev || !new_len_dev || !table_dev || (n_free > 0 && !free_dev) || !head_dev || !q_start_dev ||
      !kv_len_dev || (n_tok > 0 && (!slot_dev || !pos_dev)) || !head_out_dev || !status_dev)
    return set_error(CF_EINVAL, "NULL array");
  if (head_out_dev == head_dev) return set_error(CF_EINVAL, "head_out_dev is head_dev");
  MapArgs a;
  a.ctx = ctx_len_dev; a.nw = new_len_dev; a.freep = free_dev; a.head = head_dev;
  a.table = table_dev; a.q_start = q_start_dev; a.kv_len = kv_len_dev; a.pos = pos_dev;
  a.head_out = head_out_dev; a.status = status_dev; a.slot = slot_dev;
  a.n_seq = n_seq; a.page_log2 = log2_of(page); a.max_pages = max_pages; a.n_free = n_free; a.n_tok = n_tok;
  const int blocks = n_tok > 0 ? (n_tok - 1) / kMapTokens + 1 : 1;
  k_kv_map<<<dim3((unsigned)blocks), dim3(kMapThreads), 0, as_stream(stream)>>>(a);
  return hip_check(hipGetLastError(), "cf_kv_map");
}

extern "C" cf_status cf_kv_write(const cf_kv_cache *cache, int32_t n_tok, const void *k_dev, int64_t k_tok,
                                 int64_t k_head, const void *v_dev, int64_t v_tok, int64_t v_head,
                                 const int64_t *slot_dev, void *stream) {
  using namespace cf;
  const cf_status st = check_cache(cache);
  if (st != CF_OK) return st;
  if (n_tok < 0) return set_error(CF_EINVAL, "n_tok %d", n_tok);
  if (n_tok == 0 || cache->n_pages == 0) return CF_OK;
  if (!k_dev || !v_dev || !slot_dev) return set_error(CF_EINVAL, "NULL array");
  if ((((uintptr_t)k_dev | (uintptr_t)v_dev) & 15) || ((k_tok | k_head | v_tok | v_head) & 7))
    return set_error(CF_EINVAL, "keys and values are not 16-byte aligned");
  WriteArgs a;
  a.k = (const uint4 *)k_dev; a.v = (const uint4 *)v_dev;
  a.kc = (uint4 *)cache->k_dev; a.vc = (uint4 *)cache->v_dev;
  a.k_tok = k_tok / 8; a.k_head = k_head / 8; a.v_tok = v_tok / 8; a.v_head = v_head / 8;
  a.slot = slot_dev;
  a.n_slots = (int64_t)cache->n_pages * cache->page;
  a.n_tok = n_tok; a.Hkv = cache->n_kv_heads; a.chunks = cache->head_dim / 8; a.page_log2 = log2_of(cache->page);
  const int64_t n = (int64_t)n_tok * a.Hkv * a.chunks;
  const int64_t blocks = (n + 255) / 256;
  k_kv_write<<<dim3((unsigned)(blocks < 65536 ? blocks : 65536), 2), dim3(256), 0, as_stream(stream)>>>(a);
  return hip_check(hipGetLastError(), "cf_kv_write");
}
