// k_attn.hip -- attention of new tokens over the paged cache and of whole
// packed sequences: the plan, the few-row and the many-row kernel, the join of
// split contexts.
//
// For a query row q, out = sum_k p_k v_k / sum_k p_k with p_k = exp(scale q.k)
// over the keys it sees, in one pass: with the running maximum m of the
// scores, l = sum exp(s_k - m) and o = sum exp(s_k - m) v_k, a tile of keys
// with a larger maximum m' first scales l and o by exp(m - m').  Exponentials
// are taken in base 2, log2(e) folded into the scale.  Scores, m, l and o are
// fp32; the p_k of a tile are rounded to the element type as the matrix
// instruction's operand, by the output's own rounding: relative error at most
// 2^-8 in bf16; in fp16 2^-11, and for weights below its normal range (2^-29 of
// the largest with few rows, 2^-21 with many) an absolute one of 2^-40 and 2^-32 of the
// largest.  l sums the p_k before that rounding.
//
// A key that a row does not see has p_k = 0, but 0 times an infinity or a NaN
// in its value would still reach the row.  Values past a sequence's keys are
// loaded as zeros; in a tile with a key that some or all of a workgroup's rows
// do not see, such values are zeroed on their way to LDS, and at the end, if there
// were any, added to the rows that see them (which makes those outputs infinite or NaN).
#include "cf_attn.h"

namespace cf {

// Zeros that lanes load in place of keys and values that are not there: 16 rows
// of the widest head, so that a whole page group can be pointed at them.
__device__ i32x4 g_zeros[16 * 256 * 2 / 16];

bool page_ok(int page);
cf_status check_cache(const cf_kv_cache *c);

namespace {

// Partial results pass between workgroups behind different L2s.  They are stored and loaded
// 8 bytes at a time as atomics of device scope, which go past the L2s, and a workgroup says
// that it is done after its stores have arrived: a fence would write back and drop the whole
// L2, keys and values in flight to the other workgroups with it (few-row kernel on 256
// requests: 886 us against 330).
__device__ __forceinline__ void store_part(float *p, float x, float y) {
  __hip_atomic_store((uint64_t *)p, (uint64_t)__float_as_uint(y) << 32 | __float_as_uint(x), __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 load_part(const float *p) {
  const uint64_t u = __hip_atomic_load((uint64_t *)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((uint32_t)u), __uint_as_float((uint32_t)(u >> 32)));
}
__device__ __forceinline__ void parts_arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Weights p_k, and so l and o, are held 2^shift times too large in fp16, whose normal range
// ends at 2^-14: unscaled, weights below 2^-25 of the largest would be lost to o, but not to
// l.  The few-row kernel's largest weight is 1, the many-row kernel's at most 2^8, so the scaled
// ones stay at or below 2^15.  The factor cancels in o / l and costs an addition a tile.
template <typename T>
constexpr float weight_shift(int kind) {
  return __is_same(T, __bf16) ? 0.f : kind ? 7.f : 15.f;
}

// Log of the sum of exponentials from the running maximum and sum, natural.
__device__ __forceinline__ float log_sum(float m, float l, float s2, float shift) {
  return l == 0.f ? kNegInf : (m * s2 + (__log2f(l) - shift)) * 0.69314718055994531f;
}

// Most parts of one context: their weights for a tile's rows are held in LDS.
__host__ __device__ constexpr int max_parts(int kind) { return kind ? 16 : 128; }

__host__ __device__ inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// 16 bytes of global memory (said to the compiler, which else takes the pointer
// for one that may be into LDS, and its loads wait on both counters).
__device__ __forceinline__ i32x4 load16(const void *p) {
  typedef const __attribute__((address_space(1))) i32x4 *gp;
  return *(gp)(uintptr_t)p;
}

// The same without a place in the caches: a decode step reads each layer's keys and values
// once (1.9 GB: 290 us against 320; 131 MB not read before: 28.7 against 30.4; 131 MB read again
// and again, so that the last-level cache holds them: 27.0 against 26.9).
__device__ __forceinline__ i32x4 load16_nt(const void *p) {
  typedef const __attribute__((address_space(1))) i32x4 *gp;
  return __builtin_nontemporal_load((gp)(uintptr_t)p);
}

// Rows in LDS are DS elements (64, 128 or 256), cut into 16-byte chunks that
// are permuted within a row by an exclusive or with a function of the row, so
// that the reads below touch all 64 banks: a key operand reads one chunk of 16
// consecutive rows at once, a value operand 4 rows x 4 chunks (many-row) or 8
// rows x 2 chunks (few-row).
template <int DS>
__device__ __forceinline__ int swz(int row) {
  if (DS == 64) return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
  return ((row & 3) << 2) | ((row >> 2) & 3);
}
template <int DS>
__device__ __forceinline__ int swz8(int row) {
  if (DS == 64) return ((row >> 1) & 3) << 1;
  return (row & 7) << 1;
}

// ------------------------------------------------------------------ plan
// Sums over the block of NS numbers a thread, and maxima of NM.
template <int NT, int NS, int NM>
__device__ __forceinline__ void block_reduce(float (&x)[NS + NM], float (*lds)[8]) {
#pragma unroll
  for (int o = 32; o; o >>= 1)
#pragma unroll
    for (int i = 0; i < NS + NM; i++) {
      const float y = __shfl_xor(x[i], o);
      x[i] = i < NS ? x[i] + y : fmaxf(x[i], y);
    }
  __syncthreads();
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int i = 0; i < NS + NM; i++) lds[threadIdx.x >> 6][i] = x[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NS + NM; i++) {
    x[i] = lds[0][i];
#pragma unroll
    for (int w = 1; w < NT / 64; w++) x[i] = i < NS ? x[i] + lds[w][i] : fmaxf(x[i], lds[w][i]);
  }
}

// How the contexts of one kernel's requests are split.  n workgroups run at a time per
// key/value head; the candidates are no split, and one and two parts for each of them.  A
// candidate's time is estimated in keys: its parts in full rounds, or their sum over the
// workgroups and half a part of tail, whichever is less, and `cost` keys for starting a
// part and joining its result.
struct Split {
  int n, cost, max_parts;
};

// One workgroup.  Pass 1 sums the work of either kernel, (row tiles) x (keys), and the
// parts that each candidate length gives; pass 2 takes NT requests at a time, places their
// items by a scan and writes them, a thread per item.  Bound by the latency of its few
// steps (16 to 256 requests: 6 us; with 64-bit divisions and a scan for each count 17), so that 256 threads do better than 1024 as long as
// one step takes all requests.
template <int NT>
__global__ __launch_bounds__(NT) void k_attn_plan(PlanView v, const int32_t *q_start, const int32_t *kv_len, int n_seq,
                                                  int n_tok, int G, int Hkv, int few_only, int big_log2, Split sp0,
                                                  Split sp1) {
  __shared__ float red[NT / 64][8];
  __shared__ int64_t red64[NT / 64];
  __shared__ int64_t l_at[NT];
  __shared__ int l_n[NT], l_rows[NT][3];
  const int tid = threadIdx.x;
  int q0 = 0, nq = 0, nk = 0;  // of the request loaded last
  auto load = [&](int i, int &tiles, int &kind, int &keys) {
    q0 = clampi(q_start[i], 0, n_tok);
    nq = max(clampi(q_start[i + 1], 0, n_tok) - q0, 0);
    nk = max(kv_len[i], 0);
    const int rows = nq * G;
    kind = (!few_only && rows > kRowsSmall) ? 1 : 0;
    const int sh = kind ? big_log2 : 4;
    tiles = (rows + (1 << sh) - 1) >> sh;
    keys = min(nk, 1 << 29);  // the last part of a context has no end
  };
  int tiles0 = 0, kind0 = 0, keys0 = 0;  // the thread's first request, kept for the later passes
  if (tid < n_seq) load(tid, tiles0, kind0, keys0);
  const int first_q0 = q0, first_nq = nq, first_nk = nk;
  // the counters of finished parts start at zero
  for (int k = 0; k < 2; k++)
    for (int i = tid; i < v.cap_join[k] * Hkv; i += NT) v.done[k][i] = 0;
  float w[4] = {0.f, 0.f, 0.f, 0.f};  // work of either kernel, longest contexts
  for (int i = tid; i < n_seq; i += NT) {
    int tiles = tiles0, kind = kind0, keys = keys0;
    if (i != tid) load(i, tiles, kind, keys);
    const float t = (float)tiles * (float)keys, ks = tiles > 0 ? (float)keys : 0.f;
    w[0] += kind ? 0.f : t;
    w[1] += kind ? t : 0.f;
    w[2] = fmaxf(w[2], kind ? 0.f : ks);
    w[3] = fmaxf(w[3], kind ? ks : 0.f);
  }
  block_reduce<NT, 2, 2>(w, red);
  // Candidate lengths: no split, and c = 0, 1: one and two parts for each workgroup.  They
  // are above the even share by more than the sums' rounding, so the parts of split contexts
  // number less than 2 x 2 x n.
  int len[2][3];
#pragma unroll
  for (int k = 0; k < 2; k++) {
    const Split sp = k ? sp1 : sp0;
    const int least = max(kMinPart, (int)(w[2 + k] * 1.001f) / sp.max_parts + 2);
#pragma unroll
    for (int c = 0; c < 3; c++) {
      const float even = c == 0 ? 0x1p30f : fminf(w[k] * 1.001f / (float)(sp.n * c) + 1.f, 0x1p30f);
      len[k][c] = (max((int)even, least) + 127) & ~127;
    }
  }
  float n[6] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int i = tid; i < n_seq; i += NT) {
    int tiles = tiles0, kind = kind0, keys = keys0;
    if (i != tid) load(i, tiles, kind, keys);
#pragma unroll
    for (int c = 0; c < 3; c++) {
      const float t = (float)tiles * fmaxf(ceilf((float)keys / (float)(kind ? len[1][c] : len[0][c])), 1.f);
      n[c] += kind ? 0.f : t;
      n[3 + c] += kind ? t : 0.f;
    }
  }
  block_reduce<NT, 6, 0>(n, red);
  int part[2];
#pragma unroll
  for (int k = 0; k < 2; k++) {
    const Split sp = k ? sp1 : sp0;
    float best = 0.f;
    part[k] = len[k][0];
#pragma unroll
    for (int c = 0; c < 3; c++) {
      const float most = fminf((float)len[k][c], w[2 + k]), per = n[3 * k + c] / (float)sp.n;
      const float t = fminf(ceilf(per) * most, fmaxf(w[k] / (float)sp.n, most) + 0.5f * most) + per * (float)sp.cost;
      if (c == 0 || t < best) {
        best = t;
        part[k] = len[k][c];
      }
    }
  }
  // Items (40 bits), parts of split contexts (12) and split tiles (12) are placed by one scan:
  // the last two are bounded by the choice of the part whatever the lengths are.
  int64_t at[2] = {0, 0};
  int slots[2] = {0, 0}, joins[2] = {0, 0};
  for (int c0 = 0; c0 < n_seq; c0 += NT) {
    const int i = c0 + tid, cn = min(NT, n_seq - c0);
    int tiles = c0 ? 0 : tiles0, kind = c0 ? 0 : kind0, keys = c0 ? 0 : keys0;
    q0 = first_q0;
    nq = first_nq;
    nk = first_nk;
    if (c0 && i < n_seq) load(i, tiles, kind, keys);
    __syncthreads();  // the items of the requests before have been written
    l_rows[tid][0] = q0;
    l_rows[tid][1] = nq;
    l_rows[tid][2] = nk;
    const int parts = max((int)((unsigned)(keys + (unsigned)part[kind] - 1u) / (unsigned)part[kind]), 1);
    // Long parts first, so that the last workgroups to start are short: three classes by the
    // length of a part (256 decodes of 300 to 4300 keys: 436 us against 468).  Not for the
    // many-row kernel, whose neighbouring tiles of one request share keys in the L2.
    const float most = fminf((float)part[0], w[2]), mine_len = fminf((float)keys, (float)part[0]);
    const int cls = kind ? 3 : mine_len >= 0.67f * most ? 0 : mine_len >= 0.33f * most ? 1 : 2;
    for (int kc = 0; kc < 4; kc++) {
      const int k = kc / 3;
      const bool mine = cls == kc && tiles > 0;
      if (!__syncthreads_or(mine)) continue;
      const int64_t items = mine ? (int64_t)tiles * parts : 0;
      const int64_t x = items | (parts > 1 ? (items << 40) | ((int64_t)(mine ? tiles : 0) << 52) : 0);
      // running sums over the block
      const int lane = tid & 63, wv = tid >> 6;
      int64_t incl = x;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int64_t y = __shfl_up(incl, o);
        if (lane >= o) incl += y;
      }
      __syncthreads();
      if (lane == 63) red64[wv] = incl;
      l_n[tid] = mine ? parts : 0;
      __syncthreads();
      int64_t before = incl - x, total = 0;
#pragma unroll
      for (int e = 0; e < NT / 64; e++) {
        if (e < wv) before += red64[e];
        total += red64[e];
      }
      l_at[tid] = before;
      __syncthreads();
      const int64_t low = (1ll << 40) - 1;
      const int64_t n_items = total & low, room = v.cap_items[k] - at[k];
      for (int64_t y = tid; y < min(n_items, room); y += NT) {
        int lo = 0, hi = cn;  // the last request with items that starts at or before item y
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if ((l_at[mid] & low) <= y) lo = mid; else hi = mid;
        }
        const int64_t b = l_at[lo];
        const unsigned np = (unsigned)max(l_n[lo], 1), rest = (unsigned)(y - (b & low));
        const int tile = (int)(rest / np), pi = (int)(rest - tile * np);
        PlanItem it = {c0 + lo, tile, pi, (int)np, -1, -1, l_rows[lo][0], l_rows[lo][1], l_rows[lo][2], {0, 0, 0}};
        if (np > 1) {
          it.slot = slots[k] + (int)((uint64_t)b >> 40 & 0xfff) + tile * (int)np;
          it.join = joins[k] + (int)((uint64_t)b >> 52) + tile;
        }
        v.items[k][at[k] + y] = it;
      }
      at[k] += n_items;
      slots[k] += (int)((uint64_t)total >> 40 & 0xfff);
      joins[k] += (int)((uint64_t)total >> 52);
    }
  }
  if (tid < 2) {
    v.hdr->n_items[tid] = (int)min(at[tid], (int64_t)v.cap_items[tid]);
    v.hdr->part[tid] = part[tid];
  }
}

struct Dyn {
  int value;
};
// The kernels' state is held by reference in lambdas: not inlined, it would be memory.
#define CF_INLINE __attribute__((always_inline))

template <int N>
struct Int {
  static constexpr int value = N;
};

// Infinities and NaN: exponent all ones.
template <typename T>
constexpr uint32_t kExpMask = __is_same(T, __bf16) ? 0x7f80u : 0x7c00u;
// Eight elements: zeroes the infinities and NaN, says whether there were any.
template <typename T>
__device__ __forceinline__ bool take_specials(i32x4 &x) {
  bool b = false;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const uint32_t u = (uint32_t)x[i];
    const uint32_t lo = (u & kExpMask<T>) == kExpMask<T> ? 0u : 0xffffu;
    const uint32_t hi = ((u >> 16) & kExpMask<T>) == kExpMask<T> ? 0u : 0xffff0000u;
    b |= (lo & (hi >> 16)) == 0;
    x[i] = (int)(u & (lo | hi));
  }
  return b;
}
template <typename T>
__device__ __forceinline__ bool special(T x) {
  return (__builtin_bit_cast(uint16_t, x) & kExpMask<T>) == kExpMask<T>;
}

// The infinities and NaN among the values of keys [from, to), which not all
// of the rows row0 .. row0 + n - 1 see, added to the results just written.
template <typename T, bool PAGED>
__device__ __forceinline__ void add_specials(const AttnArgs &a, const Rows &r, int k0, int seq, int slot, int R,
                                             int head, int row0, int n, int from, int to) {
  parts_arrived();
  __syncthreads();
#pragma unroll 1
  for (int x = threadIdx.x; x < n * (a.D / 2); x += (int)blockDim.x) {
    const int rr = x / (a.D / 2), e = (x - rr * (a.D / 2)) * 2;
    const int row = row0 + rr, j = row / a.G, g = row - j * a.G;
    const int last = min(r.nk - r.nq + j, to - 1);
    float sum[2] = {0.f, 0.f};
#pragma unroll 1
    for (int key = from; key <= last; key++) {
      const T *v = (const T *)g_zeros;
      if (PAGED) {
        const int id = a.table[(int64_t)seq * a.max_pages + (key >> a.page_log2)];
        if ((unsigned)id < (unsigned)a.n_pages)
          v = (const T *)a.v + ((((int64_t)id * a.Hkv + head) << a.page_log2) + (key & ((1 << a.page_log2) - 1))) * a.D + e;
      } else {
        v = (const T *)a.v + (int64_t)(k0 + key) * a.v_tok + head * a.v_head + e;
      }
      if (special<T>(v[0])) sum[0] += (float)v[0];
      if (special<T>(v[1])) sum[1] += (float)v[1];
    }
    if (sum[0] == 0.f && sum[1] == 0.f) continue;
    if (slot >= 0) {
      float *p = a.plan.o[R > kRowsSmall] + (((int64_t)slot * a.Hkv + head) * R + rr) * a.D + e;
      const float2 o = load_part(p);
      store_part(p, o.x + sum[0], o.y + sum[1]);
    } else {
      T *p = (T *)a.out + ((int64_t)(r.q0 + j) * a.H + head * a.G + g) * a.D + e;
      p[0] = (T)((float)p[0] + sum[0]);
      p[1] = (T)((float)p[1] + sum[1]);
    }
  }
}

// ------------------------------------------------------------------ work items
struct Item {
  int seq, tile, part, n, slot, join;  // part of n of the rows' context; n 1: slot and join unused
  int lo, end;                         // its keys
};

// Item `item` of the plan, if there is one and it names what exists: work_dev may hold anything,
// a plan for other sizes or none.  Parts are multiples of 128 keys, so that a group of 16 keys lies
// in one page; tile numbers below 2^27 keep row numbers in 32 bits.
__device__ __forceinline__ bool read_item(const AttnArgs &a, int kind, int item, Item &it, Rows &r) {
  if (item >= min(a.plan.hdr->n_items[kind], a.plan.cap_items[kind])) return false;
  const PlanItem p = a.plan.items[kind][item];
  const int len = a.plan.hdr->part[kind];
  it = Item{p.seq, p.tile, p.part, p.n, p.slot, p.join, 0, 0x7fffffff};
  r.q0 = clampi(p.q0, 0, a.n_tok);
  r.nq = clampi(p.nq, 0, a.n_tok - r.q0);
  r.nk = (int)min((int64_t)max(p.nk, 0), (int64_t)a.max_pages << a.page_log2);
  if ((unsigned)p.seq >= (unsigned)a.n_seq || (unsigned)p.tile >= 1u << 27 || p.n < 1) return false;
  if (p.n > 1) {
    if (p.part < 0 || p.part >= p.n || p.slot < 0 || p.slot > a.plan.cap_slots[kind] - p.n ||
        (unsigned)p.join >= (unsigned)a.plan.cap_join[kind] || p.n > max_parts(kind) || len < 1 || len >= 1 << 30 ||
        (len & 127))
      return false;
    it.lo = (int)min((int64_t)p.part * len, (int64_t)1 << 30);
    if (p.part < p.n - 1) it.end = it.lo + len;
  }
  return true;
}

// The parts of a split context are joined by the workgroup that finishes last, in part
// order whichever it is:  m = max m_p, l = sum l_p e^(m_p - m), o = sum o_p e^(m_p - m) / l.
// w: LDS of this workgroup, at least 2 x max_parts x R floats.
template <typename T, int R>
__device__ __forceinline__ void join_parts(const AttnArgs &a, const Rows &r, const Item &it, int head, int row0,
                                           int n, float *w) {
  using V4 = typename Elem<T>::v4;
  constexpr int kind = R > kRowsSmall;
  __shared__ int last;
  __shared__ float l_sum[R];
  const int tid = threadIdx.x, nt = (int)blockDim.x;
  parts_arrived();
  __syncthreads();
  if (tid == 0) {
    int *done = a.plan.done[kind] + (int64_t)it.join * a.Hkv + head;
    last = atomicAdd(done, 1) == it.n - 1;
    if (last) *done = 0;  // for the next layer's call
  }
  __syncthreads();
  if (!last) return;
  const float *ml = a.plan.ml[kind], *o = a.plan.o[kind];
  const int64_t base = ((int64_t)it.slot * a.Hkv + head) * R, step = (int64_t)a.Hkv * R;
  // maxima and sums of all parts to LDS at once; then a row's weights of the parts, and lse
  float *wl = w + it.n * R;
  for (int x = tid; x < it.n * R; x += nt) {
    const int p = x / R, rr = x % R;
    if (rr >= n) continue;
    const float2 y = load_part(ml + (base + p * step + rr) * 2);
    w[x] = y.x;
    wl[x] = y.y;
  }
  __syncthreads();
  for (int rr = tid; rr < n; rr += nt) {
    float m = kNegInf, l = 0.f;
    for (int p = 0; p < it.n; p++) m = fmaxf(m, w[p * R + rr]);
    const float mu = m == kNegInf ? 0.f : m;
    for (int p = 0; p < it.n; p++) {
      const float f = exp2_hw((w[p * R + rr] - mu) * a.s2);
      w[p * R + rr] = f;
      l = fmaf(f, wl[p * R + rr], l);
    }
    l_sum[rr] = l > 0.f || l != l ? 1.f / l : 0.f;
    const int j = (row0 + rr) / a.G, g = row0 + rr - j * a.G;
    if (a.lse) a.lse[(int64_t)(r.q0 + j) * a.H + head * a.G + g] = log_sum(m, l, a.s2, weight_shift<T>(kind));
  }
  __syncthreads();
  const int quads = a.D / 4;
  for (int x = tid; x < n * quads; x += nt) {
    const int rr = x / quads, d4 = x - rr * quads;
    f32x4 acc = {0, 0, 0, 0};
#pragma unroll 16
    for (int p = 0; p < it.n; p++) {
      const float *src = o + (base + p * step + rr) * a.D + d4 * 4;
      const float2 x = load_part(src), y = load_part(src + 2);
      acc += f32x4{x.x, x.y, y.x, y.y} * w[p * R + rr];
    }
    const int j = (row0 + rr) / a.G, g = row0 + rr - j * a.G;
    T *out = (T *)a.out + ((int64_t)(r.q0 + j) * a.H + head * a.G + g) * a.D + d4 * 4;
    *(V4 *)out = __builtin_convertvector(acc * l_sum[rr], V4);
  }
}

// ------------------------------------------------------------------ few rows
// A workgroup of four waves takes 16 rows of one key/value head over a range
// of keys; wave w takes tiles w, w + 4, ... of 32 keys.  A tile's scores are
// S^T = K Q^T (16 keys x 16 rows a matrix instruction, K straight from memory
// to registers), so a lane has 8 scores of one row and the row's maximum takes
// two exchanges; the probabilities already lie as the second operand of
// O^T = V^T P^T, whose first operand is read transposed from the wave's own
// copy of the tile in LDS.  The next tile's keys and values are loaded while
// one is worked on.  The waves' results are joined at the end.
//
// Bound by memory: 256 requests of 1767 keys on average (32 heads on 8, 128
// columns, bf16, pages of 16) 287 us, 6.5 TB/s of cache (a kernel that only reads
// reaches 6.3 with ordinary loads); one request of 32767 keys on 32 key/value heads
// 85 us, 6.3 TB/s.  Two workgroups a CU hold 128 KB in flight; a third (168
// registers, 7 spilled) is 10 % slower.  The matrix unit is busy 4 % of the time,
// also where one of its 16 rows is used.
template <typename T, int KS, int DB, int DS>
__global__ __launch_bounds__(256, DS > 128 ? 1 : 2) void k_attn_few(AttnArgs a) {
  using V8 = typename Elem<T>::v8;
  using V4 = typename Elem<T>::v4;
  constexpr int CH = DS / 8, NV = 32 * CH / 64;
  __shared__ __attribute__((aligned(16))) char lds[4][32 * DS * 2];
  __shared__ float l_m[4][16], l_l[4][16];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = (int)(blockIdx.x % (unsigned)a.Hkv), item = (int)(blockIdx.x / (unsigned)a.Hkv);
  Item it;
  Rows r;
  if (!read_item(a, 0, item, it, r)) return;
  const int n_rows = r.nq * a.G, row0 = it.tile * kRowsSmall;
  if (row0 >= n_rows) return;
  const int row = row0 + (lane & 15), j = min(row, n_rows - 1) / a.G, g = min(row, n_rows - 1) - j * a.G;
  const int last_j = (min(row0 + kRowsSmall, n_rows) - 1) / a.G;
  const int seen = r.nk - r.nq + last_j + 1;  // keys the tile's last row sees
  const int hi = __builtin_amdgcn_readfirstlane(min(seen, it.end));
  const int lim = r.nk - r.nq + j;  // last key the lane's row sees
  const int all = r.nk - r.nq + row0 / a.G + 1;  // keys that every row sees

  const int gq = lane >> 4;
  V8 qf[KS];
  const T *qp = (const T *)a.q + (int64_t)(r.q0 + j) * a.q_tok + (int64_t)(head * a.G + g) * a.q_head;
#pragma unroll
  for (int ks = 0; ks < KS; ks++) {
    const int c = ks * 4 + gq;
    qf[ks] = __builtin_bit_cast(V8, load16(c * 8 < a.D ? (const void *)(qp + c * 8) : (const void *)g_zeros));
  }

  const int64_t page_elems = (int64_t)a.Hkv * a.D << a.page_log2;
  const int64_t head_off = (int64_t)head * a.D << a.page_log2;
  const T *kc = (const T *)a.k + head_off, *vc = (const T *)a.v + head_off;
  const int page_mask = (1 << a.page_log2) - 1;
  const int32_t *trow = a.table + (int64_t)it.seq * a.max_pages;
  const int n_tiles = hi > it.lo ? (hi - it.lo + 31) >> 5 : 0;

  f32x4 o[DB];
#pragma unroll
  for (int d = 0; d < DB; d++) o[d] = f32x4{0, 0, 0, 0};
  float m = kNegInf, l = 0.f;
  V8 kr[2][KS];
  i32x4 vr[NV];
  int ids = 0;
  T *vt = (T *)lds[w];
  bool bad = false;

  // the wave's tile n: page ids of 32 tiles at a time lie across the lanes
  auto load_ids = [&](int n) {
    const int key = it.lo + 32 * (w + 4 * (n + (lane >> 1))) + 16 * (lane & 1);
    ids = key < hi ? trow[key >> a.page_log2] : -1;
  };
  auto load = [&](int n) {
    if ((n & 31) == 0) load_ids(n);
    const int t0 = it.lo + 32 * (w + 4 * n);
    int64_t base[2];
    int valid[2];
#pragma unroll
    for (int b = 0; b < 2; b++) {
      const int id = __builtin_amdgcn_readlane(ids, ((n & 31) << 1) + b);
      const bool in = (unsigned)id < (unsigned)a.n_pages;
      base[b] = (in ? id : 0) * page_elems + (int64_t)((t0 + 16 * b) & page_mask) * a.D;
      valid[b] = in ? r.nk - (t0 + 16 * b) : 0;  // keys of the 16 that may be read
    }
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
      for (int ks = 0; ks < KS; ks++) {
        const int c = ks * 4 + gq, key = lane & 15;
        const bool ok = key < valid[b] && c * 8 < a.D;
        kr[b][ks] = __builtin_bit_cast(V8, load16_nt(ok ? (const void *)(kc + base[b] + key * a.D + c * 8) : (const void *)g_zeros));
      }
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int x = i * 64 + lane, key = x / CH, c = x % CH, b = (i * 64 / CH) >> 4;
      const bool ok = (key & 15) < valid[b] && c * 8 < a.D;
      vr[i] = load16_nt(ok ? (const void *)(vc + base[b] + (key & 15) * a.D + c * 8) : (const void *)g_zeros);
    }
  };

  if (w < n_tiles) load(0);
  for (int n = 0; w + 4 * n < n_tiles; n++) {
    const int t0 = it.lo + 32 * (w + 4 * n);
    if (t0 + 32 > all && r.nk > all) {  // also where no row sees them
#pragma unroll
      for (int i = 0; i < NV; i++) bad |= take_specials<T>(vr[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int x = i * 64 + lane, key = x / CH, c = x % CH;
      *(i32x4 *)(vt + key * DS + (c ^ swz8<DS>(key)) * 8) = vr[i];
    }
    f32x4 s[2];
#pragma unroll
    for (int b = 0; b < 2; b++) {
      s[b] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int ks = 0; ks < KS; ks++) s[b] = Elem<T>::mma16(kr[b][ks], qf[ks], s[b]);
    }
    if (w + 4 * (n + 1) < n_tiles) load(n + 1);
    float mx = kNegInf;
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const int key = t0 + 16 * b + 4 * gq + i;
        s[b][i] = key <= lim && key < hi ? s[b][i] : kNegInf;
        mx = fmaxf(mx, s[b][i]);
      }
    mx = max_halves(max_rows16(mx));
    const float mn = fmaxf(m, mx), mu = mn == kNegInf ? 0.f : mn * a.s2;
    const float mp = mu - weight_shift<T>(0);
    const float alpha = exp2_hw(fmaf(m, a.s2, -mu));
    m = mn;
    V8 pf;
    float ps = 0.f;
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const float p = exp2_hw(fmaf(s[b][i], a.s2, -mp));
        ps += p;
        pf[b * 4 + i] = (T)p;
      }
    l = fmaf(l, alpha, ps);
    __builtin_amdgcn_wave_barrier();
    const int vrow = 4 * gq + ((lane & 15) >> 2), vcol = 4 * (lane & 3);
#pragma unroll
    for (int d = 0; d < DB; d++) {
      const int c = d * 2 + (vcol >> 3), off = vcol & 7;
      const V4 lo4 = read_tr<T>(vt + vrow * DS + (c ^ swz8<DS>(vrow)) * 8 + off);
      const V4 hi4 = read_tr<T>(vt + (vrow + 16) * DS + (c ^ swz8<DS>(vrow + 16)) * 8 + off);
      o[d] = o[d] * alpha;
      o[d] = Elem<T>::mma16(join8<V8>(lo4, hi4), pf, o[d]);
    }
    __builtin_amdgcn_wave_barrier();
  }
  l = sum_halves(sum_rows16(l));

  // join the waves: o through LDS (a wave's value tile is as large as its 16 x DS floats)
  const int any_bad = __syncthreads_or(bad);
  if (gq == 0) { l_m[w][lane] = m; l_l[w][lane] = l; }
  float *ow = (float *)lds[w];
#pragma unroll
  for (int d = 0; d < DB; d++) *(f32x4 *)(ow + (lane & 15) * DS + d * 16 + 4 * gq) = o[d];
  __syncthreads();
  const int quads = a.D / 4;
  for (int x = threadIdx.x; x < kRowsSmall * quads; x += 256) {
    const int rr = x / quads, d4 = x - rr * quads;
    if (row0 + rr >= n_rows) continue;
    float mm = kNegInf;
#pragma unroll
    for (int i = 0; i < 4; i++) mm = fmaxf(mm, l_m[i][rr]);
    const float mu = mm == kNegInf ? 0.f : mm;
    float ll = 0.f;
    f32x4 oo = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const float f = exp2_hw((l_m[i][rr] - mu) * a.s2);
      ll = fmaf(f, l_l[i][rr], ll);
      oo += *(const f32x4 *)((const float *)lds[i] + rr * DS + d4 * 4) * f;
    }
    if (it.n > 1) {
      const int64_t pr = ((int64_t)(it.slot + it.part) * a.Hkv + head) * kRowsSmall + rr;
      store_part(a.plan.o[0] + pr * a.D + d4 * 4, oo[0], oo[1]);
      store_part(a.plan.o[0] + pr * a.D + d4 * 4 + 2, oo[2], oo[3]);
      if (d4 == 0) store_part(a.plan.ml[0] + pr * 2, mm, ll);
    } else {
      const int jj = (row0 + rr) / a.G, gg = row0 + rr - jj * a.G;
      const int64_t orow = (int64_t)(r.q0 + jj) * a.H + head * a.G + gg;
      const float inv = ll > 0.f || ll != ll ? 1.f / ll : 0.f;
      *(V4 *)((T *)a.out + orow * a.D + d4 * 4) = __builtin_convertvector(oo * inv, V4);
      if (a.lse && d4 == 0) a.lse[orow] = log_sum(mm, ll, a.s2, weight_shift<T>(0));
    }
  }
  if (any_bad)
    add_specials<T, true>(a, r, 0, it.seq, it.n > 1 ? it.slot + it.part : -1, kRowsSmall, head, row0, min(n_rows - row0, kRowsSmall),
                          it.lo + (max(all - it.lo, 0) & ~31), hi);
  if (it.n > 1) join_parts<T, kRowsSmall>(a, r, it, head, row0, min(n_rows - row0, kRowsSmall), (float *)lds[0]);
}

// The order of a matrix phase for the instruction scheduler: NK products with one
// operand read from LDS each, then NV with two reads each; reads run AHEAD products
// in front, so that a product's operands have arrived when the unit is free for it.
template <int NK, int NV, int AHEAD>
__device__ __forceinline__ void matrix_order() {
  constexpr int MFMA = 0x8, DSREAD = 0x100;
  __builtin_amdgcn_sched_group_barrier(DSREAD, NK > 0 ? AHEAD : 2 * AHEAD, 0);
#pragma unroll
  for (int i = 0; i < NK - AHEAD; i++) {
    __builtin_amdgcn_sched_group_barrier(MFMA, 1, 0);
    __builtin_amdgcn_sched_group_barrier(DSREAD, 1, 0);
  }
#pragma unroll
  for (int i = 0; i < (NK > 0 ? NV : NV - AHEAD); i++) {
    __builtin_amdgcn_sched_group_barrier(MFMA, 1, 0);
    __builtin_amdgcn_sched_group_barrier(DSREAD, 2, 0);
  }
  __builtin_amdgcn_sched_group_barrier(MFMA, AHEAD, 0);
}

// ------------------------------------------------------------------ many rows
// A workgroup takes NG groups of four waves; a group takes 128 rows of one
// key/value head, 32 a wave, and all share tiles of 64 keys in LDS.  S^T = K Q^T
// (32 keys x 32 rows a matrix instruction), so a lane has 32 scores of one row,
// and O^T = V^T P^T as in the few-row kernel: the order of the keys within a step
// is the order in which S^T leaves them in the lane, the values' operand is read
// to match, and no probability changes lanes.
//
// A wave alternates between a matrix phase, S of tile n and O += V P of tile
// n - 1, and a vector phase, the softmax of tile n.  The two groups are one phase
// apart: on every SIMD one wave feeds the matrix unit while the other one
// exponentiates.  A barrier ends each phase, and with phases numbered 0, 1, 2, ...
// group g has its matrix phase n at 2n + g.  In its vector phase n it stores its
// share of keys n + 1 + g and values n + g, loaded one round earlier: those go to
// the LDS halves of keys n - 1 + g and values n - 2 + g, which both groups have
// read by then, and are complete when group 0 begins its matrix phase n + 1 + g.
// With one group a workgroup runs on its own, two or three of them a CU, and needs
// one barrier a round.
//
// Bound by the matrix unit and its power: one causal sequence of 32767 tokens (32
// heads on 8, 128 columns, bf16) 7.09 ms, 1.24 PFLOP/s, as a large library matrix
// product on the same card; the unit is busy 71 % of the cycles at 1.65 GHz.  What
// the steps to it were worth on that case: a tile's work in one stream, operands
// read right before their use, 9.6 ms; the maximum allowed to lag 8.7; two groups
// out of step 9.5 and, with the operand reads ordered ahead, 8.1; the exponentials
// kept in the vector phase 7.3.  Short sequences pay 8 us a workgroup to start and
// end: 16 causal prompts of 1387 tokens on average 412 us, 0.86 PFLOP/s.  With 64
// columns the exponentials take longer than the products, and what is neither is
// the start, the end and the edge rounds of 4 to 16 tiles: 16 full images of 623
// patches, 16 heads, 53 us, 0.54 PFLOP/s, matrix unit busy 36 %.  Above 128 columns a
// wave's state does not fit the registers (32 of them spilled, 55 over a cache): one
// causal sequence of 4096 tokens, 16 heads of 256, 241 us, 0.57 PFLOP/s; two chunks of
// 1000 tokens on 24001, 32 heads on 8, 3.4 ms, 0.48 PFLOP/s.  136 to 248 columns take as long.
template <typename T, int KS, int DB, int DS, int NG, bool PAGED>
__global__ __launch_bounds__(256 * NG, DS == 64 ? 3 : DS == 128 ? 2 : 1) void k_attn_many(AttnArgs a) {
  using V8 = typename Elem<T>::v8;
  using V4 = typename Elem<T>::v4;
  constexpr int NT = 256 * NG, R = kRowsGroup * NG, CH = DS / 8, NL = 64 * CH / NT, RS = NT / CH;
  __shared__ __attribute__((aligned(16))) T lds_k[2][64 * DS], lds_v[2][64 * DS];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), grp = NG > 1 ? w >> 2 : 0;
  const int head = (int)(blockIdx.x % (unsigned)a.Hkv), item = (int)(blockIdx.x / (unsigned)a.Hkv);
  Item it;
  Rows r;
  int k0 = 0;
  if (PAGED) {
    if (!read_item(a, 1, item, it, r)) return;
  } else {
    // sequence i owns the tiles from floor(first row / R) + i on; 64 probes at a time, the
    // last round of them over neighbours, which also gives the sequence's bounds
    int lo = 0, n = a.n_seq, q, q1, e0, e1;
    for (;;) {
      const int step = (n + 63) >> 6, i = lo + min(lane * step, n - 1);
      q = clampi(a.q_start[i], 0, a.n_tok);
      q1 = clampi(a.q_start[i + 1], 0, a.n_tok);
      e0 = clampi(a.kv[i], 0, a.n_k);
      e1 = clampi(a.kv[i + 1], 0, a.n_k);
      const bool le = lane * step < n && (int)((unsigned)(q * a.G) / R) + i <= item;
      const int at = max(__builtin_popcountll(__ballot(le)) - 1, 0);
      q = __builtin_amdgcn_readlane(q, at);
      q1 = __builtin_amdgcn_readlane(q1, at);
      e0 = __builtin_amdgcn_readlane(e0, at);
      e1 = __builtin_amdgcn_readlane(e1, at);
      lo += at * step;
      if (step == 1) break;
      n = min(step, n - at * step);
    }
    it.seq = lo;
    it.tile = item - ((int)((unsigned)(q * a.G) / R) + lo);
    r.q0 = q;
    r.nq = max(q1 - q, 0);
    k0 = e0;
    r.nk = max(e1 - e0, 0);
    it.lo = 0;
    it.end = 0x7fffffff;
    it.n = 1;
  }
  const int n_rows = __builtin_amdgcn_readfirstlane(r.nq * a.G);  // below 2^31, as all row numbers
  const int n_rt = (n_rows + R - 1) / R;
  if (it.tile < 0 || it.tile >= n_rt) return;
  // the rows that see most keys first
  const int row0 = (n_rt - 1 - it.tile) * R;
  const int row = row0 + w * 32 + (lane & 31);
  const unsigned G = (unsigned)a.G;
  const int j = (int)((unsigned)min(row, n_rows - 1) / G), g = min(row, n_rows - 1) - j * a.G;
  const bool causal = PAGED || a.causal;
  const int off = causal ? r.nk - r.nq : r.nk;  // row j sees keys up to off + j, or all
  const int last_j = (int)((unsigned)(min(row0 + R, n_rows) - 1) / G);
  const int seen = causal ? min(off + last_j + 1, r.nk) : r.nk;
  const int hi = __builtin_amdgcn_readfirstlane(min(seen, it.end));
  const int lim = min(causal ? off + j : r.nk - 1, hi - 1);
  // keys that every row of the workgroup sees, and every row of the wave
  const int all_wg = causal ? off + (int)((unsigned)row0 / G) + 1 : r.nk;
  const int all = min(causal ? off + __builtin_amdgcn_readlane(j, 0) + 1 : r.nk, hi);
  const int h = lane >> 5;

  const int64_t page_elems = (int64_t)a.Hkv * a.D << a.page_log2;
  const int64_t head_off = (int64_t)head * a.D << a.page_log2;
  const T *kc = (const T *)a.k + (PAGED ? head_off : (int64_t)k0 * a.k_tok + head * a.k_head);
  const T *vc = (const T *)a.v + (PAGED ? head_off : (int64_t)k0 * a.v_tok + head * a.v_head);
  const int page_mask = (1 << a.page_log2) - 1;
  const int32_t *trow = PAGED ? a.table + (int64_t)it.seq * a.max_pages : nullptr;
  const int n_tiles = hi > it.lo ? (hi - it.lo + 63) >> 6 : 0;

  V8 qf[KS];
  f32x16 o[DB], s[2];
#pragma unroll
  for (int d = 0; d < DB; d++)
#pragma unroll
    for (int i = 0; i < 16; i++) o[d][i] = 0.f;
  V8 pf[4];
  float m = kNegInf, l = 0.f;
  i32x4 kr[NL], vr[NL];
#pragma unroll
  for (int i = 0; i < NL; i++) kr[i] = vr[i] = i32x4{0, 0, 0, 0};
  uint64_t k_at = 0, v_at = 0;
  bool bad = false;

  // Loads of a tile's keys or values; edge: some may not be there or the tile be past the
  // last, which gives zeros.  Chunks past head_dim are never loaded and stay zero.
  const int lrow = tid / CH, lcol = tid % CH;
  const bool col_ok = lcol * 8 < a.D;
  const int to_load = min(r.nk, it.lo + 64 * n_tiles);
  // Where the keys and values of tiles n .. n + 7 begin (n a multiple of 8), a lane for each 16
  // keys, the lanes of 16 tiles in two halves.  The page ids are loaded 12 tiles ahead and made
  // addresses 8 ahead of the next half's first use: a round neither waits for an id nor does
  // the arithmetic of a page at every load.
  int ids = -1;
  auto load_ids = [&](int n) CF_INLINE {
    const int key = it.lo + 64 * n + 16 * (lane & 31);
    ids = key < hi ? trow[key >> a.page_log2] : -1;
  };
  auto place = [&](int n) CF_INLINE {
    if ((lane >> 5) == ((n >> 3) & 1)) {
      const int key = it.lo + 64 * n + 16 * (lane & 31);
      const int64_t at = (int64_t)ids * page_elems + (int64_t)(key & page_mask) * a.D;
      const bool in = (unsigned)ids < (unsigned)a.n_pages;
      k_at = (uint64_t)(in ? kc + at : (const T *)g_zeros);
      v_at = (uint64_t)(in ? vc + at : (const T *)g_zeros);
    }
  };
  // packed: the lane's row of the next tile to load
  const T *kp = kc + (int64_t)lrow * a.k_tok + lcol * 8, *vp = vc + (int64_t)lrow * a.v_tok + lcol * 8;
  auto load = [&](i32x4 (&x)[NL], uint64_t where, const T *&at, int64_t tok, int n, auto edge) CF_INLINE {
    const int t0 = it.lo + 64 * n;
    if (!col_ok) return;
#pragma unroll
    for (int i = 0; i < NL; i++) {
      const int rr = i * RS + lrow;
      const T *p;
      if (PAGED) {
        const int l16 = ((n & 15) << 2) + __builtin_amdgcn_readfirstlane(rr >> 4);
        const uint32_t alo = __builtin_amdgcn_readlane((uint32_t)where, l16);
        const uint32_t ahi = __builtin_amdgcn_readlane((uint32_t)(where >> 32), l16);
        p = (const T *)((uint64_t)ahi << 32 | alo) + (unsigned)((rr & 15) * a.D + lcol * 8);
      } else {
        p = at + i * RS * tok;
      }
      if (edge.value) p = t0 + rr < to_load ? p : (const T *)g_zeros;
      x[i] = load16(p);
    }
    if (!PAGED) at += 64 * tok;
  };
  auto store = [&](const i32x4 (&x)[NL], T *dst) CF_INLINE {
#pragma unroll
    for (int i = 0; i < NL; i++) {
      const int rr = i * RS + lrow;
      *(i32x4 *)(dst + rr * DS + (lcol ^ swz<DS>(rr)) * 8) = x[i];
    }
  };
  // keys nk and values nk - 1 to registers, or from there to LDS
  auto fetch = [&](int nk, auto edge) CF_INLINE {
    load(kr, k_at, kp, a.k_tok, nk, edge);
    load(vr, v_at, vp, a.v_tok, nk - 1, edge);
    if (PAGED && (nk & 7) == 4) place(nk + 4);  // in place of tiles nk - 12 .. nk - 5
    if (PAGED && (nk & 7) == 0) load_ids(nk + 8);
  };
  auto put = [&](int nk, T *kd, T *vd, auto edge) CF_INLINE {
    store(kr, kd);
    if (edge.value && it.lo + 64 * nk > all_wg && r.nk > all_wg) {  // also where no row sees them
      asm volatile("");  // a branch: not worth computing for every tile
#pragma unroll
      for (int i = 0; i < NL; i++) bad |= take_specials<T>(vr[i]);
    }
    store(vr, vd);
  };

  auto scores = [&](const T *kt) CF_INLINE {
    const int rr = lane & 31;
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
      for (int i = 0; i < 16; i++) s[b][i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ks++)
#pragma unroll
      for (int b = 0; b < 2; b++) {
        const V8 kf = *(const V8 *)(kt + b * 32 * DS + rr * DS + (((ks * 2 + h) ^ swz<DS>(rr)) * 8));
        s[b] = Elem<T>::mma32(kf, qf[ks], s[b]);
      }
  };
  const int vcol = 16 * ((lane >> 4) & 1) + 4 * (lane & 3), vr0 = 4 * h + ((lane & 15) >> 2);
  auto values = [&](const T *vt) CF_INLINE {
#pragma unroll
    for (int k = 0; k < 4; k++)
#pragma unroll
      for (int d = 0; d < DB; d++) {
        const int c = d * 4 + (vcol >> 3), of = vcol & 7;
        const V4 lo4 = read_tr<T>(vt + k * 16 * DS + vr0 * DS + (c ^ swz<DS>(vr0)) * 8 + of);
        const V4 hi4 = read_tr<T>(vt + k * 16 * DS + (vr0 + 8) * DS + (c ^ swz<DS>(vr0 + 8)) * 8 + of);
        o[d] = Elem<T>::mma32(join8<V8>(lo4, hi4), pf[k], o[d]);
      }
  };
  auto softmax = [&](int n, auto edge) CF_INLINE {
    const int t0 = it.lo + 64 * n;
    if (edge.value && t0 + 64 > all) {
      const int room = lim - t0 - 4 * h;
      asm volatile("");
#pragma unroll
      for (int b = 0; b < 2; b++)
#pragma unroll
        for (int i = 0; i < 16; i++) {
          s[b][i] = b * 32 + 8 * (i >> 2) + (i & 3) <= room ? s[b][i] : kNegInf;
        }
    }
    float mx = kNegInf;
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
      for (int i = 0; i < 16; i++) mx = fmaxf(mx, s[b][i]);
    mx = max_halves(mx);
    // the maximum follows only when some row's has grown by more than 2^8 in its exponentials:
    // p_k up to 256 do no harm, and most tiles need not scale o
    if (__ballot((mx - m) * a.s2 > 8.f)) {
      const float mn = fmaxf(m, mx);
      const float alpha = mn == kNegInf ? 1.f : exp2_hw((m - mn) * a.s2);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int d = 0; d < DB; d++) o[d] = o[d] * alpha;
    }
    const float mp = m == kNegInf ? 0.f : m * a.s2 - weight_shift<T>(1);
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
      for (int i = 0; i < 16; i++) {
        const float p = exp2_hw(fmaf(s[b][i], a.s2, -mp));
        l += p;
        pf[b * 2 + (i >> 3)][i & 7] = (T)p;
      }
    // the probabilities are made here, not where they are used, after the barrier
#pragma unroll
    for (int k = 0; k < 4; k++) {
      i32x4 x = __builtin_bit_cast(i32x4, pf[k]);
      asm volatile("" : "+v"(x));
      pf[k] = __builtin_bit_cast(V8, x);
    }
  };

  // One round: the matrix phase of tile n, then its vector phase.  edge: some row may not see
  // all its keys or all the values it stores, or a fetched tile not be there.
  auto round = [&](int n, auto buf, auto edge) CF_INLINE {
    const int B = buf.value;
    __builtin_amdgcn_s_setprio(1);
    scores(lds_k[B]);
    values(lds_v[1 - B]);
    matrix_order<2 * KS, 4 * DB, 4>();
    __builtin_amdgcn_s_setprio(0);
    if (NG > 1) __syncthreads();
    __builtin_amdgcn_sched_barrier(0);
    softmax(n, edge);
    const int q = (1 - B) ^ grp;
    put(n + 1 + grp, lds_k[q], lds_v[1 - q], edge);
    fetch(n + 2 + grp, edge);
    asm volatile("" ::: "memory");  // the loads stay here, a round ahead of their store
    __syncthreads();
  };

  // No values before the first tile's: zeros, with probabilities of zero.
#pragma unroll
  for (int k = 0; k < 4; k++) pf[k] = __builtin_bit_cast(V8, i32x4{0, 0, 0, 0});
  store(vr, lds_v[1]);
  if (PAGED) {
    load_ids(0);
    place(0);
    load_ids(8);
  }
  {
    i32x4 first[NL];
#pragma unroll
    for (int i = 0; i < NL; i++) first[i] = i32x4{0, 0, 0, 0};
    load(first, k_at, kp, a.k_tok, 0, Int<1>());
    fetch(1, Int<1>());
    // the queries after the first keys and values: those are waited for first
    const T *qp = (const T *)a.q + (int64_t)(r.q0 + j) * a.q_tok + (int64_t)(head * a.G + g) * a.q_head;
#pragma unroll
    for (int ks = 0; ks < KS; ks++) {
      const int c = ks * 2 + h;
      qf[ks] = __builtin_bit_cast(V8, load16(c * 8 < a.D ? (const void *)(qp + c * 8) : (const void *)g_zeros));
    }
    store(first, lds_k[0]);
  }
  __syncthreads();
  if (grp == 1) {
    put(1, lds_k[1], lds_v[0], Int<1>());
    fetch(2, Int<1>());
    __syncthreads();
  }
  // rounds whose tile every row of the workgroup sees, as it does the values that they store,
  // and whose fetched keys are there; two at a time, one per LDS buffer
  const int n_main = min((min(all_wg, hi) - it.lo) / 64 + 1 - NG, (r.nk - it.lo) / 64 - 1 - NG);
  int n = 0;
  for (; n + 2 <= n_main; n += 2) {
    round(n, Int<0>(), Int<0>());
    round(n + 1, Int<1>(), Int<0>());
  }
#pragma unroll 1
  for (; n < n_tiles; n++) round(n, Dyn{n & 1}, Int<1>());
  if (n_tiles > 0) {
    values(lds_v[(n_tiles - 1) & 1]);
    matrix_order<0, 4 * DB, 4>();
  }
  if (NG > 1 && grp == 0) __syncthreads();

  l = sum_halves(l);
  const int any_bad = __syncthreads_or(bad);
  if (row < n_rows && it.n > 1) {
    const int64_t pr = ((int64_t)(it.slot + it.part) * a.Hkv + head) * R + w * 32 + (lane & 31);
#pragma unroll
    for (int d = 0; d < DB; d++)
#pragma unroll
      for (int q = 0; q < 4; q++) {
        const int e = d * 32 + 8 * q + 4 * h;
        if (e < a.D) {
          store_part(a.plan.o[1] + pr * a.D + e, o[d][4 * q], o[d][4 * q + 1]);
          store_part(a.plan.o[1] + pr * a.D + e + 2, o[d][4 * q + 2], o[d][4 * q + 3]);
        }
      }
    if (h == 0) store_part(a.plan.ml[1] + pr * 2, m, l);
  } else if (row < n_rows) {
    const int64_t orow = (int64_t)(r.q0 + j) * a.H + head * a.G + g;
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
    // Of two neighbouring groups of 8 columns, each of which lies half in this lane and half in
    // the one 32 away, either lane takes one whole: 16-byte stores.
#pragma unroll
    for (int d = 0; d < DB; d++)
#pragma unroll
      for (int q = 0; q < 4; q += 2) {
        uint2 x[2];
#pragma unroll
        for (int e = 0; e < 2; e++) {
          const int i = 4 * (q + e);
          const f32x4 y = {o[d][i] * inv, o[d][i + 1] * inv, o[d][i + 2] * inv, o[d][i + 3] * inv};
          x[e] = __builtin_bit_cast(uint2, __builtin_convertvector(y, V4));
        }
        const auto lo = __builtin_amdgcn_permlane32_swap(x[0].x, x[1].x, false, false);
        const auto hi2 = __builtin_amdgcn_permlane32_swap(x[0].y, x[1].y, false, false);
        const int e = d * 32 + 8 * (q + h);
        if (e < a.D) *(uint4 *)((T *)a.out + orow * a.D + e) = make_uint4(lo[0], hi2[0], lo[1], hi2[1]);
      }
    if (a.lse && h == 0) a.lse[orow] = log_sum(m, l, a.s2, weight_shift<T>(1));
  }
  if (any_bad)
    add_specials<T, PAGED>(a, r, k0, it.seq, it.n > 1 ? it.slot + it.part : -1, R, head, row0, min(n_rows - row0, R),
                           it.lo + (max(all_wg - it.lo, 0) & ~63), hi);
  if (PAGED && it.n > 1) join_parts<T, R>(a, r, it, head, row0, min(n_rows - row0, R), (float *)lds_k[0]);
}

// ------------------------------------------------------------------ host
cf_status check_heads(int H, int Hkv, int D) {
  if (H < 1 || Hkv < 1 || H > 65535 || H % Hkv)
    return set_error(CF_EINVAL, "n_heads %d is not a multiple of n_kv_heads %d", H, Hkv);
  if (D < 8 || D > 256 || D % 8) return set_error(CF_EINVAL, "head_dim %d is not a multiple of 8 in 8..256", D);
  return CF_OK;
}

cf_status check_desc(const cf_attn_desc *d) {
  if (!d) return set_error(CF_EINVAL, "descriptor is NULL");
  if (d->n_seq < 1 || d->n_tok < 0 || d->max_new < 0)
    return set_error(CF_EINVAL, "n_seq %d, n_tok %d, max_new %d", d->n_seq, d->n_tok, d->max_new);
  const cf_status st = check_heads(d->n_heads, d->n_kv_heads, d->head_dim);
  if (st != CF_OK) return st;
  // row numbers are 32-bit and a grid has fewer than 2^24 workgroups of 256 threads
  if ((int64_t)d->n_tok * d->n_heads > 0x7fffffffll ||
      ((int64_t)d->n_tok * d->n_heads / d->n_kv_heads / kRowsSmall + d->n_seq + 4096) * d->n_kv_heads >=
          (1ll << 24))
    return set_error(CF_EINVAL, "n_tok x n_heads or n_seq x n_kv_heads too large");
  return CF_OK;
}

bool few_only(const cf_attn_desc *d) {
  return (int64_t)(d->max_new < d->n_tok ? d->max_new : d->n_tok) * (d->n_heads / d->n_kv_heads) <= kRowsSmall;
}

// The many-row kernel with two groups of four waves, out of step on one CU, or with one
// group (two or three of its workgroups on a CU).  Two are faster on long contexts (one full
// sequence of 16384, 16 heads of 128: 1771 us against 2079), one where the work is in short
// ones (4 x 1024, 32 heads: 56 us against 62) or too little for one workgroup of 256 rows a
// CU (1 x 1024, 32 heads on 8: 25 us against 30); with 64 columns one group is never slower
// (16 images: 52 us against 67; 16384 tokens: 1164 against 1166), with 256 two do not fit the
// registers.  The work counts as long where the mean sequence is, or a longest one that makes a
// quarter of all rows (a chunk of 2048 on 6000 among 100 decodes: 359 us with two groups, 378
// with one).  The packed call does not know its longest sequence and goes by the mean alone
// (8192 tokens among 60 prompts of 100: 558 us with the one group it takes, 517 with two).  A grid
// of 2^23 workgroups of two groups would have 2^32 threads, which no launch takes: one group,
// whose grid the callers' checks bound.
int groups_of(int D, int64_t rows, int64_t longest, int n_seq, int Hkv) {
  if ((rows / (2 * kRowsGroup) + n_seq + 4096) * Hkv >= (1ll << 23)) return 1;
  const bool is_long = rows >= 2048ll * n_seq || (longest >= 4096 && 4 * longest >= rows);
  return D > 64 && D <= 128 && is_long && rows * Hkv >= 192 * 256 ? 2 : 1;
}

template <typename T, bool PAGED>
void launch_many(const AttnArgs &a, int groups, int64_t blocks, hipStream_t s) {
  const dim3 g((unsigned)blocks), b((unsigned)(256 * groups));
  if (a.D <= 64) k_attn_many<T, 4, 2, 64, 1, PAGED><<<g, b, 0, s>>>(a);
  else if (a.D <= 96 && groups == 1) k_attn_many<T, 6, 3, 128, 1, PAGED><<<g, b, 0, s>>>(a);
  else if (a.D <= 96) k_attn_many<T, 6, 3, 128, 2, PAGED><<<g, b, 0, s>>>(a);
  else if (a.D <= 128 && groups == 1) k_attn_many<T, 8, 4, 128, 1, PAGED><<<g, b, 0, s>>>(a);
  else if (a.D <= 128) k_attn_many<T, 8, 4, 128, 2, PAGED><<<g, b, 0, s>>>(a);
  else k_attn_many<T, 16, 8, 256, 1, PAGED><<<g, b, 0, s>>>(a);
}
template <typename T>
void launch_few(const AttnArgs &a, int64_t blocks, hipStream_t s) {
  const dim3 g((unsigned)blocks), b(256);
  if (a.D <= 64) k_attn_few<T, 2, 4, 64><<<g, b, 0, s>>>(a);
  else if (a.D <= 96) k_attn_few<T, 3, 6, 128><<<g, b, 0, s>>>(a);
  else if (a.D <= 128) k_attn_few<T, 4, 8, 128><<<g, b, 0, s>>>(a);
  else k_attn_few<T, 8, 16, 256><<<g, b, 0, s>>>(a);
}
template <typename T>
void launch_paged(const AttnArgs &a, bool few, int groups, hipStream_t s) {
  launch_few<T>(a, (int64_t)a.plan.cap_items[0] * a.Hkv, s);
  if (!few) launch_many<T, true>(a, groups, (int64_t)a.plan.cap_items[1] * a.Hkv, s);
}

// Most keys of a sequence: the kernels' key numbers are 32-bit and run past the last key by the
// tiles whose page ids and rows they fetch ahead (at most 32 x 4 x 33 + 16 keys).
constexpr int64_t kMaxKeys = 0x7fffffffll - 65535;

bool scale_ok(float s) { return s > 0.f && s <= 1e38f; }

}  // namespace

static int desc_groups(const cf_attn_desc *d) {
  const int64_t G = d->n_heads / d->n_kv_heads;
  return groups_of(d->head_dim, d->n_tok * G, (d->max_new < d->n_tok ? d->max_new : d->n_tok) * G, d->n_seq,
                   d->n_kv_heads);
}

// Workgroups of the kernels that run at a time per key/value head, as the plan counts on
// them, and what a part costs beside its keys (measured: starting and joining one takes the
// few-row kernel as long as 64 keys, the many-row kernel as long as 400).
static Split split_of(const cf_attn_desc *d, int kind) {
  const int per_cu = kind ? (desc_groups(d) > 1 || d->head_dim > 128 ? 1 : 2) : (d->head_dim > 128 ? 1 : 2);
  return Split{(256 * per_cu + d->n_kv_heads - 1) / d->n_kv_heads, kind ? 400 : 64, max_parts(kind)};
}

uint64_t plan_view(const cf_attn_desc *d, PlanView *v) {
  const int64_t G = d->n_heads / d->n_kv_heads, rows = (int64_t)d->n_tok * G;
  const bool few = few_only(d);
  uint64_t at = 0;
  char *base = (char *)d->work_dev;
  auto take = [&](uint64_t bytes) {
    char *p = base + at;
    at += (bytes + 255) & ~255ull;
    return p;
  };
  v->hdr = (PlanHdr *)take(sizeof(PlanHdr));
  for (int k = 0; k < 2; k++) {
    const int R = k ? kRowsGroup * desc_groups(d) : kRowsSmall;
    const int64_t parts = 2 * split_of(d, k).n;
    const int64_t with = d->n_seq < d->n_tok ? d->n_seq : d->n_tok;  // requests with new tokens
    // a request has at most floor(rows / R) + 1 tiles; with both kernels in use the few-row
    // one takes requests of one tile
    const int64_t tiles = k == 0 ? (few ? rows / R + with : with) : (few ? 0 : rows / R + with);
    const bool used = k == 0 || !few;
    // parts of a tile: ceil(keys / part) <= 1 + keys / part, and the sum of keys / part over
    // all tiles is at most `parts`; a split tile has at most 2 keys / part
    v->cap_items[k] = used ? (int32_t)(tiles + parts) : 0;
    v->cap_slots[k] = used ? (int32_t)(2 * parts) : 0;
    v->cap_join[k] = used ? (int32_t)parts : 0;
    v->items[k] = (PlanItem *)take(sizeof(PlanItem) * v->cap_items[k]);
    v->done[k] = (int32_t *)take(sizeof(int32_t) * v->cap_join[k] * d->n_kv_heads);
    const uint64_t pr = (uint64_t)v->cap_slots[k] * d->n_kv_heads * R;
    v->ml[k] = (float *)take(pr * 8);
    v->o[k] = (float *)take(pr * d->head_dim * 4);
  }
  return at;
}

}  // namespace cf

extern "C" cf_status cf_attn_plan_bytes(const cf_attn_desc *d, uint64_t *bytes) {
  using namespace cf;
  const cf_status st = check_desc(d);
  if (st != CF_OK) return st;
  if (!bytes) return set_error(CF_EINVAL, "bytes is NULL");
  PlanView v;
  *bytes = plan_view(d, &v);
  return CF_OK;
}

static cf_status check_plan(const cf_attn_desc *d, cf::PlanView *v) {
  using namespace cf;
  const cf_status st = check_desc(d);
  if (st != CF_OK) return st;
  if (!d->q_start_dev || !d->kv_len_dev || !d->work_dev) return set_error(CF_EINVAL, "NULL array");
  if ((uintptr_t)d->work_dev & 15) return set_error(CF_EINVAL, "work_dev is not 16-byte aligned");
  const uint64_t need = plan_view(d, v);
  if (d->work_bytes < need)
    return set_error(CF_EINVAL, "work_bytes %llu, %llu needed", (unsigned long long)d->work_bytes,
                     (unsigned long long)need);
  return CF_OK;
}

extern "C" cf_status cf_attn_plan(const cf_attn_desc *d, void *stream) {
  using namespace cf;
  PlanView v;
  const cf_status st = check_plan(d, &v);
  if (st != CF_OK) return st;
  const auto kernel = d->n_seq <= 256 ? k_attn_plan<256> : k_attn_plan<1024>;
  kernel<<<dim3(1), dim3(d->n_seq <= 256 ? 256 : 1024), 0, as_stream(stream)>>>(
      v, d->q_start_dev, d->kv_len_dev, d->n_seq, d->n_tok, d->n_heads / d->n_kv_heads, d->n_kv_heads,
      few_only(d) ? 1 : 0, desc_groups(d) > 1 ? 8 : 7, split_of(d, 0), split_of(d, 1));
  return hip_check(hipGetLastError(), "cf_attn_plan");
}

extern "C" cf_status cf_attn_paged(const cf_attn_desc *d, const cf_kv_cache *cache, const int32_t *table_dev,
                                   int32_t max_pages, const void *q_dev, int64_t q_tok, int64_t q_head, float scale,
                                   void *out_dev, float *lse_dev, void *stream) {
  using namespace cf;
  AttnArgs a{};
  cf_status st = check_plan(d, &a.plan);
  if (st == CF_OK) st = check_cache(cache);
  if (st != CF_OK) return st;
  if (cache->n_kv_heads != d->n_kv_heads || cache->head_dim != d->head_dim)
    return set_error(CF_EINVAL, "the cache has %d heads of %d, the descriptor %d of %d", cache->n_kv_heads,
                     cache->head_dim, d->n_kv_heads, d->head_dim);
  if (max_pages < 1 || !table_dev) return set_error(CF_EINVAL, "table: max_pages %d", max_pages);
  if ((int64_t)max_pages * cache->page > kMaxKeys)
    return set_error(CF_EINVAL, "table: a row of %d pages of %d is too long", max_pages, cache->page);
  if (!scale_ok(scale)) return set_error(CF_EINVAL, "scale %g is not finite and > 0", (double)scale);
  if (d->n_tok == 0) return CF_OK;
  if (!q_dev || !out_dev) return set_error(CF_EINVAL, "NULL array");
  if ((((uintptr_t)q_dev | (uintptr_t)out_dev) & 15) || ((q_tok | q_head) & 7))
    return set_error(CF_EINVAL, "queries or output are not 16-byte aligned");
  a.q = q_dev; a.k = cache->k_dev; a.v = cache->v_dev;
  a.q_tok = q_tok; a.q_head = q_head;
  a.table = table_dev;
  a.max_pages = max_pages; a.n_pages = cache->n_pages; a.page_log2 = log2_of(cache->page);
  a.n_seq = d->n_seq; a.n_tok = d->n_tok;
  a.H = d->n_heads; a.Hkv = d->n_kv_heads; a.G = a.H / a.Hkv; a.D = d->head_dim; a.causal = 1;
  a.s2 = scale * 1.44269504088896340736f;
  a.out = out_dev; a.lse = lse_dev;
  const hipStream_t s = as_stream(stream);
  if (cache->dtype == CF_BF16) launch_paged<__bf16>(a, few_only(d), desc_groups(d), s);
  else launch_paged<_Float16>(a, few_only(d), desc_groups(d), s);
  return hip_check(hipGetLastError(), "cf_attn_paged");
}

extern "C" cf_status cf_attn_prompt(const cf_attn_seqs *p, float scale, void *out_dev, float *lse_dev, void *stream) {
  using namespace cf;
  if (!p) return set_error(CF_EINVAL, "sequences are NULL");
  if (p->n_seq < 1 || p->n_q < 0 || p->n_k < 0)
    return set_error(CF_EINVAL, "n_seq %d, n_q %d, n_k %d", p->n_seq, p->n_q, p->n_k);
  const cf_status st = check_heads(p->n_heads, p->n_kv_heads, p->head_dim);
  if (st != CF_OK) return st;
  if (p->dtype != CF_BF16 && p->dtype != CF_F16) return set_error(CF_EINVAL, "dtype %d", p->dtype);
  if (!scale_ok(scale)) return set_error(CF_EINVAL, "scale %g is not finite and > 0", (double)scale);
  const int64_t G = p->n_heads / p->n_kv_heads;
  const int groups = groups_of(p->head_dim, p->n_q * G, 0, p->n_seq, p->n_kv_heads);
  const int64_t blocks = ((int64_t)p->n_q * G / (kRowsGroup * groups) + p->n_seq) * p->n_kv_heads;
  if ((int64_t)p->n_q * p->n_heads > 0x7fffffffll || blocks >= (1ll << 24) || p->n_k > kMaxKeys)
    return set_error(CF_EINVAL, "n_q x n_heads, n_seq x n_kv_heads or n_k too large");
  if (p->n_q == 0) return CF_OK;
  if (!p->q_start_dev || !p->k_start_dev || !p->q_dev || !out_dev || (p->n_k > 0 && (!p->k_dev || !p->v_dev)))
    return set_error(CF_EINVAL, "NULL array");
  if (((uintptr_t)p->q_dev | (uintptr_t)p->k_dev | (uintptr_t)p->v_dev | (uintptr_t)out_dev) & 15 ||
      ((p->q_tok | p->q_head | p->k_tok | p->k_head | p->v_tok | p->v_head) & 7))
    return set_error(CF_EINVAL, "queries, keys, values or output are not 16-byte aligned");
  AttnArgs a{};
  a.q = p->q_dev; a.k = p->k_dev; a.v = p->v_dev;
  a.q_tok = p->q_tok; a.q_head = p->q_head; a.k_tok = p->k_tok; a.k_head = p->k_head;
  a.v_tok = p->v_tok; a.v_head = p->v_head;
  a.q_start = p->q_start_dev; a.kv = p->k_start_dev;
  a.n_seq = p->n_seq; a.n_tok = p->n_q; a.n_k = p->n_k;
  a.H = p->n_heads; a.Hkv = p->n_kv_heads; a.G = (int)G; a.D = p->head_dim; a.causal = p->causal != 0;
  a.s2 = scale * 1.44269504088896340736f;
  a.out = out_dev; a.lse = lse_dev;
  const hipStream_t s = as_stream(stream);
  if (p->dtype == CF_BF16) launch_many<__bf16, false>(a, groups, blocks, s);
  else launch_many<_Float16, false>(a, groups, blocks, s);
  return hip_check(hipGetLastError(), "cf_attn_prompt");
}
