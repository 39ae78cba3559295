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
// instruction's operand (relative error at most 2^-8 in bf16, 2^-11 in fp16,
// as the output's own rounding).
//
// A key that a row does not see has p_k = 0, but 0 times an infinity or a NaN
// in its value would still reach the row.  Values past a sequence's keys are
// loaded as zeros; in a tile that only some of a workgroup's rows see, such
// values are zeroed on their way to LDS, and at the end, if there were any,
// added to the rows that see them (which makes those outputs infinite or NaN).
#include "cf_attn.h"

namespace cf {

__device__ const i32x4 g_zero16 = {0, 0, 0, 0};

bool page_ok(int page);
cf_status check_cache(const cf_kv_cache *c);

namespace {

__host__ __device__ inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

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
__device__ __forceinline__ int64_t block_sum(int64_t x, int64_t *lds) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nw = blockDim.x >> 6;
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  __syncthreads();
  if (lane == 0) lds[w] = x;
  __syncthreads();
  int64_t s = 0;
  for (int i = 0; i < nw; i++) s += lds[i];
  return s;
}
__device__ __forceinline__ int64_t block_before(int64_t x, int64_t *lds, int64_t &total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nw = blockDim.x >> 6;
  int64_t incl = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up(incl, o);
    if (lane >= o) incl += y;
  }
  __syncthreads();
  if (lane == 63) lds[w] = incl;
  __syncthreads();
  int64_t before = incl - x;
  total = 0;
  for (int i = 0; i < nw; i++) {
    if (i < w) before += lds[i];
    total += lds[i];
  }
  return before;
}

constexpr int kPlanThreads = 1024;

// One workgroup.  Pass 1 sums the work of either kernel, (row tiles) x (keys),
// which gives the keys of a part; pass 2 takes 1024 requests at a time, places
// their items by a scan and writes them, a thread per item.
__global__ __launch_bounds__(kPlanThreads) void k_attn_plan(PlanView v, const int32_t *q_start, const int32_t *kv_len,
                                                            int n_seq, int n_tok, int G, int Hkv, int few_only) {
  __shared__ int64_t red[kPlanThreads / 64];
  __shared__ int64_t l_at[kPlanThreads], l_slot[kPlanThreads], l_join[kPlanThreads];
  __shared__ int l_n[kPlanThreads];
  const int tid = threadIdx.x;
  auto load = [&](int i, int &tiles, int &kind, int &keys) {
    const int q0 = clampi(q_start[i], 0, n_tok), n = max(clampi(q_start[i + 1], 0, n_tok) - q0, 0);
    const int64_t rows = (int64_t)n * G;
    kind = (!few_only && rows > kRowsSmall) ? 1 : 0;
    tiles = (int)ceil_div(rows, kind ? kRowsBig : kRowsSmall);
    keys = max(kv_len[i], 0);
  };
  int64_t w0 = 0, w1 = 0;
  for (int i = tid; i < n_seq; i += kPlanThreads) {
    int tiles, kind, keys;
    load(i, tiles, kind, keys);
    (kind ? w1 : w0) += (int64_t)tiles * keys;
  }
  w0 = block_sum(w0, red);
  w1 = block_sum(w1, red);
  int part[2];
  for (int k = 0; k < 2; k++) {
    const int64_t target = ceil_div(k ? kPartsBig : kPartsSmall, Hkv);
    const int64_t p = ceil_div(k ? w1 : w0, target);
    part[k] = (int)min((int64_t)(1 << 30), ceil_div(max(p, (int64_t)kMinPart), 128) * 128);
  }
  // 64-bit: starts that do not ascend could name more rows than there are
  int64_t at[2] = {0, 0}, slots[2] = {0, 0}, joins[2] = {0, 0};
  for (int c0 = 0; c0 < n_seq; c0 += kPlanThreads) {
    const int i = c0 + tid, cn = min(kPlanThreads, n_seq - c0);
    int tiles = 0, kind = 0, keys = 0, parts = 1;
    if (i < n_seq) {
      load(i, tiles, kind, keys);
      parts = max((int)ceil_div(keys, part[kind]), 1);
    }
    for (int k = 0; k < 2; k++) {
      const bool mine = kind == k && tiles > 0;
      const int64_t items = mine ? (int64_t)tiles * parts : 0;
      int64_t n, ns, nj;
      l_n[tid] = mine ? parts : 0;
      l_at[tid] = block_before(items, red, n);
      l_slot[tid] = block_before(parts > 1 ? items : 0, red, ns);
      l_join[tid] = block_before(mine && parts > 1 ? tiles : 0, red, nj);
      __syncthreads();
      const int64_t room = v.cap_items[k] - at[k];
      for (int64_t x = tid; x < min(n, room); x += kPlanThreads) {
        int lo = 0, hi = cn;  // the last request with items that starts at or before item x
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (l_at[mid] <= x) lo = mid; else hi = mid;
        }
        const int p = max(l_n[lo], 1);
        const int64_t rest = x - l_at[lo];
        const int tile = (int)(rest / p), pi = (int)(rest - (int64_t)tile * p);
        const int64_t slot = p > 1 ? slots[k] + l_slot[lo] + rest : -1;
        const int64_t join = joins[k] + l_join[lo] + tile;
        if (slot + p > v.cap_slots[k] + pi) continue;
        v.items[k][at[k] + x] = PlanItem{c0 + lo, tile, pi * part[k], (int)slot};
        if (p > 1 && pi == 0 && join < v.cap_join[k]) v.join[k][join] = PlanJoin{c0 + lo, tile, (int)slot, p};
      }
      __syncthreads();
      at[k] += n; slots[k] += ns; joins[k] += nj;
    }
  }
  if (tid < 2) {
    v.hdr->n_items[tid] = (int)min(at[tid], (int64_t)v.cap_items[tid]);
    v.hdr->n_join[tid] = (int)min(joins[tid], (int64_t)v.cap_join[tid]);
    v.hdr->part[tid] = part[tid];
  }
}

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

// The infinities and NaN among the values of keys [from, to), which only some
// of the rows row0 .. row0 + n - 1 see, added to the results just written.
template <typename T, bool PAGED>
__device__ __forceinline__ void add_specials(const AttnArgs &a, const Rows &r, int k0, int seq, int slot, int kind,
                                             int head, int64_t row0, int n, int from, int to) {
  __syncthreads();
#pragma unroll 1
  for (int x = threadIdx.x; x < n * a.D; x += 256) {
    const int rr = x / a.D, e = x - rr * a.D;
    const int64_t row = row0 + rr;
    const int j = (int)(row / a.G), g = (int)(row - (int64_t)j * a.G);
    const int last = min(r.nk - r.nq + j, to - 1);
    float sum = 0.f;
#pragma unroll 1
    for (int key = from; key <= last; key++) {
      T v = (T)0.f;
      if (PAGED) {
        const int id = a.table[(int64_t)seq * a.max_pages + (key >> a.page_log2)];
        if ((unsigned)id < (unsigned)a.n_pages)
          v = ((const T *)a.v)[((((int64_t)id * a.Hkv + head) << a.page_log2) + (key & ((1 << a.page_log2) - 1))) * a.D + e];
      } else {
        v = ((const T *)a.v)[(int64_t)(k0 + key) * a.v_tok + head * a.v_head + e];
      }
      if (special<T>(v)) sum += (float)v;
    }
    if (sum == 0.f) continue;
    if (slot >= 0) {
      const int R = kind ? kRowsBig : kRowsSmall;
      a.plan.o[kind][(((int64_t)slot * a.Hkv + head) * R + rr) * a.D + e] += sum;
    } else {
      T *p = (T *)a.out + ((int64_t)(r.q0 + j) * a.H + head * a.G + g) * a.D + e;
      *p = (T)((float)*p + sum);
    }
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
template <typename T, int KS, int DB, int DS>
__global__ __launch_bounds__(256, DS > 128 ? 1 : 2) void k_attn_few(AttnArgs a) {
  using V8 = typename Elem<T>::v8;
  using V4 = typename Elem<T>::v4;
  constexpr int CH = DS / 8, NV = 32 * CH / 64;
  __shared__ __attribute__((aligned(16))) char lds[4][32 * DS * 2];
  __shared__ float l_m[4][16], l_l[4][16];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = (int)(blockIdx.x % (unsigned)a.Hkv), item = (int)(blockIdx.x / (unsigned)a.Hkv);
  if (item >= min(a.plan.hdr->n_items[0], a.plan.cap_items[0])) return;
  const PlanItem it = a.plan.items[0][item];
  if ((unsigned)it.seq >= (unsigned)a.n_seq || it.tile < 0 || it.lo < 0 || it.slot >= a.plan.cap_slots[0]) return;
  int k0;
  const Rows r = rows_of<true>(a, it.seq, k0);
  const int n_rows = r.nq * a.G, row0 = it.tile * kRowsSmall;
  if (row0 >= n_rows) return;
  const int row = row0 + (lane & 15), j = min(row, n_rows - 1) / a.G, g = min(row, n_rows - 1) - j * a.G;
  const int last_j = (min(row0 + kRowsSmall, n_rows) - 1) / a.G;
  const int seen = r.nk - r.nq + last_j + 1;  // keys the tile's last row sees
  const int hi = __builtin_amdgcn_readfirstlane(
      min(seen, it.slot >= 0 ? it.lo + a.plan.hdr->part[0] : 0x7fffffff));
  const int lim = r.nk - r.nq + j;  // last key the lane's row sees
  const int all = r.nk - r.nq + row0 / a.G + 1;  // keys that every row sees

  const int gq = lane >> 4;
  V8 qf[KS];
  const T *qp = (const T *)a.q + (int64_t)(r.q0 + j) * a.q_tok + (int64_t)(head * a.G + g) * a.q_head;
#pragma unroll
  for (int ks = 0; ks < KS; ks++) {
    const int c = ks * 4 + gq;
    qf[ks] = *(const V8 *)(c * 8 < a.D ? (const void *)(qp + c * 8) : (const void *)&g_zero16);
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
        kr[b][ks] = *(const V8 *)(ok ? (const void *)(kc + base[b] + key * a.D + c * 8) : (const void *)&g_zero16);
      }
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int x = i * 64 + lane, key = x / CH, c = x % CH, b = (i * 64 / CH) >> 4;
      const bool ok = (key & 15) < valid[b] && c * 8 < a.D;
      vr[i] = *(const i32x4 *)(ok ? (const void *)(vc + base[b] + (key & 15) * a.D + c * 8) : (const void *)&g_zero16);
    }
  };

  if (w < n_tiles) load(0);
  for (int n = 0; w + 4 * n < n_tiles; n++) {
    const int t0 = it.lo + 32 * (w + 4 * n);
    if (t0 + 32 > all && seen > all) {
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
    const float alpha = exp2_hw(fmaf(m, a.s2, -mu));
    m = mn;
    V8 pf;
    float ps = 0.f;
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const float p = exp2_hw(fmaf(s[b][i], a.s2, -mu));
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
    if (it.slot >= 0) {
      const int64_t pr = ((int64_t)it.slot * a.Hkv + head) * kRowsSmall + rr;
      *(f32x4 *)(a.plan.o[0] + pr * a.D + d4 * 4) = oo;
      if (d4 == 0) { a.plan.ml[0][pr * 2] = mm; a.plan.ml[0][pr * 2 + 1] = ll; }
    } else {
      const int jj = (row0 + rr) / a.G, gg = row0 + rr - jj * a.G;
      const int64_t orow = (int64_t)(r.q0 + jj) * a.H + head * a.G + gg;
      const float inv = ll > 0.f || ll != ll ? 1.f / ll : 0.f;
      *(V4 *)((T *)a.out + orow * a.D + d4 * 4) = __builtin_convertvector(oo * inv, V4);
      if (a.lse && d4 == 0) a.lse[orow] = ll == 0.f ? kNegInf : (mm * a.s2 + __log2f(ll)) * 0.69314718055994531f;
    }
  }
  if (any_bad)
    add_specials<T, true>(a, r, 0, it.seq, it.slot, 0, head, row0, min(n_rows - row0, kRowsSmall),
                          it.lo + (max(all - it.lo, 0) & ~31), hi);
}

// ------------------------------------------------------------------ many rows
// A workgroup of four waves takes 128 rows of one key/value head, 32 a wave,
// and tiles of 64 keys.  Keys and values go through registers to LDS, the next
// tile's loads in flight while one is worked on.  S^T = K Q^T (32 keys x 32
// rows a matrix instruction), so a lane has 32 scores of one row, and O^T =
// V^T P^T as in the few-row kernel: the order of the keys within a step is the
// order in which S^T leaves them in the lane, the values' operand is read to
// match, and no probability changes lanes.
template <typename T, int KS, int DB, int DS, bool PAGED>
__global__ __launch_bounds__(256, DS > 128 ? 1 : 2) void k_attn_many(AttnArgs a) {
  using V8 = typename Elem<T>::v8;
  using V4 = typename Elem<T>::v4;
  constexpr int CH = DS / 8, NL = 64 * CH / 256;
  __shared__ __attribute__((aligned(16))) T lds[2][2][64 * DS];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = (int)(blockIdx.x % (unsigned)a.Hkv), item = (int)(blockIdx.x / (unsigned)a.Hkv);
  PlanItem it;
  if (PAGED) {
    if (item >= min(a.plan.hdr->n_items[1], a.plan.cap_items[1])) return;
    it = a.plan.items[1][item];
    if ((unsigned)it.seq >= (unsigned)a.n_seq || it.tile < 0 || it.lo < 0 || it.slot >= a.plan.cap_slots[1]) return;
  } else {
    // sequence i owns the tiles from floor(first row / 128) + i on; 64 probes at a time
    auto start = [&](int i) { return (int)((int64_t)clampi(a.q_start[i], 0, a.n_tok) * a.G / kRowsBig) + i; };
    int lo = 0, n = a.n_seq;
    while (n > 1) {
      const int step = (n + 63) >> 6, i = lo + lane * step;
      const bool le = lane * step < n && start(i) <= item;
      const int cnt = __builtin_popcountll(__ballot(le));
      const int skip = cnt > 0 ? (cnt - 1) * step : 0;
      lo += skip;
      n = min(step, n - skip);
    }
    it.seq = __builtin_amdgcn_readfirstlane(lo);
    it.tile = item - __builtin_amdgcn_readfirstlane(start(lo));
    it.lo = 0;
    it.slot = -1;
  }
  int k0;
  const Rows r = rows_of<PAGED>(a, it.seq, k0);
  const int64_t n_rows = (int64_t)r.nq * a.G;
  const int n_rt = (int)ceil_div(n_rows, kRowsBig);
  if (it.tile < 0 || it.tile >= n_rt) return;
  // the rows that see most keys first
  const int64_t row0 = (int64_t)(n_rt - 1 - it.tile) * kRowsBig;
  const int64_t row = row0 + w * 32 + (lane & 31);
  const int64_t rc = min(row, n_rows - 1);
  const int j = (int)(rc / a.G), g = (int)(rc - (int64_t)j * a.G);
  const int off = (PAGED || a.causal) ? r.nk - r.nq : r.nk;  // row j sees keys up to off + j, or all
  const int last_j = (int)((min(row0 + kRowsBig, n_rows) - 1) / a.G);
  const int seen = (PAGED || a.causal) ? min(off + last_j + 1, r.nk) : r.nk;
  const int hi = __builtin_amdgcn_readfirstlane(
      min(seen, it.slot >= 0 ? it.lo + a.plan.hdr->part[1] : 0x7fffffff));
  const int lim = min((PAGED || a.causal) ? off + j : r.nk - 1, hi - 1);
  // keys that every row of the wave sees need no mask
  const int64_t wrow = min(row0 + w * 32, n_rows - 1);
  const int all = __builtin_amdgcn_readfirstlane(
      min((PAGED || a.causal) ? off + (int)(wrow / a.G) + 1 : r.nk, hi));
  const int all_wg = (PAGED || a.causal) ? off + (int)(row0 / a.G) + 1 : r.nk;  // and of the workgroup
  const int h = lane >> 5;

  V8 qf[KS];
  const T *qp = (const T *)a.q + (int64_t)(r.q0 + j) * a.q_tok + (int64_t)(head * a.G + g) * a.q_head;
#pragma unroll
  for (int ks = 0; ks < KS; ks++) {
    const int c = ks * 2 + h;
    qf[ks] = *(const V8 *)(c * 8 < a.D ? (const void *)(qp + c * 8) : (const void *)&g_zero16);
  }

  const int64_t page_elems = (int64_t)a.Hkv * a.D << a.page_log2;
  const int64_t head_off = (int64_t)head * a.D << a.page_log2;
  const T *kc = (const T *)a.k + (PAGED ? head_off : (int64_t)k0 * a.k_tok + head * a.k_head);
  const T *vc = (const T *)a.v + (PAGED ? head_off : (int64_t)k0 * a.v_tok + head * a.v_head);
  const int page_mask = (1 << a.page_log2) - 1;
  const int32_t *trow = PAGED ? a.table + (int64_t)it.seq * a.max_pages : nullptr;
  const int n_tiles = hi > it.lo ? (hi - it.lo + 63) >> 6 : 0;

  f32x16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; d++)
#pragma unroll
    for (int i = 0; i < 16; i++) o[d][i] = 0.f;
  float m = kNegInf, l = 0.f;
  i32x4 kr[NL], vr[NL];
  int ids = 0;
  bool bad = false;

  auto load = [&](int n) {
    const int t0 = it.lo + 64 * n;
    if (PAGED && (n & 15) == 0) {  // page ids of 16 tiles across the lanes, one per 16 keys
      const int key = t0 + 16 * lane;
      ids = key < hi ? trow[key >> a.page_log2] : -1;
    }
#pragma unroll
    for (int i = 0; i < NL; i++) {
      const int x = i * 256 + tid, rr = x / CH, c = x % CH;
      const void *kp, *vp;
      if (PAGED) {
        const int grp = __builtin_amdgcn_readfirstlane(rr >> 4);
        const int id = __builtin_amdgcn_readlane(ids, ((n & 15) << 2) + grp);
        const bool in = (unsigned)id < (unsigned)a.n_pages;
        const int64_t base = (in ? id : 0) * page_elems + (int64_t)((t0 + 16 * grp) & page_mask) * a.D;
        const bool ok = in && t0 + rr < r.nk && c * 8 < a.D;
        const int e = (rr & 15) * a.D + c * 8;
        kp = ok ? (const void *)(kc + base + e) : (const void *)&g_zero16;
        vp = ok ? (const void *)(vc + base + e) : (const void *)&g_zero16;
      } else {
        const bool ok = t0 + rr < r.nk && c * 8 < a.D;
        kp = ok ? (const void *)(kc + (int64_t)(t0 + rr) * a.k_tok + c * 8) : (const void *)&g_zero16;
        vp = ok ? (const void *)(vc + (int64_t)(t0 + rr) * a.v_tok + c * 8) : (const void *)&g_zero16;
      }
      kr[i] = *(const i32x4 *)kp;
      vr[i] = *(const i32x4 *)vp;
    }
  };
  auto store = [&](int n) {
    const int b = n & 1;
    if (it.lo + 64 * (n + 1) > all_wg && seen > all_wg) {
#pragma unroll
      for (int i = 0; i < NL; i++) bad |= take_specials<T>(vr[i]);
    }
#pragma unroll
    for (int i = 0; i < NL; i++) {
      const int x = i * 256 + tid, rr = x / CH, c = x % CH, at = rr * DS + (c ^ swz<DS>(rr)) * 8;
      *(i32x4 *)(&lds[b][0][at]) = kr[i];
      *(i32x4 *)(&lds[b][1][at]) = vr[i];
    }
  };

  if (n_tiles > 0) {
    load(0);
    store(0);
  }
  __syncthreads();
  for (int n = 0; n < n_tiles; n++) {
    const int t0 = it.lo + 64 * n;
    if (n + 1 < n_tiles) load(n + 1);
    const T *kt = lds[n & 1][0], *vt = lds[n & 1][1];
    f32x16 s[2];
#pragma unroll
    for (int b = 0; b < 2; b++) {
#pragma unroll
      for (int i = 0; i < 16; i++) s[b][i] = 0.f;
      const int rr = b * 32 + (lane & 31);
#pragma unroll
      for (int ks = 0; ks < KS; ks++) {
        const V8 kf = *(const V8 *)(kt + rr * DS + (((ks * 2 + h) ^ swz<DS>(rr)) * 8));
        s[b] = Elem<T>::mma32(kf, qf[ks], s[b]);
      }
    }
    if (t0 + 64 > all) {
#pragma unroll
      for (int b = 0; b < 2; b++)
#pragma unroll
        for (int i = 0; i < 16; i++) {
          const int key = t0 + b * 32 + 8 * (i >> 2) + 4 * h + (i & 3);
          s[b][i] = key <= lim ? s[b][i] : kNegInf;
        }
    }
    float mx = kNegInf;
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
      for (int i = 0; i < 16; i++) mx = fmaxf(mx, s[b][i]);
    mx = max_halves(mx);
    const float mn = fmaxf(m, mx), mu = mn == kNegInf ? 0.f : mn * a.s2;
    const float alpha = exp2_hw(fmaf(m, a.s2, -mu));
    m = mn;
    V8 pf[4];
    float ps = 0.f;
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
      for (int i = 0; i < 16; i++) {
        const float p = exp2_hw(fmaf(s[b][i], a.s2, -mu));
        ps += p;
        pf[b * 2 + (i >> 3)][i & 7] = (T)p;
      }
    l = fmaf(l, alpha, ps);
#pragma unroll
    for (int d = 0; d < DB; d++) o[d] = o[d] * alpha;
    const int vcol = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
#pragma unroll
    for (int k = 0; k < 4; k++) {
      const int vrow = k * 16 + 4 * h + ((lane & 15) >> 2);
#pragma unroll
      for (int d = 0; d < DB; d++) {
        const int c = d * 4 + (vcol >> 3), of = vcol & 7;
        const V4 lo4 = read_tr<T>(vt + vrow * DS + (c ^ swz<DS>(vrow)) * 8 + of);
        const V4 hi4 = read_tr<T>(vt + (vrow + 8) * DS + (c ^ swz<DS>(vrow + 8)) * 8 + of);
        o[d] = Elem<T>::mma32(join8<V8>(lo4, hi4), pf[k], o[d]);
      }
    }
    if (n + 1 < n_tiles) store(n + 1);
    __syncthreads();
  }
  l = sum_halves(l);
  const int any_bad = __syncthreads_or(bad);
  if (row < n_rows && it.slot >= 0) {
    const int64_t pr = ((int64_t)it.slot * a.Hkv + head) * kRowsBig + w * 32 + (lane & 31);
#pragma unroll
    for (int d = 0; d < DB; d++)
#pragma unroll
      for (int q = 0; q < 4; q++) {
        const int e = d * 32 + 8 * q + 4 * h;
        if (e < a.D)
          *(f32x4 *)(a.plan.o[1] + pr * a.D + e) = f32x4{o[d][4 * q], o[d][4 * q + 1], o[d][4 * q + 2], o[d][4 * q + 3]};
      }
    if (h == 0) { a.plan.ml[1][pr * 2] = m; a.plan.ml[1][pr * 2 + 1] = l; }
  } else if (row < n_rows) {
    const int64_t orow = (int64_t)(r.q0 + j) * a.H + head * a.G + g;
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
    for (int d = 0; d < DB; d++)
#pragma unroll
      for (int q = 0; q < 4; q++) {
        const int e = d * 32 + 8 * q + 4 * h;
        const f32x4 x = {o[d][4 * q] * inv, o[d][4 * q + 1] * inv, o[d][4 * q + 2] * inv, o[d][4 * q + 3] * inv};
        if (e < a.D) *(V4 *)((T *)a.out + orow * a.D + e) = __builtin_convertvector(x, V4);
      }
    if (a.lse && h == 0) a.lse[orow] = l == 0.f ? kNegInf : (m * a.s2 + __log2f(l)) * 0.69314718055994531f;
  }
  if (any_bad)
    add_specials<T, PAGED>(a, r, k0, it.seq, it.slot, 1, head, row0, (int)min(n_rows - row0, (int64_t)kRowsBig),
                           it.lo + (max(all_wg - it.lo, 0) & ~63), hi);
}

// ------------------------------------------------------------------ join of split contexts
// A workgroup per (split rows, key/value head); its parts are added in key order.
template <typename T>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a, int kind) {
  using V4 = typename Elem<T>::v4;
  const int head = (int)(blockIdx.x % (unsigned)a.Hkv), x = (int)(blockIdx.x / (unsigned)a.Hkv);
  if (x >= min(a.plan.hdr->n_join[kind], a.plan.cap_join[kind])) return;
  const PlanJoin jn = a.plan.join[kind][x];
  if ((unsigned)jn.seq >= (unsigned)a.n_seq || jn.tile < 0 || jn.slot < 0 || jn.n > a.plan.cap_slots[kind] - jn.slot)
    return;
  const int R = kind ? kRowsBig : kRowsSmall;
  int k0;
  const Rows r = rows_of<true>(a, jn.seq, k0);
  const int64_t n_rows = (int64_t)r.nq * a.G;
  const int n_rt = (int)ceil_div(n_rows, R);
  if (jn.tile >= n_rt) return;
  const int64_t row0 = (int64_t)(kind ? n_rt - 1 - jn.tile : jn.tile) * R;
  const int quads = a.D / 4;
  for (int y = threadIdx.x; y < R * quads; y += 256) {
    const int rr = y / quads, d4 = y - rr * quads;
    if (row0 + rr >= n_rows) break;
    float mm = kNegInf;
    for (int p = 0; p < jn.n; p++)
      mm = fmaxf(mm, a.plan.ml[kind][((((int64_t)jn.slot + p) * a.Hkv + head) * R + rr) * 2]);
    const float mu = mm == kNegInf ? 0.f : mm;
    float ll = 0.f;
    f32x4 oo = {0, 0, 0, 0};
    for (int p = 0; p < jn.n; p++) {
      const int64_t pr = (((int64_t)jn.slot + p) * a.Hkv + head) * R + rr;
      const float f = exp2_hw((a.plan.ml[kind][pr * 2] - mu) * a.s2);
      ll = fmaf(f, a.plan.ml[kind][pr * 2 + 1], ll);
      oo += *(const f32x4 *)(a.plan.o[kind] + pr * a.D + d4 * 4) * f;
    }
    const int j = (int)((row0 + rr) / a.G), g = (int)(row0 + rr - (int64_t)j * a.G);
    const int64_t orow = (int64_t)(r.q0 + j) * a.H + head * a.G + g;
    const float inv = ll > 0.f || ll != ll ? 1.f / ll : 0.f;
    *(V4 *)((T *)a.out + orow * a.D + d4 * 4) = __builtin_convertvector(oo * inv, V4);
    if (a.lse && d4 == 0) a.lse[orow] = ll == 0.f ? kNegInf : (mm * a.s2 + __log2f(ll)) * 0.69314718055994531f;
  }
}

// ------------------------------------------------------------------ host
int log2_of(int x) { return 31 - __builtin_clz((unsigned)x); }

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
  // row numbers are 32-bit and a grid has at most 2^24 - 1 workgroups of 256 threads
  if ((int64_t)d->n_tok * d->n_heads > 0x7fffffffll ||
      ((int64_t)d->n_tok * d->n_heads / d->n_kv_heads / kRowsSmall + d->n_seq + 2 * kPartsSmall) * d->n_kv_heads >=
          (1ll << 24))
    return set_error(CF_EINVAL, "n_tok x n_heads or n_seq x n_kv_heads too large");
  return CF_OK;
}

bool few_only(const cf_attn_desc *d) {
  return (int64_t)(d->max_new < d->n_tok ? d->max_new : d->n_tok) * (d->n_heads / d->n_kv_heads) <= kRowsSmall;
}

template <typename T, bool PAGED>
void launch_many(const AttnArgs &a, int64_t blocks, hipStream_t s) {
  const dim3 g((unsigned)blocks), b(256);
  if (a.D <= 64) k_attn_many<T, 4, 2, 64, PAGED><<<g, b, 0, s>>>(a);
  else if (a.D <= 96) k_attn_many<T, 6, 3, 128, PAGED><<<g, b, 0, s>>>(a);
  else if (a.D <= 128) k_attn_many<T, 8, 4, 128, PAGED><<<g, b, 0, s>>>(a);
  else k_attn_many<T, 16, 8, 256, PAGED><<<g, b, 0, s>>>(a);
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
void launch_paged(const AttnArgs &a, bool few, hipStream_t s) {
  launch_few<T>(a, (int64_t)a.plan.cap_items[0] * a.Hkv, s);
  k_attn_join<T><<<dim3((unsigned)(a.plan.cap_join[0] * a.Hkv)), dim3(256), 0, s>>>(a, 0);
  if (few) return;
  launch_many<T, true>(a, (int64_t)a.plan.cap_items[1] * a.Hkv, s);
  k_attn_join<T><<<dim3((unsigned)(a.plan.cap_join[1] * a.Hkv)), dim3(256), 0, s>>>(a, 1);
}

bool scale_ok(float s) { return s > 0.f && s <= 1e38f; }

}  // namespace

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
    const int R = k ? kRowsBig : kRowsSmall;
    const int64_t parts = ceil_div(k ? kPartsBig : kPartsSmall, d->n_kv_heads);
    const int64_t with = d->n_seq < d->n_tok ? d->n_seq : d->n_tok;  // requests with new tokens
    // a request has at most floor(rows / R) + 1 tiles; with both kernels in use the few-row
    // one takes requests of one tile
    int64_t tiles = k == 0 ? (few ? rows / R + with : with) : (few ? 0 : rows / R + with);
    const bool used = k == 0 || !few;
    // parts of a tile: ceil(keys / part) <= 1 + keys / part, and the sum of keys / part over
    // all tiles is at most `parts`; a split tile has at most 2 keys / part
    v->cap_items[k] = used ? (int32_t)(tiles + parts) : 0;
    v->cap_slots[k] = used ? (int32_t)(2 * parts) : 0;
    v->cap_join[k] = used ? (int32_t)parts : 0;
    v->items[k] = (PlanItem *)take(sizeof(PlanItem) * v->cap_items[k]);
    v->join[k] = (PlanJoin *)take(sizeof(PlanJoin) * v->cap_join[k]);
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
  k_attn_plan<<<dim3(1), dim3(kPlanThreads), 0, as_stream(stream)>>>(
      v, d->q_start_dev, d->kv_len_dev, d->n_seq, d->n_tok, d->n_heads / d->n_kv_heads, d->n_kv_heads,
      few_only(d) ? 1 : 0);
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
  if (!scale_ok(scale)) return set_error(CF_EINVAL, "scale %g is not finite and > 0", (double)scale);
  if (d->n_tok == 0) return CF_OK;
  if (!q_dev || !out_dev) return set_error(CF_EINVAL, "NULL array");
  if ((((uintptr_t)q_dev | (uintptr_t)out_dev) & 15) || ((q_tok | q_head) & 7))
    return set_error(CF_EINVAL, "queries or output are not 16-byte aligned");
  a.q = q_dev; a.k = cache->k_dev; a.v = cache->v_dev;
  a.q_tok = q_tok; a.q_head = q_head;
  a.q_start = d->q_start_dev; a.kv = d->kv_len_dev; a.table = table_dev;
  a.max_pages = max_pages; a.n_pages = cache->n_pages; a.page_log2 = log2_of(cache->page);
  a.n_seq = d->n_seq; a.n_tok = d->n_tok;
  a.H = d->n_heads; a.Hkv = d->n_kv_heads; a.G = a.H / a.Hkv; a.D = d->head_dim; a.causal = 1;
  a.s2 = scale * 1.44269504088896340736f;
  a.out = out_dev; a.lse = lse_dev;
  const hipStream_t s = as_stream(stream);
  if (cache->dtype == CF_BF16) launch_paged<__bf16>(a, few_only(d), s);
  else launch_paged<_Float16>(a, few_only(d), s);
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
  const int64_t blocks = ((int64_t)p->n_q * G / kRowsBig + p->n_seq) * p->n_kv_heads;
  if ((int64_t)p->n_q * p->n_heads > 0x7fffffffll || blocks >= (1ll << 24))
    return set_error(CF_EINVAL, "n_q x n_heads or n_seq x n_kv_heads too large");
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
  if (p->dtype == CF_BF16) launch_many<__bf16, false>(a, blocks, s);
  else launch_many<_Float16, false>(a, blocks, s);
  return hip_check(hipGetLastError(), "cf_attn_prompt");
}
