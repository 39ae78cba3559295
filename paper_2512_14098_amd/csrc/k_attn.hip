// k_attn.hip -- attention of new tokens over the paged cache and of whole
// packed sequences: the plan, the few-row kernel over a 16-bit cache, the calls.  The
// mathematics, the many-row kernel and what caches of either width share are in
// cf_attn_kern.h, the few-row kernel over an 8-bit cache in cf_attn_few8.h.
#include "cf_attn_few8.h"

namespace cf {

bool page_ok(int page);
cf_status check_cache(const cf_kv_cache *c);
cf_status check_cache8(const cf_kv_cache8 *c);

namespace {

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
// workgroups and half a part of tail, whichever is less, and `start` keys for starting a
// part.  Where some context is split, `join` keys for joining at all and `part` for storing and reading
// the result of each part, less where tiles are not full: only rows that there are have one.
struct Split {
  int n, start, part, join, max_parts;
};

constexpr int kClasses = 18;  // of requests, by the length of their parts

// One workgroup.  Pass 1 sums the work of either kernel, (row tiles) x (keys), and the
// parts that each candidate length gives; pass 2 takes NT requests at a time, places their
// items by a scan and writes them, a thread per item.  Bound by the latency of its few
// steps (4 to 16 requests 6 us, 64 7 us, 256 8 to 10; with 64-bit divisions and a scan for each count 17), so that 256
// threads do better than 1024 as long as one step takes all requests.
template <int NT>
__global__ __launch_bounds__(NT) void k_attn_plan(PlanView v, const int32_t *q_start, const int32_t *kv_len, int n_seq,
                                                  int n_tok, int G, int Hkv, int few_only, int big_log2, Split sp0,
                                                  Split sp1) {
  __shared__ float red[NT / 64][8];
  __shared__ int64_t red64[NT / 64];
  __shared__ int64_t l_at[NT];
  __shared__ int l_n[NT], l_rows[NT][3], l_seq[NT], l_tiles[NT], l_parts[NT], l_cls[NT / 64][kClasses];
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
  for (int i = tid; i < v.cap_join[0] * Hkv; i += NT) v.done[0][i] = 0;
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
    const int least = max(min_part(k), (int)(w[2 + k] * 1.001f) / sp.max_parts + 2);
#pragma unroll
    for (int c = 0; c < 3; c++) {
      const float even = c == 0 ? 0x1p30f : fminf(w[k] * 1.001f / (float)(sp.n * c) + 1.f, 0x1p30f);
      len[k][c] = (max((int)even, least) + 127) & ~127;
    }
  }
  float n[7] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};  // parts of either kernel's candidates; rows of the many-row kernel
  for (int i = tid; i < n_seq; i += NT) {
    int tiles = tiles0, kind = kind0, keys = keys0;
    if (i != tid) load(i, tiles, kind, keys);
#pragma unroll
    for (int c = 0; c < 3; c++) {
      const float t = (float)tiles * fmaxf(ceilf((float)keys / (float)(kind ? len[1][c] : len[0][c])), 1.f);
      n[c] += kind ? 0.f : t;
      n[3 + c] += kind ? t : 0.f;
    }
    n[6] += kind ? (float)(i == tid ? first_nq : nq) * (float)G : 0.f;
  }
  if (few_only) {  // a decode step's: the other sums are zero
    float few[3] = {n[0], n[1], n[2]};
    block_reduce<NT, 3, 0>(few, red);
#pragma unroll
    for (int c = 0; c < 3; c++) n[c] = few[c];
  } else {
    block_reduce<NT, 7, 0>(n, red);
  }
  const float full = n[6] / fmaxf(n[3] * (float)(1 << big_log2), 1.f);  // of the rows of the many-row kernel's tiles
  int part[2];
#pragma unroll
  for (int k = 0; k < 2; k++) {
    const Split sp = k ? sp1 : sp0;
    float best = 0.f;
    part[k] = len[k][0];
#pragma unroll
    for (int c = 0; c < 3; c++) {
      const float most = fminf((float)len[k][c], w[2 + k]), per = n[3 * k + c] / (float)sp.n;
      const float over = n[3 * k + c] > n[3 * k] ? per * (float)sp.part * full + (float)sp.join : 0.f;
      const float t = fminf(ceilf(per) * most, fmaxf(w[k] / (float)sp.n, most) + 0.5f * most) + per * (float)sp.start + over;
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
  const bool order = 2.f * n[0] >= (float)sp0.n;
  for (int c0 = 0; c0 < n_seq; c0 += NT) {
    const int i = c0 + tid, cn = min(NT, n_seq - c0);
    int tiles = c0 ? 0 : tiles0, kind = c0 ? 0 : kind0, keys = c0 ? 0 : keys0;
    q0 = first_q0;
    nq = first_nq;
    nk = first_nk;
    if (c0 && i < n_seq) load(i, tiles, kind, keys);
    const int parts = max((int)((unsigned)(keys + (unsigned)part[kind] - 1u) / (unsigned)part[kind]), 1);
    // Long parts first, so that the last workgroups to start are short: a stable sort by the length of a
    // part in 16 classes (256 decodes of 300 to 4300 keys: 282 us, 292 with three classes; 8-bit cache
    // 162 and 169; in order of the requests 64 decodes 70 us, 66 sorted, 256 268 and 233).  Not for the many-row kernel, whose
    // neighbouring tiles of one request share keys in the L2: its requests come last, in order, and after them those
    // without tiles.  Nor for fewer tiles than half of the workgroups that run at a time (32 decodes 49 us either
    // way): all start at once, and the sort takes 0.9 of the plan's 6.9 us.
    const int lane = tid & 63, wv = tid >> 6;
    int rank = tid;
    __syncthreads();  // the items of the requests before have been written
    if (order) {
      const float most = fminf((float)part[0], w[2]), mine_len = fminf((float)keys, (float)part[0]);
      const int cls = tiles == 0 ? kClasses - 1 : kind ? kClasses - 2 : 15 - (int)(mine_len / fmaxf(most, 1.f) * 15.99f);
      int n_cls = 0;  // rank among the wave's of the class; lane c: how many of class c
#pragma unroll
      for (int c = 0; c < kClasses; c++) {
        const uint64_t same = __ballot(cls == c);
        if (cls == c) rank = __builtin_popcountll(same & ((1ull << lane) - 1));
        if (lane == c) n_cls = __builtin_popcountll(same);
      }
      if (lane < kClasses) l_cls[wv][lane] = n_cls;
      __syncthreads();
      int first = 0, all = 0;
      if (lane < kClasses)
#pragma unroll
        for (int e = 0; e < NT / 64; e++) {
          const int y = l_cls[e][lane];
          if (e < wv) first += y;
          all += y;
        }
      int incl_cls = all;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up(incl_cls, o);
        if (lane >= o) incl_cls += y;
      }
      rank += __shfl(first + incl_cls - all, cls);
    }
    l_rows[rank][0] = q0;
    l_rows[rank][1] = nq;
    l_rows[rank][2] = nk;
    l_seq[rank] = i;
    l_tiles[rank] = tiles;
    l_parts[rank] = parts;
    __syncthreads();
    tiles = l_tiles[tid];
    const int my_parts = l_parts[tid];
    kind = !few_only && l_rows[tid][1] * G > kRowsSmall;
    for (int k = 0; k < 2; k++) {
      const bool mine = kind == k && tiles > 0;
      if (!__syncthreads_or(mine)) continue;
      const int64_t items = mine ? (int64_t)tiles * my_parts : 0;
      const int64_t x = items | (my_parts > 1 ? (items << 40) | ((int64_t)(mine ? tiles : 0) << 52) : 0);
      // running sums over the block
      int64_t incl = x;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int64_t y = __shfl_up(incl, o);
        if (lane >= o) incl += y;
      }
      __syncthreads();
      if (lane == 63) red64[wv] = incl;
      l_n[tid] = mine ? my_parts : 0;
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
        PlanItem it = {l_seq[lo], tile, pi, (int)np, -1, -1, l_rows[lo][0], l_rows[lo][1], l_rows[lo][2], {0, 0, 0}};
        if (np > 1) {
          it.slot = slots[k] + (int)((uint64_t)b >> 40 & 0xfff) + tile * (int)np;
          it.join = joins[k] + (int)((uint64_t)b >> 52) + tile;
          if (k == 1 && pi == 0 && it.join < v.cap_join[1]) v.done[1][it.join] = (int)(at[k] + y);
        }
        v.items[k][at[k] + y] = it;
      }
      at[k] += n_items;
      slots[k] += (int)((uint64_t)total >> 40 & 0xfff);
      joins[k] += (int)((uint64_t)total >> 52);
    }
  }
  if (tid == 0) v.hdr->n_split = min(joins[1], v.cap_join[1]);
  if (tid < 2) {
    v.hdr->n_items[tid] = (int)min(at[tid], (int64_t)v.cap_items[tid]);
    v.hdr->part[tid] = part[tid];
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
// columns, bf16, pages of 16) 280 us, 6.6 TB/s of cache (a kernel that only reads
// reaches 6.3 with ordinary loads); one request of 32767 keys on 32 key/value heads
// 85 us, 6.3 TB/s.  Two workgroups a CU hold 128 KB in flight; a third (168
// registers, 7 spilled) is 10 % slower.  The matrix unit is busy 4 % of the time,
// also where one of its 16 rows is used.
template <typename T, int KS, int DB, int DS, bool JOIN>
__global__ __launch_bounds__(256, DS > 128 ? 1 : 2) void k_attn_few(AttnArgs a, int own_blocks, int join_rows) {
  using V8 = typename Elem<T>::v8;
  using V4 = typename Elem<T>::v4;
  constexpr int CH = DS / 8, NV = 32 * CH / 64;
  __shared__ __attribute__((aligned(16))) char lds[4][32 * DS * 2];
  static_assert(sizeof(JoinLds) <= sizeof(lds), "");
  __shared__ float l_m[4][16], l_l[4][16];
  if (JOIN && (int)blockIdx.x >= own_blocks) {
    join_many<T>(a, join_rows, (int)blockIdx.x - own_blocks, *(JoinLds *)lds[0]);
    return;
  }
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
  if (it.n > 1) join_parts<T>(a, r, it, head, row0, min(n_rows - row0, kRowsSmall), (float *)lds[0]);
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

template <typename T, bool PAGED, bool C8 = false>
void launch_many(const AttnArgs &a, int groups, int64_t blocks, hipStream_t s) {
  const dim3 g((unsigned)blocks), b((unsigned)(256 * groups));
  if (a.D <= 64) k_attn_many<T, 4, 2, 64, 1, PAGED, C8><<<g, b, 0, s>>>(a);
  else if (a.D <= 96 && groups == 1) k_attn_many<T, 6, 3, 128, 1, PAGED, C8><<<g, b, 0, s>>>(a);
  else if (a.D <= 96) k_attn_many<T, 6, 3, 128, 2, PAGED, C8><<<g, b, 0, s>>>(a);
  else if (a.D <= 128 && groups == 1) k_attn_many<T, 8, 4, 128, 1, PAGED, C8><<<g, b, 0, s>>>(a);
  else if (a.D <= 128) k_attn_many<T, 8, 4, 128, 2, PAGED, C8><<<g, b, 0, s>>>(a);
  else k_attn_many<T, 16, 8, 256, 1, PAGED, C8><<<g, b, 0, s>>>(a);
}
// JOIN: after the many-row kernel, with workgroups that join its parts; rows: of its tiles.  A decode step's calls
// have no such workgroups and keep the registers of the kernel without them (8-bit cache, one request of
// 32767 keys 49 us, 50.4 with them).
template <typename T, bool JOIN>
void launch_few(const AttnArgs &a, int64_t blocks, int rows, hipStream_t s) {
  const dim3 g((unsigned)blocks + (JOIN ? kJoinBlocks : 0)), b(256);
  const int own = (int)blocks;
  if (a.D <= 64) k_attn_few<T, 2, 4, 64, JOIN><<<g, b, 0, s>>>(a, own, rows);
  else if (a.D <= 96) k_attn_few<T, 3, 6, 128, JOIN><<<g, b, 0, s>>>(a, own, rows);
  else if (a.D <= 128) k_attn_few<T, 4, 8, 128, JOIN><<<g, b, 0, s>>>(a, own, rows);
  else k_attn_few<T, 8, 16, 256, JOIN><<<g, b, 0, s>>>(a, own, rows);
}
template <typename T, bool JOIN>
void launch_few8(const AttnArgs &a, int64_t blocks, int rows, hipStream_t s) {
  const int64_t round = 8 * few8_heads(a.Hkv, a.page_log2);
  const int own = (int)((blocks + round - 1) / round * round);
  const dim3 g((unsigned)own + (JOIN ? kJoinBlocks : 0)), b(256);
  if (a.D <= 64) k_attn_few8<T, 2, 4, 64, JOIN><<<g, b, 0, s>>>(a, own, rows);
  else if (a.D <= 96) k_attn_few8<T, 4, 6, 128, JOIN><<<g, b, 0, s>>>(a, own, rows);
  else if (a.D <= 128) k_attn_few8<T, 4, 8, 128, JOIN><<<g, b, 0, s>>>(a, own, rows);
  else k_attn_few8<T, 8, 16, 256, JOIN><<<g, b, 0, s>>>(a, own, rows);
}
template <typename T>
void launch_paged(const AttnArgs &a, bool c8, bool few, int groups, hipStream_t s) {
  const int64_t blocks0 = (int64_t)a.plan.cap_items[0] * a.Hkv, blocks1 = (int64_t)a.plan.cap_items[1] * a.Hkv;
  const int rows = kRowsGroup * groups;
  if (few) {
    if (c8) launch_few8<T, false>(a, blocks0, 0, s);
    else launch_few<T, false>(a, blocks0, 0, s);
  } else if (c8) {
    launch_many<T, true, true>(a, groups, blocks1, s);
    launch_few8<T, true>(a, blocks0, rows, s);
  } else {
    launch_many<T, true>(a, groups, blocks1, s);
    launch_few<T, true>(a, blocks0, rows, s);
  }
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
// them, and what a part costs beside its keys.  The few-row kernel takes as long as for 64 keys to start and join
// one.  Many rows are joined by a kernel that follows, and the parts' results go past the caches: fitted to 1,140 forms
// (1 to 40 requests, 1 to 2,100 new tokens on 0 to 59,200, heads of 64 to 256), each whole and with either length of
// part: 250 keys to join at all and, for each part of full tiles, 1500 with one wave group, 700 and 250 with two, 50 and
// 600 above 128 columns, where a key takes three times as long.  With 400 a part, split or not, and nothing for the join,
// short contexts were split at a loss (32 heads on 8 of 128: a prompt of 200 tokens 22.7 us, 13.3 whole; 20 tokens on 150
// 17.4 and 12.3), and long ones too (a prompt of 1000, 96 columns: 49 and 27).  With each part's cost that of a full tile, 5 tokens on each
// of three contexts of 30,000, 20 of a tile's 128 rows, had 22 parts each, not 40: 111 us and 89.
static Split split_of(const cf_attn_desc *d, int kind) {
  const int per_cu = kind ? (desc_groups(d) > 1 || d->head_dim > 128 ? 1 : 2) : (d->head_dim > 128 ? 1 : 2);
  const int n = (256 * per_cu + d->n_kv_heads - 1) / d->n_kv_heads;
  if (!kind) return Split{n, 64, 0, 0, max_parts(0)};
  if (d->head_dim > 128) return Split{n, 0, 600, 50, max_parts(1)};
  return desc_groups(d) > 1 ? Split{n, 0, 250, 700, max_parts(1)} : Split{n, 0, 1500, 250, max_parts(1)};
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

// A step's attention over either cache: what the calls share once the cache is checked.
static cf_status attn_paged(const cf_attn_desc *d, bool c8, int n_kv_heads, int head_dim, int dtype, int page,
                            cf::AttnArgs &a, const int32_t *table_dev, int32_t max_pages, const void *q_dev,
                            int64_t q_tok, int64_t q_head, float scale, void *out_dev, float *lse_dev, void *stream) {
  using namespace cf;
  if (n_kv_heads != d->n_kv_heads || head_dim != d->head_dim)
    return set_error(CF_EINVAL, "the cache has %d heads of %d, the descriptor %d of %d", n_kv_heads, head_dim,
                     d->n_kv_heads, d->head_dim);
  if (max_pages < 1 || !table_dev) return set_error(CF_EINVAL, "table: max_pages %d", max_pages);
  if ((int64_t)max_pages * page > kMaxKeys)
    return set_error(CF_EINVAL, "table: a row of %d pages of %d is too long", max_pages, page);
  if (!scale_ok(scale)) return set_error(CF_EINVAL, "scale %g is not finite and > 0", (double)scale);
  if (d->n_tok == 0) return CF_OK;
  if (!q_dev || !out_dev) return set_error(CF_EINVAL, "NULL array");
  if ((((uintptr_t)q_dev | (uintptr_t)out_dev) & 15) || ((q_tok | q_head) & 7))
    return set_error(CF_EINVAL, "queries or output are not 16-byte aligned");
  a.q = q_dev;
  a.q_tok = q_tok; a.q_head = q_head;
  a.table = table_dev;
  a.max_pages = max_pages; a.page_log2 = log2_of(page);
  a.n_seq = d->n_seq; a.n_tok = d->n_tok;
  a.H = d->n_heads; a.Hkv = d->n_kv_heads; a.G = a.H / a.Hkv; a.D = d->head_dim; a.causal = 1;
  a.s2 = scale * 1.44269504088896340736f;
  a.out = out_dev; a.lse = lse_dev;
  const hipStream_t s = as_stream(stream);
  if (dtype == CF_BF16) launch_paged<__bf16>(a, c8, few_only(d), desc_groups(d), s);
  else launch_paged<_Float16>(a, c8, few_only(d), desc_groups(d), s);
  return hip_check(hipGetLastError(), c8 ? "cf_attn_paged8" : "cf_attn_paged");
}

extern "C" cf_status cf_attn_paged(const cf_attn_desc *d, const cf_kv_cache *cache, const int32_t *table_dev,
                                   int32_t max_pages, const void *q_dev, int64_t q_tok, int64_t q_head, float scale,
                                   void *out_dev, float *lse_dev, void *stream) {
  using namespace cf;
  AttnArgs a{};
  cf_status st = check_plan(d, &a.plan);
  if (st == CF_OK) st = check_cache(cache);
  if (st != CF_OK) return st;
  a.k = cache->k_dev; a.v = cache->v_dev; a.n_pages = cache->n_pages;
  return attn_paged(d, false, cache->n_kv_heads, cache->head_dim, cache->dtype, cache->page, a, table_dev, max_pages,
                    q_dev, q_tok, q_head, scale, out_dev, lse_dev, stream);
}

extern "C" cf_status cf_attn_paged8(const cf_attn_desc *d, const cf_kv_cache8 *cache, const int32_t *table_dev,
                                    int32_t max_pages, const void *q_dev, int64_t q_tok, int64_t q_head, float scale,
                                    void *out_dev, float *lse_dev, void *stream) {
  using namespace cf;
  AttnArgs a{};
  cf_status st = check_plan(d, &a.plan);
  if (st == CF_OK) st = check_cache8(cache);
  if (st != CF_OK) return st;
  a.k = cache->k_dev; a.v = cache->v_dev; a.exps = cache->exp_dev; a.n_pages = cache->n_pages;
  return attn_paged(d, true, cache->n_kv_heads, cache->head_dim, cache->dtype, cache->page, a, table_dev, max_pages,
                    q_dev, q_tok, q_head, scale, out_dev, lse_dev, stream);
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
