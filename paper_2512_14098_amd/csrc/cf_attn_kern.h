// cf_attn_kern.h -- device code of the attention kernels that caches of either
// width share: loads, specials, work items, the join of split contexts and the
// many-row kernel.
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
#pragma once
#include "cf_attn.h"

namespace cf {

// Zeros that lanes load in place of keys and values that are not there: 16 rows
// of the widest head, so that a whole page group can be pointed at them.
__device__ i32x4 g_zeros[16 * 256 * 2 / 16];

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
__host__ __device__ constexpr int max_parts(int kind) { return kind ? 64 : 128; }
// Fewest keys of a part (many rows, 40 tokens on 1000: 22 us, 29 with 256).
__host__ __device__ constexpr int min_part(int kind) { return kind ? 128 : 256; }

__host__ __device__ inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// 16 bytes of global memory (said to the compiler, which else takes the pointer
// for one that may be into LDS, and its loads wait on both counters).
__device__ __forceinline__ i32x4 load16(const void *p) {
  typedef const __attribute__((address_space(1))) i32x4 *gp;
  return *(gp)(uintptr_t)p;
}

__device__ __forceinline__ uint32_t load1(const void *p) {
  typedef const __attribute__((address_space(1))) uint8_t *gp;
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
struct Dyn {
  int value;
};

// Half j of 16 e4m3 codes, times their row's scale, as eight elements.
template <typename T>
__device__ __forceinline__ i32x4 widen16(const i32x4 &x, float scale, int j) {
  return i32x4{(int)widen8<T>(x[2 * j], scale, 0), (int)widen8<T>(x[2 * j], scale, 1),
               (int)widen8<T>(x[2 * j + 1], scale, 0), (int)widen8<T>(x[2 * j + 1], scale, 1)};
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

// The infinities and NaN among the values of keys [from, to), which not all
// of the rows row0 .. row0 + n - 1 see, added to the results just written.
template <typename T, bool PAGED, bool C8 = false>
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
      [[maybe_unused]] typename Elem<T>::v4 wide;
      if constexpr (C8) {
        const int id = a.table[(int64_t)seq * a.max_pages + (key >> a.page_log2)];
        if ((unsigned)id >= (unsigned)a.n_pages) continue;
        const int64_t row = (int64_t)id * a.Hkv + head;
        const int off = key & ((1 << a.page_log2) - 1);
        const uint32_t codes = *(const uint16_t *)((const uint8_t *)a.v + ((row << a.page_log2) + off) * a.D + e);
        const uint32_t byte = a.exps[((row * 2 + 1) << a.page_log2) + off];
        wide = __builtin_bit_cast(typename Elem<T>::v4, make_uint2(widen8<T>(codes, __uint_as_float(byte << 23), 0), 0u));
        v = (const T *)&wide;
      } else if (PAGED) {
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
  if (item >= a.plan.cap_items[kind]) return false;
  const PlanItem p = a.plan.items[kind][item];  // beside the header, not after it
  const int len = a.plan.hdr->part[kind];
  if (item >= a.plan.hdr->n_items[kind]) return false;
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

// The parts of a split context are joined:  m = max m_p, l = sum l_p e^(m_p - m), o = sum o_p e^(m_p - m) / l, in an
// order that the sizes alone decide, so that results repeat: with few rows part by part, with many every fourth
// part by one of four lanes (l) and every share-th by one of `share` threads (o), then those.

// Few rows: by the workgroup that finishes last, whichever it is.
// w: LDS of this workgroup, at least 2 x max_parts x kRowsSmall floats.
template <typename T>
__device__ __forceinline__ void join_parts(const AttnArgs &a, const Rows &r, const Item &it, int head, int row0,
                                           int n, float *w) {
  using V4 = typename Elem<T>::v4;
  constexpr int R = kRowsSmall;
  __shared__ int last;
  __shared__ float l_sum[R];
  const int tid = threadIdx.x, nt = (int)blockDim.x;
  parts_arrived();
  __syncthreads();
  if (tid == 0) {
    int *done = a.plan.done[0] + (int64_t)it.join * a.Hkv + head;
    last = atomicAdd(done, 1) == it.n - 1;
    if (last) *done = 0;  // for the next layer's call
  }
  __syncthreads();
  if (!last) return;
  const float *ml = a.plan.ml[0], *o = a.plan.o[0];
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
    if (a.lse) a.lse[(int64_t)(r.q0 + j) * a.H + head * a.G + g] = log_sum(m, l, a.s2, weight_shift<T>(0));
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

// Many rows: by workgroups of the few-row kernel, which is launched after the many-row kernel, past those of its
// own items: kJoinBlocks of them share the split tiles and, where those are few, their rows.
// One workgroup reads past its L2 at 8 GB/s only, and a part of 128 rows of 128 columns has 64 KB; after the kernel
// that wrote them every workgroup may read them through its own (40 tokens of 32 heads on 8 on 1000: 48 us where the
// last workgroup joined, 22 so; 100 on 10,000 twice 111 and 76).  R: rows of a tile.
constexpr int kJoinBlocks = 512, kJoinRows = 16;
struct JoinLds {
  float w[kJoinRows][max_parts(1)], wl[kJoinRows][max_parts(1)], l_sum[kJoinRows];  // weights, sums, 1 / l
  f32x4 part[256];
};
template <typename T>
__device__ __forceinline__ void join_many(const AttnArgs &a, int R, int block, JoinLds &s) {
  using V4 = typename Elem<T>::v4;
  const int tid = threadIdx.x, quads = a.D / 4;
  const int64_t tiles = (int64_t)clampi(a.plan.hdr->n_split, 0, a.plan.cap_join[1]) * a.Hkv;
  if (tiles == 0) return;
  const int shares = clampi((int)(kJoinBlocks / tiles), 1, R / 8);
  for (int64_t work = block; work < tiles * shares; work += kJoinBlocks) {
    const int64_t tile = work / shares;
    const int share_no = (int)(work - tile * shares), split = (int)(tile / a.Hkv), head = (int)(tile - (int64_t)split * a.Hkv);
    Item it;
    Rows r;
    const int item = a.plan.done[1][split];
    if (item < 0 || !read_item(a, 1, item, it, r) || it.n < 2) continue;
    const int n_rows = r.nq * a.G, n_rt = (n_rows + R - 1) / R;
    if (it.tile >= n_rt) continue;
    const int row0 = (n_rt - 1 - it.tile) * R, n = min(n_rows - row0, R);
    const int per = (n + shares - 1) / shares, first = share_no * per, end = min(first + per, n);
    const int64_t base = ((int64_t)it.slot * a.Hkv + head) * R, step = (int64_t)a.Hkv * R;
    const float *ml = a.plan.ml[1], *o = a.plan.o[1];
    for (int r0 = first; r0 < end; r0 += kJoinRows) {
      const int m_rows = min(kJoinRows, end - r0);
      __syncthreads();
      for (int x = tid; x < m_rows * it.n; x += 256) {
        const int p = x / m_rows, rr = x - p * m_rows;
        const float2 y = *(const float2 *)(ml + (base + p * step + r0 + rr) * 2);
        s.w[rr][p] = y.x;
        s.wl[rr][p] = y.y;
      }
      __syncthreads();
      for (int x = tid; x < m_rows * 4; x += 256) {  // four lanes a row
        const int rr = x >> 2;
        float m = kNegInf, l = 0.f;
        for (int p = x & 3; p < it.n; p += 4) m = fmaxf(m, s.w[rr][p]);
        m = fmaxf(m, __shfl_xor(m, 1));
        m = fmaxf(m, __shfl_xor(m, 2));
        const float mu = m == kNegInf ? 0.f : m;
        for (int p = x & 3; p < it.n; p += 4) {
          const float f = exp2_hw((s.w[rr][p] - mu) * a.s2);
          s.w[rr][p] = f;
          l = fmaf(f, s.wl[rr][p], l);
        }
        l += __shfl_xor(l, 1);
        l += __shfl_xor(l, 2);
        if ((x & 3) == 0) {
          s.l_sum[rr] = l > 0.f || l != l ? 1.f / l : 0.f;
          const int row = row0 + r0 + rr, j = row / a.G, g = row - j * a.G;
          if (a.lse) a.lse[(int64_t)(r.q0 + j) * a.H + head * a.G + g] = log_sum(m, l, a.s2, weight_shift<T>(1));
        }
      }
      __syncthreads();
      // where there are more threads than groups of four columns, they share a row's parts
      const int total = m_rows * quads, share = max(256 / total, 1), mine = share > 1 ? tid / total : 0;
      for (int x = tid - mine * total; x < total; x += 256) {
        const int rr = x / quads, d4 = x - rr * quads;
        const float *src = o + (base + r0 + rr) * a.D + d4 * 4;
        f32x4 acc = {0, 0, 0, 0};
        if (mine < share) {
#pragma unroll 8
          for (int p = mine; p < it.n; p += share) acc += *(const f32x4 *)(src + p * step * a.D) * s.w[rr][p];
        }
        if (share > 1) {
          s.part[tid] = acc;
          __syncthreads();  // every thread comes here, and once
          if (mine > 0) break;
          for (int i = 1; i < share; i++) acc += s.part[i * total + tid];
        }
        const int row = row0 + r0 + rr, j = row / a.G, g = row - j * a.G;
        T *out = (T *)a.out + ((int64_t)(r.q0 + j) * a.H + head * a.G + g) * a.D + d4 * 4;
        *(V4 *)out = __builtin_convertvector(acc * s.l_sum[rr], V4);
      }
    }
  }
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
// 1000 tokens on 24001, 32 heads on 8, 3.8 ms, 0.42 PFLOP/s.  136 to 248 columns take as long.
// C8, an 8-bit cache: codes are widened between registers and LDS, half the bytes are loaded and staged.
// Lanes hold the addresses of 16 keys' codes and exponents; worked out by the scalar unit at each load from a row number
// they cost a third (two chunks of 1000 on 24001, 32 heads on 8: 925 us against 719; the 16-bit cache 746).
template <typename T, int KS, int DB, int DS, int NG, bool PAGED, bool C8 = false>
__global__ __launch_bounds__(256 * NG, DS == 64 ? 3 : DS == 128 ? 2 : 1) void k_attn_many(AttnArgs a) {
  using V8 = typename Elem<T>::v8;
  using V4 = typename Elem<T>::v4;
  // CE elements in the 16 bytes that a thread loads, CH such chunks a row
  constexpr int NT = 256 * NG, R = kRowsGroup * NG, CE = C8 ? 16 : 8, CH = DS / CE, NL = 64 * CH / NT, RS = NT / CH;
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
  [[maybe_unused]] uint32_t ke[NL] = {}, ve[NL] = {};  // 8-bit cache: the rows' exponent bytes
  uint64_t k_at = 0, v_at = 0;
  [[maybe_unused]] uint64_t e_at = 0;  // 8-bit cache: exponent bytes of the keys, the values' a page further
  bool bad = false;

  // Loads of a tile's keys or values; edge: some may not be there or the tile be past the
  // last, which gives zeros.  Chunks past head_dim are never loaded and stay zero.
  const int lrow = tid / CH, lcol = tid % CH;
  const bool col_ok = lcol * CE < a.D;
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
      const bool in = (unsigned)ids < (unsigned)a.n_pages;
      if constexpr (C8) {
        const int64_t page = (int64_t)ids * a.Hkv + head, row = (page << a.page_log2) + (key & page_mask);
        k_at = (uint64_t)(in ? (const uint8_t *)a.k + row * a.D : (const uint8_t *)g_zeros);
        v_at = (uint64_t)(in ? (const uint8_t *)a.v + row * a.D : (const uint8_t *)g_zeros);
        e_at = (uint64_t)(in ? a.exps + row + (page << a.page_log2) : (const uint8_t *)g_zeros);
      } else {
        const int64_t at = (int64_t)ids * page_elems + (int64_t)(key & page_mask) * a.D;
        k_at = (uint64_t)(in ? kc + at : (const T *)g_zeros);
        v_at = (uint64_t)(in ? vc + at : (const T *)g_zeros);
      }
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
  // the same of an 8-bit cache, with the rows' exponent bytes, e_off from where the keys' are
  auto lane_address = [&](uint64_t x, int l) CF_INLINE {
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)x, l), hi = __builtin_amdgcn_readlane((uint32_t)(x >> 32), l);
    return (const uint8_t *)((uint64_t)hi << 32 | lo);
  };
  auto load8 = [&](i32x4 (&x)[NL], uint32_t (&xe)[NL], uint64_t where, unsigned e_off, int n, auto edge) CF_INLINE {
    const int t0 = it.lo + 64 * n;
    if (!col_ok) return;
#pragma unroll
    for (int i = 0; i < NL; i++) {
      const int rr = i * RS + lrow;
      const int l16 = ((n & 15) << 2) + __builtin_amdgcn_readfirstlane(rr >> 4);
      const uint8_t *p = lane_address(where, l16) + (unsigned)((rr & 15) * a.D + lcol * 16);
      const uint8_t *e = lane_address(e_at, l16) + (unsigned)((rr & 15) + e_off);
      if (edge.value) {
        p = t0 + rr < to_load ? p : (const uint8_t *)g_zeros;
        e = t0 + rr < to_load ? e : (const uint8_t *)g_zeros;
      }
      x[i] = load16(p);
      xe[i] = load1(e);
    }
  };
  auto store8 = [&](const i32x4 (&x)[NL], const uint32_t (&xe)[NL], T *dst, auto specials) CF_INLINE {
#pragma unroll
    for (int i = 0; i < NL; i++) {
      const int rr = i * RS + lrow;
      const float scale = __uint_as_float(xe[i] << 23);
#pragma unroll
      for (int j = 0; j < 2; j++) {
        i32x4 y = widen16<T>(x[i], scale, j);
        if (specials.value) bad |= take_specials<T>(y);
        *(i32x4 *)(dst + rr * DS + ((2 * lcol + j) ^ swz<DS>(rr)) * 8) = y;
      }
    }
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
    if constexpr (C8) {
      load8(kr, ke, k_at, 0, nk, edge);
      load8(vr, ve, v_at, page_mask + 1, nk - 1, edge);
    } else {
      load(kr, k_at, kp, a.k_tok, nk, edge);
      load(vr, v_at, vp, a.v_tok, nk - 1, edge);
    }
    if (PAGED && (nk & 7) == 4) place(nk + 4);  // in place of tiles nk - 12 .. nk - 5
    if (PAGED && (nk & 7) == 0) load_ids(nk + 8);
  };
  auto put = [&](int nk, T *kd, T *vd, auto edge) CF_INLINE {
    if constexpr (C8) {
      store8(kr, ke, kd, Int<0>());
      if (edge.value && it.lo + 64 * nk > all_wg && r.nk > all_wg) store8(vr, ve, vd, Int<1>());
      else store8(vr, ve, vd, Int<0>());
    } else {
      store(kr, kd);
      if (edge.value && it.lo + 64 * nk > all_wg && r.nk > all_wg) {  // also where no row sees them
        asm volatile("");  // a branch: not worth computing for every tile
#pragma unroll
        for (int i = 0; i < NL; i++) bad |= take_specials<T>(vr[i]);
      }
      store(vr, vd);
    }
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
  if constexpr (C8) store8(vr, ve, lds_v[1], Int<0>());
  else store(vr, lds_v[1]);
  if (PAGED) {
    load_ids(0);
    place(0);
    load_ids(8);
  }
  {
    i32x4 first[NL];
#pragma unroll
    for (int i = 0; i < NL; i++) first[i] = i32x4{0, 0, 0, 0};
    [[maybe_unused]] uint32_t fe[NL] = {};
    if constexpr (C8) load8(first, fe, k_at, 0, 0, Int<1>());
    else load(first, k_at, kp, a.k_tok, 0, Int<1>());
    fetch(1, Int<1>());
    // the queries after the first keys and values: those are waited for first
    const T *qp = (const T *)a.q + (int64_t)(r.q0 + j) * a.q_tok + (int64_t)(head * a.G + g) * a.q_head;
#pragma unroll
    for (int ks = 0; ks < KS; ks++) {
      const int c = ks * 2 + h;
      qf[ks] = __builtin_bit_cast(V8, load16(c * 8 < a.D ? (const void *)(qp + c * 8) : (const void *)g_zeros));
    }
    if constexpr (C8) store8(first, fe, lds_k[0], Int<0>());
    else store(first, lds_k[0]);
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
    add_specials<T, PAGED, C8>(a, r, k0, it.seq, it.n > 1 ? it.slot + it.part : -1, R, head, row0, min(n_rows - row0, R),
                           it.lo + (max(all_wg - it.lo, 0) & ~63), hi);
}

}  // namespace
}  // namespace cf
