// cf_attn_few8.h -- the few-row attention kernel over an 8-bit cache.
#pragma once
#include "cf_attn_kern.h"

namespace cf {
namespace {

// Heads of a page whose exponent bytes, 2 x page each, share a 128-byte line.
__host__ __device__ inline unsigned few8_heads(int Hkv, int page_log2) {
  unsigned n = page_log2 < 6 ? 64u >> page_log2 : 1u;
  while (Hkv % n) n >>= 1;
  return n;
}

// As k_attn_few, with codes widened to the element type, their row's scale
// applied, on the way into the matrix instruction (keys) and into LDS (values): the
// attention of the values held, in that kernel's arithmetic.  A lane loads 16 codes of
// a key, the two halves of which go to two products: the order of the columns within a
// product is free as long as the queries have the same.  The exponent bytes of the
// tile's 32 keys and 32 values lie across the lanes, one load.  The next tile's keys are
// loaded as soon as this one's are in their products, the values when they are in LDS.
//
// Bound by memory: 256 requests of 1767 keys on average (32 heads on 8, 128 columns,
// pages of 16) 156 us, 6.1 TB/s of cache, 153 us with pages of 64; one request of 32767 keys on 32
// key/value heads 49 us, 5.5 TB/s, of which 8 us are the launch, the first loads and the join.
// Leaving out the conversions, the products or the stores to LDS changes no time.  Three
// workgroups a CU (161 registers) hold as much in flight as two of tiles of 64 keys (236
// registers), which take 162 us and 52.
template <typename T, int KS, int DB, int DS, bool JOIN>
__global__ __launch_bounds__(256, DS > 128 ? 1 : 2) void k_attn_few8(AttnArgs a, int own_blocks, int join_rows) {
  using V8 = typename Elem<T>::v8;
  using V4 = typename Elem<T>::v4;
  constexpr int CH = DS / 16, KP = KS / 2, NV = 32 * CH / 64;  // chunks of a row, loads of 16 keys and of 32 values
  __shared__ __attribute__((aligned(16))) char lds[4][32 * DS * 2];
  static_assert(sizeof(JoinLds) <= sizeof(lds), "");
  __shared__ float l_m[4][16], l_l[4][16];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (JOIN && (int)blockIdx.x >= own_blocks) {
    join_many<T>(a, join_rows, (int)blockIdx.x - own_blocks, *(JoinLds *)lds[0]);
    return;
  }
  // Workgroups go round the XCDs, each with an L2 of its own.  The heads whose exponent bytes share a line
  // follow each other on one XCD, so that it need not be fetched by each (64 columns 79 us against 81).
  const unsigned hg = few8_heads(a.Hkv, a.page_log2), units = (unsigned)a.Hkv / hg;
  const unsigned k = blockIdx.x >> 3, unit = k / hg * 8 + (blockIdx.x & 7);
  const int item = (int)(unit / units), head = (int)(unit % units * hg + k % hg);
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
  const int all = __builtin_amdgcn_readfirstlane(r.nk - r.nq + row0 / a.G + 1);  // keys that every row sees

  const int gq = lane >> 4;
  V8 qf[KS];
  const T *qp = (const T *)a.q + (int64_t)(r.q0 + j) * a.q_tok + (int64_t)(head * a.G + g) * a.q_head;
#pragma unroll
  for (int ks = 0; ks < KS; ks++) {
    const int c = 16 * ((ks >> 1) * 4 + gq) + 8 * (ks & 1);
    qf[ks] = __builtin_bit_cast(V8, load16(c < a.D ? (const void *)(qp + c) : (const void *)g_zeros));
  }

  const uint8_t *kc = (const uint8_t *)a.k, *vc = (const uint8_t *)a.v;
  const int page_mask = (1 << a.page_log2) - 1;
  const int32_t *trow = a.table + (int64_t)it.seq * a.max_pages;
  const int n_tiles = hi > it.lo ? (hi - it.lo + 31) >> 5 : 0;

  f32x4 o[DB];
#pragma unroll
  for (int d = 0; d < DB; d++) o[d] = f32x4{0, 0, 0, 0};
  float m = kNegInf, l = 0.f;
  i32x4 kr[2][KP], vr[NV];
  uint32_t ex = 0;  // exponent byte of key (lanes 0 to 31) or value (32 to 63) lane % 32 of the tile
  int ids = 0;
  T *vt = (T *)lds[w];
  bool bad = false;

  // the wave's tile n: page ids of 32 tiles at a time lie across the lanes
  auto load_ids = [&](int n) CF_INLINE {
    const int key = it.lo + 32 * (w + 4 * (n + (lane >> 1))) + 16 * (lane & 1);
    ids = key < hi ? trow[key >> a.page_log2] : -1;
  };
  int64_t base[2];
  int valid[2];  // keys of the 16 that may be read
  auto load_keys = [&](int n) CF_INLINE {
    if ((n & 31) == 0) load_ids(n);
    const int t0 = it.lo + 32 * (w + 4 * n), i0 = (n & 31) << 1;
    {
      const int key = t0 + (lane & 31);
      const int id = __builtin_amdgcn_ds_bpermute((i0 + (gq & 1)) << 2, ids);
      const bool ok = (unsigned)id < (unsigned)a.n_pages && key < r.nk;
      const int64_t row = ((int64_t)id * a.Hkv + head) * 2 + (lane >> 5);
      ex = load1(ok ? (const void *)(a.exps + (row << a.page_log2) + (key & page_mask)) : (const void *)g_zeros);
    }
#pragma unroll
    for (int b = 0; b < 2; b++) {
      const int id = __builtin_amdgcn_readlane(ids, i0 + b);
      const bool in = (unsigned)id < (unsigned)a.n_pages;
      base[b] = ((((int64_t)(in ? id : 0) * a.Hkv + head) << a.page_log2) + ((t0 + 16 * b) & page_mask)) * a.D;
      valid[b] = in ? r.nk - (t0 + 16 * b) : 0;
    }
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
      for (int kp = 0; kp < KP; kp++) {
        const int c = kp * 4 + gq, key = lane & 15;
        const bool ok = key < valid[b] && c * 16 < a.D;
        kr[b][kp] = load16_nt(ok ? (const void *)(kc + base[b] + key * a.D + c * 16) : (const void *)g_zeros);
      }
  };
  auto load_values = [&]() CF_INLINE {
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int x = i * 64 + lane, key = x / CH, c = x % CH, b = (i * 64 / CH) >> 4;
      const bool ok = (key & 15) < valid[b] && c * 16 < a.D;
      vr[i] = load16_nt(ok ? (const void *)(vc + base[b] + (key & 15) * a.D + c * 16) : (const void *)g_zeros);
    }
  };
  auto scale_of = [&](uint32_t bits, int from) CF_INLINE {
    return __uint_as_float((uint32_t)__builtin_amdgcn_ds_bpermute(from << 2, (int)bits));
  };

  if (w < n_tiles) {
    load_keys(0);
    load_values();
  }
  for (int n = 0; w + 4 * n < n_tiles; n++) {
    const int t0 = it.lo + 32 * (w + 4 * n);
    const bool more = w + 4 * (n + 1) < n_tiles;
    f32x4 s[2];
    const uint32_t bits = ex << 23;
#pragma unroll
    for (int b = 0; b < 2; b++) {
      const float scale = scale_of(bits, 16 * b + (lane & 15));
      s[b] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int ks = 0; ks < KS; ks++)
        s[b] = Elem<T>::mma16(__builtin_bit_cast(V8, widen16<T>(kr[b][ks >> 1], scale, ks & 1)), qf[ks], s[b]);
    }
    if (more) load_keys(n + 1);
    // A key that not every row sees, or none.  Asked for each chunk: with two loops, one for either answer,
    // all chunks are waited for first (160 us against 156, 256 columns 106 against 100).
    const bool some = t0 + 32 > all && r.nk > all;
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int x = i * 64 + lane, key = x / CH, c = x % CH;
      const float scale = scale_of(bits, 32 + key);
#pragma unroll
      for (int h = 0; h < 2; h++) {
        i32x4 y = widen16<T>(vr[i], scale, h);
        if (some) bad |= take_specials<T>(y);
        *(i32x4 *)(vt + key * DS + ((2 * c + h) ^ swz8<DS>(key)) * 8) = y;
      }
    }
    if (more) load_values();
    if (t0 + 32 > min(all, hi)) {
#pragma unroll
      for (int b = 0; b < 2; b++)
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const int key = t0 + 16 * b + 4 * gq + i;
          s[b][i] = key <= lim && key < hi ? s[b][i] : kNegInf;
        }
    }
    float mx = kNegInf;
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
      for (int i = 0; i < 4; i++) mx = fmaxf(mx, s[b][i]);
    mx = max_halves(max_rows16(mx));
    const float mn = fmaxf(m, mx), mu = mn == kNegInf ? 0.f : mn * a.s2;
    const float alpha = exp2_hw(fmaf(m, a.s2, -mu));
    m = mn;
    l *= alpha;
#pragma unroll
    for (int d = 0; d < DB; d++) o[d] = o[d] * alpha;
    const float mp = (m == kNegInf ? 0.f : m * a.s2) - weight_shift<T>(0);
    V8 pf;
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const float p = exp2_hw(fmaf(s[b][i], a.s2, -mp));
        l += p;
        pf[b * 4 + i] = (T)p;
      }
    __builtin_amdgcn_wave_barrier();
    const int vrow = 4 * gq + ((lane & 15) >> 2), vcol = 4 * (lane & 3);
#pragma unroll
    for (int d = 0; d < DB; d++) {
      const int c = d * 2 + (vcol >> 3), off = vcol & 7;
      const V4 lo4 = read_tr<T>(vt + vrow * DS + (c ^ swz8<DS>(vrow)) * 8 + off);
      const V4 hi4 = read_tr<T>(vt + (vrow + 16) * DS + (c ^ swz8<DS>(vrow + 16)) * 8 + off);
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
    add_specials<T, true, true>(a, r, 0, it.seq, it.n > 1 ? it.slot + it.part : -1, kRowsSmall, head, row0, min(n_rows - row0, kRowsSmall),
                          it.lo + (max(all - it.lo, 0) & ~31), hi);
  if (it.n > 1) join_parts<T>(a, r, it, head, row0, min(n_rows - row0, kRowsSmall), (float *)lds[0]);
}

}  // namespace
}  // namespace cf
