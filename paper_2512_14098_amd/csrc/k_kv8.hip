// k_kv8.hip -- rotary positions, the quantisation of new keys and values into
// an 8-bit paged cache, and the way back to 16-bit rows.
//
// Pair i of a head's rotated columns turns by phi = pos[axis[i]][t] freq[i]:
// y_a = x_a cos phi - x_b sin phi, y_b = x_b cos phi + x_a sin phi.  The angle
// (one rounding of the 64-bit product), its sine and cosine and the turn itself are in
// 64 bits: at position 32767 an angle in 32 bits would be off by 2^-10, and a
// turned key next to a border between two e4m3 codes would fall to either side.
// The result is rounded to fp32 and from there to the element type.
//
// A row of head_dim elements of the cache is head_dim e4m3 codes and the byte
// e + 127 of its scale 2^e, the smallest with max |x| <= 448 2^e.  A power of two
// makes the scaling exact, and a floating code's relative error does not depend on
// where in the range the largest element falls; the same power undoes it in the
// conversion instruction, v_cvt_scalef32_pk_*.  |x| is cut at 1.875 times the type's
// largest power of two first, so that a value held is always one of the element
// type: without that, fp16 values from 63488 on would be held as 65536.
#include "cf_attn.h"
#include "cf_overlap.h"

namespace cf {
bool page_ok(int page);

namespace {

struct TurnArgs {
  const void *q, *k, *v;
  void *q_out, *k_out;
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head, qo_tok, qo_head, ko_tok, ko_head;  // elements
  const int32_t *pos, *axis;
  const double *freq;
  int32_t n_axes, rot, interleaved, inverse;
  uint8_t *kc, *vc, *ec;  // the cache's codes and exponent bytes
  const int64_t *slot;
  int64_t n_slots;
  int32_t n_tok, Hq, Hk, D, page_log2, waves;  // waves: per token
};

template <typename T>
__device__ __forceinline__ float widen(uint32_t half) {
  return (float)__builtin_bit_cast(T, (uint16_t)half);
}
template <>
__device__ __forceinline__ float widen<__bf16>(uint32_t half) {
  return __uint_as_float(half << 16);
}
template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  typedef T V2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, V2{(T)lo, (T)hi});
}

// The largest of the L lanes (a power of two from 8 to 32) of this lane's group.
template <int L>
__device__ __forceinline__ float max_group(float x) {
  auto step = [&](auto ctrl) {
    x = fmaxf(x, __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), ctrl.value, 15, 15, true)));
  };
  step(Int<0xB1>());   // lanes 1, 0, 3, 2 of four
  step(Int<0x4E>());   // lanes 2, 3, 0, 1
  step(Int<0x141>());  // mirrored in eight
  if (L >= 16) step(Int<0x140>());  // mirrored in sixteen
  if (L >= 32) x = max_rows16(x);
  return x;
}

// Eight elements of a row whose largest magnitude over the group is wanted: codes and the
// row's exponent byte.  Infinities and NaN become the e4m3 NaN and do not count for the scale.
template <typename T, int L>
__device__ __forceinline__ uint2 quantise(float (&x)[8], uint32_t &byte) {
  constexpr float kTop = __is_same(T, __bf16) ? 0x1.ep127f : 0x1.ep15f;
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; i++) m = fmaxf(m, fabsf(x[i]));
  if (__ballot(m > kTop)) {
    m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float y = fabsf(x[i]);
      const bool fine = y < __builtin_inff();
      m = fmaxf(m, fine ? fminf(y, kTop) : 0.f);
      x[i] = fine ? fminf(fmaxf(x[i], -kTop), kTop) : x[i];
    }
  }
  m = max_group<L>(m);
  // 448 = 1.75 2^8: the exponent of m, one more where m's fraction is above 1.75, less 8
  byte = (uint32_t)max((int)((__float_as_uint(m) + 0x1fffffu) >> 23) - 8, 1);
  const float inv = __uint_as_float((254u - byte) << 23);
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[4] * inv, x[5] * inv, hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[6] * inv, x[7] * inv, hi, true);
  return make_uint2((uint32_t)lo, (uint32_t)hi);
}

// How columns are paired: no turn; i and rot / 2 + i, the halves cut in 16 bytes or not; 2i and 2i + 1.
enum Pairs { kNone, kHalves, kApart, kNeighbours };

// A lane's eight elements: in a row, but four and four `apart` bytes away in kApart.
template <Pairs P>
__device__ __forceinline__ uint4 load_row(const void *p, int apart) {
  if (P != kApart) return *(const uint4 *)p;
  const uint2 x = *(const uint2 *)p, y = *(const uint2 *)((const char *)p + apart);
  return make_uint4(x.x, x.y, y.x, y.y);
}
template <Pairs P>
__device__ __forceinline__ void store_row(void *p, int apart, const uint4 &x) {
  if (P == kApart) {
    *(uint2 *)p = make_uint2(x.x, x.y);
    *(uint2 *)((char *)p + apart) = make_uint2(x.z, x.w);
  } else {
    *(uint4 *)p = x;
  }
}

// x of the lane next to this one in a pair of lanes
__device__ __forceinline__ uint32_t neighbour(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 15, 15, true);
}
// kHalves: of two lanes the even one holds eight elements of the first half and the odd one those that
// they are paired with.  They exchange four, so that each has four pairs, and back: 16-byte loads and
// stores where four and four elements would be loaded and stored (335 MB turned 129 us, 147 with 8 bytes).
__device__ __forceinline__ uint4 meet(const uint4 &x, bool odd) {
  const uint32_t a = neighbour(odd ? x.x : x.z), b = neighbour(odd ? x.y : x.w);
  return odd ? make_uint4(a, b, x.z, x.w) : make_uint4(x.x, x.y, a, b);
}

template <typename T>
__device__ __forceinline__ void widen_row(const uint4 &x, float (&e)[8]) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; i++) {
    e[2 * i] = widen<T>(w[i] & 0xffff);
    e[2 * i + 1] = widen<T>(w[i] >> 16);
  }
}

// One token's rows (queries, then keys, then values) by one wave, or by four where tokens are few, a row by L
// lanes of eight elements each: four pairs where they turn.  A wave has read all of a row when it writes
// it, so that a turn may be done in place.  The token's sines and cosines are computed once by each wave,
// passed through LDS and kept in registers over its rows.
//
// Bound by memory: 32,767 tokens of 32 + 8 heads of 128 turned in 129 us, 5.2 TB/s read and written (a
// large copy: 4.8 to 5.1), 52,808 tokens of 2 x 8 heads quantised in 71 us, 5.2 TB/s, both in one launch over 22,190
// tokens 128 us, 4.9 TB/s.  The 64-bit products are hidden behind that as long as the rest is short: with one loop over
// all rows that asks each for its kind 150, 72 and 152 us.
template <typename T, int L, Pairs P, bool Q8>
__global__ __launch_bounds__(256) void k_turn(TurnArgs a) {
  constexpr bool ROPE = P != kNone;
  __shared__ double2 l_cs[4][ROPE ? 128 : 1];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int u = lane & (L - 1), per_pass = 64 / L * a.waves;
  const int r_first = (w & (a.waves - 1)) * (64 / L) + lane / L;
  const int tokens = 4 / a.waves;  // of a workgroup
  const int half = a.rot / 2;
  const bool has = u * 8 < a.D, turns = ROPE && u * 8 < a.rot;
  const bool pairs = P == kHalves && turns, split = P == kApart && turns, odd = u & 1;
  // the lane's first element; bytes to its fifth
  const int oa = pairs ? (odd ? half + 4 * (u - 1) : 4 * u) : split ? 4 * u : 8 * u, apart = split ? 2 * half : 8;
  for (int64_t t = (int64_t)blockIdx.x * tokens + w / a.waves; t < a.n_tok; t += (int64_t)gridDim.x * tokens) {
    int64_t slot = -1;
    if (Q8) slot = a.slot[t];
    double c[4], s[4];
    if (ROPE) {
      for (int i = lane; i < half; i += 64) {
        const int ax = a.axis ? a.axis[i] : 0;
        const int p = (unsigned)ax < (unsigned)a.n_axes ? a.pos[(int64_t)ax * a.n_tok + t] : 0;
        double sn, cn;
        sincos((double)p * a.freq[i], &sn, &cn);
        l_cs[w][i] = make_double2(cn, a.inverse ? -sn : sn);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const double2 y = turns ? l_cs[w][4 * u + i] : make_double2(1., 0.);
        c[i] = y.x;
        s[i] = y.y;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    // turned rows: pairs (e[i], e[i + 4]), or (e[2i], e[2i + 1]), as elements and as the type's values
    auto turn = [&](uint4 &x) CF_INLINE {
      if (P == kHalves) {
        const uint4 y = meet(x, odd);
        if (turns) x = y;
      }
      float e[8];
      widen_row<T>(x, e);
#pragma unroll
      for (int i = 0; i < 4; i++) {
        float &p = e[P == kNeighbours ? 2 * i : i], &q = e[P == kNeighbours ? 2 * i + 1 : i + 4];
        const double dp = p, dq = q;
        p = (float)fma(dp, c[i], -(dq * s[i]));
        q = (float)fma(dq, c[i], dp * s[i]);
      }
      if (turns)  // else as they are, infinities and NaN too
        x = make_uint4(pack2<T>(e[0], e[1]), pack2<T>(e[2], e[3]), pack2<T>(e[4], e[5]), pack2<T>(e[6], e[7]));
    };
    // rows that are turned and stored
    auto turn_rows = [&](int n, const void *in, int64_t tok, int64_t head, void *out, int64_t otok, int64_t ohead) CF_INLINE {
      const T *src = (const T *)in + t * tok + r_first * head + oa;
      T *dst = (T *)out + t * otok + r_first * ohead + oa;
      for (int r0 = 0; r0 < n; r0 += per_pass) {
        const bool on = has && r0 + r_first < n;
        if (P == kHalves) {  // every lane takes part in the exchange
          uint4 x = make_uint4(0, 0, 0, 0);
          if (on) x = load_row<P>(src, apart);
          turn(x);
          const uint4 y = meet(x, odd);  // its own inverse
          if (turns) x = y;
          if (on) store_row<P>(dst, apart, x);
        } else if (on) {
          uint4 x = load_row<P>(src, apart);
          turn(x);
          store_row<P>(dst, apart, x);
        }
        src += per_pass * head;
        dst += per_pass * ohead;
      }
    };
    // rows that go to the cache; which: 0 keys, 1 values
    const int64_t page = slot >> a.page_log2, off = slot & ((1ll << a.page_log2) - 1);
    auto hold_rows = [&](auto which, const void *in, int64_t tok, int64_t head, uint8_t *codes) CF_INLINE {
      constexpr bool K = which.value == 0;
      constexpr Pairs PR = K ? P : kNone;
      const int o0 = K ? oa : 8 * u;
      const T *src = (const T *)in + t * tok + r_first * head + o0;
      for (int r0 = 0; r0 < a.Hk; r0 += per_pass) {
        const int h = r0 + r_first;
        const bool on = has && h < a.Hk;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (on) x = load_row<PR>(src, apart);
        if (PR != kNone) turn(x);
        float e[8];
        widen_row<T>(x, e);
        uint32_t byte;
        uint2 code = quantise<T, L>(e, byte);
        if (PR == kHalves) {
          const uint32_t got = neighbour(odd ? code.x : code.y);
          if (turns) code = odd ? make_uint2(got, code.y) : make_uint2(code.x, got);
        }
        if (on) {
          const int64_t row = page * a.Hk + h;
          uint8_t *dst = codes + ((row << a.page_log2) + off) * a.D + o0;
          if (PR == kApart && split) {
            *(uint32_t *)dst = code.x;
            *(uint32_t *)(dst + half) = code.y;
          } else {
            *(uint2 *)dst = code;
          }
          if (u == 0) a.ec[((row * 2 + which.value) << a.page_log2) + off] = (uint8_t)byte;
        }
        src += per_pass * head;
      }
    };
    if (ROPE) turn_rows(a.Hq, a.q, a.q_tok, a.q_head, a.q_out, a.qo_tok, a.qo_head);
    if constexpr (Q8) {
      if (slot >= 0 && slot < a.n_slots) {
        hold_rows(Int<0>(), a.k, a.k_tok, a.k_head, a.kc);
        hold_rows(Int<1>(), a.v, a.v_tok, a.v_head, a.vc);
      }
    } else {
      turn_rows(a.Hk, a.k, a.k_tok, a.k_head, a.k_out, a.ko_tok, a.ko_head);
    }
  }
}

struct ReadArgs {
  const uint8_t *kc, *vc, *ec;
  const int32_t *table, *start;
  void *k_out, *v_out;
  int32_t n_seq, n_tok, max_pages, n_pages, Hkv, D, page_log2, tokens;  // tokens: of a workgroup
};

constexpr int kReadTokens = 16;

// Each wave finds the requests and pages of a quarter of the workgroup's tokens, 64 starts at
// a time; then a thread takes 16 codes of one token's head a step, keys before values.
// Bound by memory: 113,000 tokens of 64 requests, 2 x 8 heads of 128, in 137 us, 5.3 TB/s read and written.
template <typename T, int U>
__global__ __launch_bounds__(256) void k_kv_read8(ReadArgs a) {
  __shared__ int32_t l_page[kReadTokens], l_off[kReadTokens];  // page -1: zeros, -2: nobody's token
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const unsigned chunks = (unsigned)a.D / 16, per_half = a.Hkv * chunks, per_tok = 2 * per_half;
  for (int64_t t0 = (int64_t)blockIdx.x * a.tokens; t0 < a.n_tok; t0 += (int64_t)gridDim.x * a.tokens) {
    const int n_here = (int)min((int64_t)a.tokens, a.n_tok - t0);
    __syncthreads();
    for (int i = w; i < n_here; i += 4) {
      const int t = (int)t0 + i;
      int lo = 0, n = a.n_seq, from, to;
      for (;;) {  // the last request that starts at or before t
        const int step = (n + 63) >> 6, at = lo + min(lane * step, n - 1);
        from = clampi(a.start[at], 0, a.n_tok);
        to = clampi(a.start[at + 1], 0, a.n_tok);
        const int last = max(__builtin_popcountll(__ballot(lane * step < n && from <= t)) - 1, 0);
        from = __builtin_amdgcn_readlane(from, last);
        to = __builtin_amdgcn_readlane(to, last);
        lo += last * step;
        if (step == 1) break;
        n = min(step, n - last * step);
      }
      if (lane == 0) {
        int page = -2;
        if (t >= from && t < to) {
          const int col = (t - from) >> a.page_log2;
          page = col < a.max_pages ? a.table[(int64_t)lo * a.max_pages + col] : -1;
          if ((unsigned)page >= (unsigned)a.n_pages) page = -1;
        }
        l_page[i] = page;
        l_off[i] = (t - from) & ((1 << a.page_log2) - 1);
      }
    }
    __syncthreads();
    const unsigned total = (unsigned)n_here * per_tok;
    for (unsigned x0 = tid; x0 < total; x0 += 256 * U) {
      uint4 code[U];
      uint32_t byte[U];
      T *dst[U];
#pragma unroll
      for (int i = 0; i < U; i++) {
        const unsigned x = x0 + 256 * i;
        code[i] = make_uint4(0, 0, 0, 0);
        byte[i] = 0;
        dst[i] = nullptr;
        if (x >= total) continue;
        const unsigned at = x / per_tok, rest = x - at * per_tok;
        const bool is_v = rest >= per_half;
        const unsigned hc = is_v ? rest - per_half : rest, h = hc / chunks, c = hc - h * chunks;
        const int page = l_page[at], off = l_off[at];
        if (page == -2) continue;
        dst[i] = (T *)(is_v ? a.v_out : a.k_out) + ((t0 + at) * a.Hkv + h) * a.D + c * 16;
        if (page < 0) continue;
        const int64_t row = (int64_t)page * a.Hkv + h;
        // read once: without a place in the caches (719 MB: 152 us against 162 with 16 tokens a workgroup)
        typedef uint32_t V4 __attribute__((ext_vector_type(4)));
        const V4 y = __builtin_nontemporal_load(
            (const V4 *)((is_v ? a.vc : a.kc) + ((row << a.page_log2) + off) * a.D + c * 16));
        code[i] = make_uint4(y[0], y[1], y[2], y[3]);
        byte[i] = a.ec[((row * 2 + is_v) << a.page_log2) + off];
      }
#pragma unroll
      for (int i = 0; i < U; i++) {
        if (!dst[i]) continue;
        const float scale = __uint_as_float(byte[i] << 23);
        uint4 y[2];
        y[0] = make_uint4(widen8<T>(code[i].x, scale, 0), widen8<T>(code[i].x, scale, 1), widen8<T>(code[i].y, scale, 0),
                          widen8<T>(code[i].y, scale, 1));
        y[1] = make_uint4(widen8<T>(code[i].z, scale, 0), widen8<T>(code[i].z, scale, 1), widen8<T>(code[i].w, scale, 0),
                          widen8<T>(code[i].w, scale, 1));
        ((uint4 *)dst[i])[0] = y[0];
        ((uint4 *)dst[i])[1] = y[1];
      }
    }
  }
}

template <typename T, int L>
void launch_turn(const TurnArgs &a, bool rope, bool q8, unsigned blocks, hipStream_t s) {
  const dim3 g(blocks), b(256);
  if (!rope) k_turn<T, L, kNone, true><<<g, b, 0, s>>>(a);
  else if (a.interleaved && q8) k_turn<T, L, kNeighbours, true><<<g, b, 0, s>>>(a);
  else if (a.interleaved) k_turn<T, L, kNeighbours, false><<<g, b, 0, s>>>(a);
  else if (a.rot % 16 && q8) k_turn<T, L, kApart, true><<<g, b, 0, s>>>(a);
  else if (a.rot % 16) k_turn<T, L, kApart, false><<<g, b, 0, s>>>(a);
  else if (q8) k_turn<T, L, kHalves, true><<<g, b, 0, s>>>(a);
  else k_turn<T, L, kHalves, false><<<g, b, 0, s>>>(a);
}

void launch(TurnArgs &a, int dtype, bool rope, bool q8, hipStream_t s) {
  // Four waves a token where the tokens are few: 256 tokens of 40 heads turned in 5.1 us, with one wave 7.6;
  // 700 in 7.4 and 9.1, 1500 in 10.5 and 11.0 (turned and written 13.0 and 12.7), 5000 in 23 and 19.
  a.waves = a.n_tok < 1500 ? 4 : 1;
  const int64_t tokens = 4 / a.waves, need = ((int64_t)a.n_tok + tokens - 1) / tokens;
  const unsigned blocks = (unsigned)(need < (1 << 20) ? need : 1 << 20);
  if (dtype == CF_BF16) {
    if (a.D <= 64) launch_turn<__bf16, 8>(a, rope, q8, blocks, s);
    else if (a.D <= 128) launch_turn<__bf16, 16>(a, rope, q8, blocks, s);
    else launch_turn<__bf16, 32>(a, rope, q8, blocks, s);
  } else {
    if (a.D <= 64) launch_turn<_Float16, 8>(a, rope, q8, blocks, s);
    else if (a.D <= 128) launch_turn<_Float16, 16>(a, rope, q8, blocks, s);
    else launch_turn<_Float16, 32>(a, rope, q8, blocks, s);
  }
}

// Checks of a call's rotary description and of one strided tensor; the arguments they fill.
cf_status take_rope(const cf_rope_desc *r, int D, TurnArgs *a) {
  if (!r) return set_error(CF_EINVAL, "rotary description is NULL");
  if (r->n_axes < 1 || r->n_axes > 16) return set_error(CF_EINVAL, "n_axes %d is not in 1..16", r->n_axes);
  if (r->rot_dim < 8 || r->rot_dim % 8 || r->rot_dim > D)
    return set_error(CF_EINVAL, "rot_dim %d is not a multiple of 8 in 8..head_dim %d", r->rot_dim, D);
  a->pos = r->pos_dev; a->axis = r->axis_dev; a->freq = r->freq_dev;
  a->n_axes = r->n_axes; a->rot = r->rot_dim;
  a->interleaved = r->interleaved != 0; a->inverse = r->inverse != 0;
  return CF_OK;
}
bool rows_ok(const void *p, int64_t tok, int64_t head) { return !((uintptr_t)p & 15) && !((tok | head) & 7); }
// In place means element by element: the same strides.
bool place_ok(const void *in, int64_t tok, int64_t head, const void *out, int64_t otok, int64_t ohead) {
  return in != out || (tok == otok && head == ohead);
}
// An output beside its input shares no element with it.
bool beside_ok(const RowSet &in, const RowSet &out) { return in.p == out.p || !rows_meet(out, in); }

cf_status take_write(const cf_kv_cache8 *c, const void *k, int64_t k_tok, int64_t k_head, const void *v, int64_t v_tok,
                     int64_t v_head, const int64_t *slot, TurnArgs *a) {
  if (!k || !v || !slot) return set_error(CF_EINVAL, "NULL array");
  if (!rows_ok(k, k_tok, k_head) || !rows_ok(v, v_tok, v_head))
    return set_error(CF_EINVAL, "keys and values are not 16-byte aligned");
  const uint64_t rows = (uint64_t)c->n_pages * c->n_kv_heads * c->page, codes = rows * c->head_dim;
  if (bytes_meet(c->k_dev, codes, c->v_dev, codes) || bytes_meet(c->exp_dev, 2 * rows, c->k_dev, codes) ||
      bytes_meet(c->exp_dev, 2 * rows, c->v_dev, codes))
    return set_error(CF_EINVAL, "arrays of a cache that is written overlap");
  a->k = k; a->k_tok = k_tok; a->k_head = k_head;
  a->v = v; a->v_tok = v_tok; a->v_head = v_head;
  a->kc = (uint8_t *)c->k_dev; a->vc = (uint8_t *)c->v_dev; a->ec = c->exp_dev;
  a->slot = slot; a->n_slots = (int64_t)c->n_pages * c->page;
  a->Hk = c->n_kv_heads; a->D = c->head_dim; a->page_log2 = log2_of(c->page);
  return CF_OK;
}

}  // namespace

cf_status check_cache8(const cf_kv_cache8 *c) {
  if (!c) return set_error(CF_EINVAL, "cache is NULL");
  if (c->n_pages < 0 || c->n_kv_heads < 1 || c->n_kv_heads > 65535)
    return set_error(CF_EINVAL, "cache: n_pages %d, n_kv_heads %d", c->n_pages, c->n_kv_heads);
  if (!page_ok(c->page)) return set_error(CF_EINVAL, "page %d is not a power of two in 16..256", c->page);
  if (c->head_dim < 16 || c->head_dim > 256 || c->head_dim % 16)
    return set_error(CF_EINVAL, "head_dim %d is not a multiple of 16 in 16..256", c->head_dim);
  if (c->dtype != CF_BF16 && c->dtype != CF_F16) return set_error(CF_EINVAL, "dtype %d", c->dtype);
  if (c->n_pages > 0 && (!c->k_dev || !c->v_dev || !c->exp_dev)) return set_error(CF_EINVAL, "NULL cache");
  if (((uintptr_t)c->k_dev | (uintptr_t)c->v_dev | (uintptr_t)c->exp_dev) & 15)
    return set_error(CF_EINVAL, "cache is not 16-byte aligned");
  return CF_OK;
}

}  // namespace cf

extern "C" cf_status cf_rope(const cf_rope_desc *r, int32_t n_tok, int32_t n_heads, int32_t n_kv_heads,
                             int32_t head_dim, int32_t dtype, const void *q_dev, int64_t q_tok, int64_t q_head,
                             void *q_out_dev, int64_t qo_tok, int64_t qo_head, const void *k_dev, int64_t k_tok,
                             int64_t k_head, void *k_out_dev, int64_t ko_tok, int64_t ko_head, void *stream) {
  using namespace cf;
  if (n_tok < 0 || n_heads < 1 || n_heads > 65535 || n_kv_heads < 0 || n_kv_heads > 65535)
    return set_error(CF_EINVAL, "n_tok %d, n_heads %d, n_kv_heads %d", n_tok, n_heads, n_kv_heads);
  if (head_dim < 8 || head_dim > 256 || head_dim % 8)
    return set_error(CF_EINVAL, "head_dim %d is not a multiple of 8 in 8..256", head_dim);
  if (dtype != CF_BF16 && dtype != CF_F16) return set_error(CF_EINVAL, "dtype %d", dtype);
  TurnArgs a{};
  const cf_status st = take_rope(r, head_dim, &a);
  if (st != CF_OK) return st;
  if (n_tok == 0) return CF_OK;
  if (!a.pos || !a.freq || !q_dev || !q_out_dev || (n_kv_heads > 0 && (!k_dev || !k_out_dev)))
    return set_error(CF_EINVAL, "NULL array");
  if (!rows_ok(q_dev, q_tok, q_head) || !rows_ok(q_out_dev, qo_tok, qo_head) ||
      (n_kv_heads > 0 && (!rows_ok(k_dev, k_tok, k_head) || !rows_ok(k_out_dev, ko_tok, ko_head))))
    return set_error(CF_EINVAL, "queries or keys are not 16-byte aligned");
  if (!place_ok(q_dev, q_tok, q_head, q_out_dev, qo_tok, qo_head) ||
      (n_kv_heads > 0 && !place_ok(k_dev, k_tok, k_head, k_out_dev, ko_tok, ko_head)))
    return set_error(CF_EINVAL, "in place with other strides");
  if (n_kv_heads > 0 && q_out_dev == k_out_dev) return set_error(CF_EINVAL, "q_out_dev is k_out_dev");
  // rows are turned in any order
  const RowSet q{q_dev, n_tok, n_heads, q_tok, q_head, head_dim}, qo{q_out_dev, n_tok, n_heads, qo_tok, qo_head, head_dim};
  const RowSet k{k_dev, n_tok, n_kv_heads, k_tok, k_head, head_dim}, ko{k_out_dev, n_tok, n_kv_heads, ko_tok, ko_head, head_dim};
  if (rows_overlap(qo) || rows_overlap(ko)) return set_error(CF_EINVAL, "rows of an output overlap, in place or not");
  if (!beside_ok(q, qo) || !beside_ok(k, ko)) return set_error(CF_EINVAL, "an output shares elements with its input");
  if (rows_meet(qo, k) || rows_meet(qo, ko) || rows_meet(ko, q))
    return set_error(CF_EINVAL, "q_out_dev shares elements with the keys, or k_out_dev with the queries");
  a.q = q_dev; a.q_tok = q_tok; a.q_head = q_head;
  a.q_out = q_out_dev; a.qo_tok = qo_tok; a.qo_head = qo_head;
  a.k = k_dev; a.k_tok = k_tok; a.k_head = k_head;
  a.k_out = k_out_dev; a.ko_tok = ko_tok; a.ko_head = ko_head;
  a.n_tok = n_tok; a.Hq = n_heads; a.Hk = n_kv_heads; a.D = head_dim;
  launch(a, dtype, true, false, as_stream(stream));
  return hip_check(hipGetLastError(), "cf_rope");
}

extern "C" cf_status cf_kv_write8(const cf_kv_cache8 *cache, int32_t n_tok, const void *k_dev, int64_t k_tok,
                                  int64_t k_head, const void *v_dev, int64_t v_tok, int64_t v_head,
                                  const int64_t *slot_dev, void *stream) {
  using namespace cf;
  cf_status st = check_cache8(cache);
  if (st != CF_OK) return st;
  if (n_tok < 0) return set_error(CF_EINVAL, "n_tok %d", n_tok);
  if (n_tok == 0 || cache->n_pages == 0) return CF_OK;
  TurnArgs a{};
  st = take_write(cache, k_dev, k_tok, k_head, v_dev, v_tok, v_head, slot_dev, &a);
  if (st != CF_OK) return st;
  a.n_tok = n_tok;
  launch(a, cache->dtype, false, true, as_stream(stream));
  return hip_check(hipGetLastError(), "cf_kv_write8");
}

extern "C" cf_status cf_rope_write8(const cf_rope_desc *r, const cf_kv_cache8 *cache, int32_t n_tok, int32_t n_heads,
                                    const void *q_dev, int64_t q_tok, int64_t q_head, void *q_out_dev, int64_t qo_tok,
                                    int64_t qo_head, const void *k_dev, int64_t k_tok, int64_t k_head,
                                    const void *v_dev, int64_t v_tok, int64_t v_head, const int64_t *slot_dev,
                                    void *stream) {
  using namespace cf;
  cf_status st = check_cache8(cache);
  if (st != CF_OK) return st;
  if (n_tok < 0 || n_heads < 1 || n_heads > 65535) return set_error(CF_EINVAL, "n_tok %d, n_heads %d", n_tok, n_heads);
  TurnArgs a{};
  st = take_rope(r, cache->head_dim, &a);
  if (st != CF_OK) return st;
  if (n_tok == 0) return CF_OK;
  st = take_write(cache, k_dev, k_tok, k_head, v_dev, v_tok, v_head, slot_dev, &a);
  if (st != CF_OK) return st;
  if (!a.pos || !a.freq || !q_dev || !q_out_dev) return set_error(CF_EINVAL, "NULL array");
  if (!rows_ok(q_dev, q_tok, q_head) || !rows_ok(q_out_dev, qo_tok, qo_head))
    return set_error(CF_EINVAL, "queries are not 16-byte aligned");
  if (!place_ok(q_dev, q_tok, q_head, q_out_dev, qo_tok, qo_head))
    return set_error(CF_EINVAL, "in place with other strides");
  // a token's queries are written before its keys and values are read
  const RowSet qo{q_out_dev, n_tok, n_heads, qo_tok, qo_head, a.D};
  if (rows_overlap(qo)) return set_error(CF_EINVAL, "rows of an output overlap, in place or not");
  if (!beside_ok(RowSet{q_dev, n_tok, n_heads, q_tok, q_head, a.D}, qo))
    return set_error(CF_EINVAL, "an output shares elements with its input");
  if (rows_meet(qo, RowSet{k_dev, n_tok, a.Hk, k_tok, k_head, a.D}) ||
      rows_meet(qo, RowSet{v_dev, n_tok, a.Hk, v_tok, v_head, a.D}))
    return set_error(CF_EINVAL, "q_out_dev shares elements with k_dev or v_dev");
  a.q = q_dev; a.q_tok = q_tok; a.q_head = q_head;
  a.q_out = q_out_dev; a.qo_tok = qo_tok; a.qo_head = qo_head;
  a.n_tok = n_tok; a.Hq = n_heads;
  launch(a, cache->dtype, true, true, as_stream(stream));
  return hip_check(hipGetLastError(), "cf_rope_write8");
}

extern "C" cf_status cf_kv_read8(const cf_kv_cache8 *cache, const int32_t *table_dev, int32_t max_pages, int32_t n_seq,
                                 const int32_t *k_start_dev, int32_t n_tok, void *k_out_dev, void *v_out_dev,
                                 void *stream) {
  using namespace cf;
  const cf_status st = check_cache8(cache);
  if (st != CF_OK) return st;
  if (n_seq < 1 || n_seq > 1 << 30 || n_tok < 0 || max_pages < 1)
    return set_error(CF_EINVAL, "n_seq %d, n_tok %d, max_pages %d", n_seq, n_tok, max_pages);
  if (n_tok == 0) return CF_OK;
  if (!table_dev || !k_start_dev || !k_out_dev || !v_out_dev) return set_error(CF_EINVAL, "NULL array");
  if (((uintptr_t)k_out_dev | (uintptr_t)v_out_dev) & 15) return set_error(CF_EINVAL, "output is not 16-byte aligned");
  const uint64_t out_bytes = 2ull * n_tok * cache->n_kv_heads * cache->head_dim;
  if (bytes_meet(k_out_dev, out_bytes, v_out_dev, out_bytes)) return set_error(CF_EINVAL, "outputs overlap");
  ReadArgs a;
  a.kc = (const uint8_t *)cache->k_dev; a.vc = (const uint8_t *)cache->v_dev; a.ec = cache->exp_dev;
  a.table = table_dev; a.start = k_start_dev;
  a.k_out = k_out_dev; a.v_out = v_out_dev;
  a.n_seq = n_seq; a.n_tok = n_tok; a.max_pages = max_pages; a.n_pages = cache->n_pages;
  a.Hkv = cache->n_kv_heads; a.D = cache->head_dim; a.page_log2 = log2_of(cache->page);
  // About 1024 loads a workgroup (113,000 tokens of 2 x 8 heads of 128, 8 tokens: 137 us, with 4 146, with 16
  // 143; heads of 64, 16 tokens: 76 us, with 8 83), less where that leaves CUs without one.
  const int loads = cache->n_kv_heads * (cache->head_dim / 8);  // of a token
  a.tokens = n_tok < 16384 || loads >= 512 ? 4 : loads >= 128 ? 8 : kReadTokens;
  const int64_t need = ((int64_t)n_tok + a.tokens - 1) / a.tokens;
  const dim3 g((unsigned)(need < (1 << 20) ? need : 1 << 20)), b(256);
  const hipStream_t s = as_stream(stream);
  if (cache->dtype == CF_BF16) {
    if (a.tokens == 4) k_kv_read8<__bf16, 4><<<g, b, 0, s>>>(a);
    else k_kv_read8<__bf16, 8><<<g, b, 0, s>>>(a);
  } else {
    if (a.tokens == 4) k_kv_read8<_Float16, 4><<<g, b, 0, s>>>(a);
    else k_kv_read8<_Float16, 8><<<g, b, 0, s>>>(a);
  }
  return hip_check(hipGetLastError(), "cf_kv_read8");
}
