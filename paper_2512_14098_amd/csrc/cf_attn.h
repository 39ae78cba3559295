// cf_attn.h -- shared pieces of the attention kernels: element types and
// their matrix instructions, row and key bookkeeping, the plan in memory.
#pragma once
#include "cf_internal.h"

namespace cf {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

template <typename T>
struct Elem;
template <>
struct Elem<__bf16> {
  typedef __bf16 v4 __attribute__((ext_vector_type(4)));
  typedef __bf16 v8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x16 mma32(v8 a, v8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mma16(v8 a, v8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Elem<_Float16> {
  typedef _Float16 v4 __attribute__((ext_vector_type(4)));
  typedef _Float16 v8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x16 mma32(v8 a, v8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mma16(v8 a, v8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};

constexpr float kNegInf = -__builtin_inff();
constexpr int kRowsSmall = 16;   // (token, head) rows of a workgroup of the few-row kernel
constexpr int kRowsGroup = 128;  // of a group of four waves of the many-row kernel
constexpr int kMinPart = 256;    // fewest keys of a part of a split context

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// x of this lane and of the lane 32 away
__device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float max_rows16(float x) {  // and of the lanes 16 away
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_rows16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Four elements of one column of a 16-column tile in LDS: the 16 lanes of a
// group give the addresses of 4 rows x 16 columns (8 bytes each, lane 4r + c
// row r, columns 4c..4c+3), and lane i receives column i of the four rows.
template <typename T>
__device__ __forceinline__ typename Elem<T>::v4 read_tr(const T *p) {
  typedef __attribute__((address_space(3))) s16x4 *lds_p;
  const s16x4 r = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)(const_cast<T *>(p)));
  return __builtin_bit_cast(typename Elem<T>::v4, r);
}

template <typename V8, typename V4>
__device__ __forceinline__ V8 join8(V4 a, V4 b) {
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// ------------------------------------------------------------------ the plan in memory
struct PlanHdr {
  int32_t n_items[2];  // few-row and many-row kernel
  int32_t part[2];     // keys of a part of a split context
  int32_t pad[12];
};
struct PlanItem {
  int32_t seq, tile, part, n;  // part of n of the context of a tile of rows
  int32_t slot, join;          // n > 1: the tile's first partial result, its counter
  int32_t q0, nq, nk;          // the request's first token, new tokens and keys
  int32_t pad[3];
};
struct PlanView {
  PlanHdr *hdr;
  PlanItem *items[2];
  int32_t *done[2];    // [split tile][key/value head]: parts finished, zero between calls
  float *o[2], *ml[2];  // partial results: [slot][key/value head][row]
  int32_t cap_items[2], cap_slots[2], cap_join[2];
};

// Host: the parts of work_dev for a descriptor; bytes needed.
uint64_t plan_view(const cf_attn_desc *d, PlanView *v);

// A sequence's packed query rows: row r is token r / G, query head r % G of a
// key/value head's group of G.
struct Rows {
  int q0, nq, nk;  // first token, tokens, keys
};

struct AttnArgs {
  const void *q, *k, *v;
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head;  // elements
  const int32_t *q_start, *kv;  // packed sequences: query and key starts
  const int32_t *table;
  int32_t max_pages, n_pages, page_log2;
  int32_t n_seq, n_tok, n_k, H, Hkv, G, D, causal;
  float s2;  // scale * log2(e)
  void *out;
  float *lse;
  PlanView plan;
};

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return min(max(x, lo), hi); }

}  // namespace cf
