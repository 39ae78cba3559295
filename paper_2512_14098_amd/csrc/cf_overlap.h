// cf_overlap.h -- host: whether rows of strided tensors share elements.
#pragma once
#include <cstdint>

namespace cf {

// Rows (t, h), t < n and h < heads, of d 16-bit elements each, at p + t * tok + h * head elements.
struct RowSet {
  const void *p;
  int64_t n, heads, tok, head, d;
};

// Whether two ranges of bytes meet.
inline bool bytes_meet(const void *p, uint64_t np, const void *q, uint64_t nq) {
  const uint64_t a = (uint64_t)(uintptr_t)p, b = (uint64_t)(uintptr_t)q;
  return np > 0 && nq > 0 && (a <= b ? b - a < np : a - b < nq);
}

namespace overlap {

constexpr int64_t kFar = 1ll << 56;  // elements: no memory reaches that far

// First and past-the-last element from p; false where that is further than memory reaches.
inline bool span(const RowSet &a, int64_t &lo, int64_t &hi) {
  const __int128 t = a.n > 1 ? (__int128)(a.n - 1) * a.tok : 0, h = a.heads > 1 ? (__int128)(a.heads - 1) * a.head : 0;
  const __int128 l = (t < 0 ? t : 0) + (h < 0 ? h : 0), u = (t > 0 ? t : 0) + (h > 0 ? h : 0) + a.d;
  if (l < -kFar || u > kFar) return false;
  lo = (int64_t)l;
  hi = (int64_t)u;
  return true;
}

// Whether some i, |i| < n, has |x + i * step| < d.
inline bool near(int64_t x, int64_t step, int64_t n, int64_t d) {
  if (step < 0) step = -step;
  if (x < 0) x = -x;
  if (step == 0 || n == 1) return x < d;
  const int64_t i = x / step < n - 1 ? x / step : n - 1;  // the last step that does not pass 0
  return x - i * step < d || (i < n - 1 && (i + 1) * step - x < d);
}

// Whether some i, 0 <= i < n, has |x - i * step| < d.
inline bool near_from(int64_t x, int64_t step, int64_t n, int64_t d) {
  if (step < 0) {
    step = -step;
    x = -x;
  }
  if (step == 0 || x <= 0) return x < d && -x < d;
  const int64_t i = x / step < n - 1 ? x / step : n - 1;
  return x - i * step < d || (i < n - 1 && (i + 1) * step - x < d);
}

}  // namespace overlap

// Whether a row of a and one of b, of as many tokens, share an element.  Past 2^20 comparisons, which tensors whose
// memory meets take only with strides that differ or hundreds of heads: "yes".
inline bool rows_meet(RowSet a, RowSet b) {
  if (a.n < 1 || a.heads < 1 || b.heads < 1) return false;
  int64_t alo, ahi, blo, bhi;
  if (!overlap::span(a, alo, ahi) || !overlap::span(b, blo, bhi)) return true;
  const __int128 apart = ((__int128)(uintptr_t)b.p - (__int128)(uintptr_t)a.p) / 2;
  if (apart + blo >= ahi || apart + bhi <= alo) return false;
  int64_t x = (int64_t)apart;  // below 2 kFar, as they meet
  if (a.n == 1) a.tok = b.tok = 0;
  if (a.heads == 1) a.head = b.head;
  if (b.heads == 1) b.head = a.head;
  if (a.tok == 0 && b.tok != 0) {
    const RowSet y = a;
    a = b;
    b = y;
    x = -x;
  }
  const bool one = a.tok == b.tok;
  if (one && a.tok != 0) {  // parts of one projection's output: each has a range of its own in every token
    const int64_t step = a.tok < 0 ? -a.tok : a.tok, ha = a.head * (a.heads - 1), hb = b.head * (b.heads - 1);
    const int64_t from = x + (hb < 0 ? hb : 0) - (ha < 0 ? ha : 0), r = (from % step + step) % step;
    if (r >= (ha < 0 ? -ha : ha) + a.d && r + (hb < 0 ? -hb : hb) + b.d <= step) return false;
  }
  const bool apace = a.head == b.head;  // rows of heads as far apart as their numbers
  const int64_t heads = apace ? a.heads + b.heads - 1 : a.heads * b.heads, tokens = one || b.tok == 0 ? 1 : b.n;
  if (heads * tokens > 1 << 20) return true;
  for (int64_t g = 0; g < heads; g++) {
    const int64_t y = x + (apace ? (g - a.heads + 1) * a.head : g / a.heads * b.head - g % a.heads * a.head);
    for (int64_t t = 0; t < tokens; t++)
      if (one ? overlap::near(y, a.tok, a.n, a.d) : overlap::near_from(y + t * b.tok, a.tok, a.n, a.d)) return true;
  }
  return false;
}

// Whether two rows of a share an element.
inline bool rows_overlap(const RowSet &a) {
  if (a.n < 1 || a.heads < 1) return false;
  int64_t lo, hi;
  if (!overlap::span(a, lo, hi)) return true;
  const int64_t tok = a.tok < 0 ? -a.tok : a.tok, head = a.head < 0 ? -a.head : a.head;
  if (a.heads == 1) return a.n > 1 && tok < a.d;
  if (a.n == 1) return head < a.d;
  if (tok < a.d || head < a.d) return true;
  if (tok >= head * (a.heads - 1) + a.d || head >= tok * (a.n - 1) + a.d) return false;  // one inside the other
  // rows g numbers apart along the shorter side, at any distance along the other
  const bool by_head = a.heads <= a.n;
  const int64_t m = by_head ? a.heads : a.n, sm = by_head ? a.head : a.tok;
  for (int64_t g = 1; g < m; g++)
    if (overlap::near(g * sm, by_head ? a.tok : a.head, by_head ? a.n : a.heads, a.d)) return true;
  return false;
}

}  // namespace cf
