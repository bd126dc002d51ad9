// Arrays of rows as the checks of a call's arguments see them (host only); not part of the public ABI.
#pragma once

#include <initializer_list>

#include "hg_internal.cuh"

namespace hg {

// Row (i, t), i < n, t < T, is the w bytes at p + i sn + t st.
struct RowSet {
  uintptr_t p;
  int64_t n, T, sn, st, w;
};

inline RowSet row_set(const void* p, int64_t n, int64_t T, int64_t sn, int64_t st, int64_t width, size_t esz) {
  const int64_t b = (int64_t)esz;
  return {(uintptr_t)p, n, T, n < 2 ? 0 : sn * b, T < 2 ? 0 : st * b, width * b};
}

// Whether lo < d - i S - t s < hi for some i, t within the given ends, where the inner steps stay within an outer one:
// the outer steps that come near are tried, the inner ones follow by division.
inline __int128 floor_div(__int128 a, __int128 b) { return a / b - (a % b != 0 && (a < 0) != (b < 0)); }
struct Steps {
  __int128 step;
  int64_t first, last;
};
inline bool step_within(__int128 d, Steps S, Steps s, int64_t lo, int64_t hi) {
  if (S.step < s.step) {
    const Steps x = S;
    S = s;
    s = x;
  }
  auto near = [&](__int128 num, const Steps& x) -> Steps {  // the steps that can come near num
    if (x.step == 0) return {0, 0, 0};
    const __int128 q = num / x.step, m = (hi - (__int128)lo) / x.step + 2;
    const __int128 a = q - m < x.first ? x.first : q - m, b = q + m > x.last ? x.last : q + m;
    return a > b ? Steps{0, 1, 0} : Steps{0, (int64_t)a, (int64_t)b};
  };
  const Steps I = near(d, S);
  for (int64_t i = I.first; i <= I.last; ++i) {
    const __int128 r = d - i * S.step;
    if (s.step == 0) {
      if (lo < r && r < hi) return true;
      continue;
    }
    const __int128 a = floor_div(r - hi, s.step) + 1, b = -floor_div(lo - r, s.step) - 1;  // a <= t <= b
    if ((a < s.first ? s.first : a) <= (b > s.last ? s.last : b)) return true;
  }
  return false;
}

// Whether the rows of an array that is written (its rows nest: positions within sequences or the other way round) meet
// those of another: found wherever the two have the same strides, else where a corner row of one meets the other.
inline bool rows_meet(const RowSet& out, const RowSet& in) {
  auto end = [](const RowSet& r, int c) {  // place of a corner row, from the first
    return (c & 1 ? (__int128)(r.n - 1) * r.sn : 0) + (c & 2 ? (__int128)(r.T - 1) * r.st : 0);
  };
  const __int128 d = (__int128)in.p - (__int128)out.p;
  if (d >= end(out, 3) + out.w || -d >= end(in, 3) + in.w) return false;
  if (out.sn == in.sn && out.st == in.st)
    return step_within(d, {out.sn, 1 - out.n, out.n - 1}, {out.st, 1 - out.T, out.T - 1}, -in.w, out.w);
  // rows of an input that lie over one another are not searched: too many come near a place
  const bool search = (in.n < 2 || in.sn >= in.w) && (in.T < 2 || in.st >= in.w);
  for (int c = 0; c < 4; ++c) {
    if (step_within(d + end(in, c), {out.sn, 0, out.n - 1}, {out.st, 0, out.T - 1}, -in.w, out.w)) return true;
    if (search && step_within(end(out, c) - d, {in.sn, 0, in.n - 1}, {in.st, 0, in.T - 1}, -out.w, in.w)) return true;
  }
  return false;
}

// A contiguous array (null: none); the rows of a sequence argument.
inline RowSet block_set(const void* p, int64_t bytes) { return {(uintptr_t)p, 1, 1, 0, 0, p ? bytes : 0}; }
inline RowSet seq_set(const hg_seq* r, int64_t n, int64_t T, int64_t width, size_t esz) {
  return row_set(r->p, n, T, r->stride_n, r->stride_t, width, esz);
}

inline hg_status check_seq(const hg_seq* r, const char* name, int64_t n, int64_t T, int64_t width, size_t esz,
                           bool written) {
  HG_REQUIRE(r != nullptr && r->p != nullptr, "%s must be non-null", name);
  HG_REQUIRE(((uintptr_t)r->p & 15) == 0, "%s must be 16-byte aligned", name);
  const int64_t lim = int64_t(1) << 40, st = r->stride_t, sn = r->stride_n, u = 16 / (int64_t)esz;
  HG_REQUIRE(T < 2 || (st >= 0 && st < lim && st % u == 0),
             "%s: stride_t must be a non-negative multiple of 16 bytes", name);
  HG_REQUIRE(n < 2 || (sn >= 0 && sn < lim && sn % u == 0),
             "%s: stride_n must be a non-negative multiple of 16 bytes", name);
  if (written) {  // rows nest: positions within sequences, or sequences within positions
    const bool ok_t = T < 2 || st >= width, ok_n = n < 2 || sn >= width;
    // sn >= (T - 1) st + width, or st >= (n - 1) sn + width, without the products, which may pass 64 bits
    const bool nest = n < 2 || T < 2 || (sn >= width && st <= (sn - width) / (T - 1)) ||
                      (st >= width && sn <= (st - width) / (n - 1));
    HG_REQUIRE(ok_t && ok_n && nest, "%s: rows that are written must not overlap", name);
  }
  return HG_OK;
}

// Rows that are written meet none of the others.
inline hg_status check_apart(const RowSet& out, const char* name, std::initializer_list<RowSet> others) {
  for (const RowSet& r : others) HG_REQUIRE(!rows_meet(out, r), "%s must not overlap another array", name);
  return HG_OK;
}

// Whether two arrays of the same size (null: none) share memory; whether they do without being the same.
inline bool shared(const void* a, const void* b, size_t bytes) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return a && b && x < y + bytes && y < x + bytes;
}
inline bool shifted(const void* a, const void* b, size_t bytes) { return a != b && shared(a, b, bytes); }

}  // namespace hg
