// Arrays of rows as the checks of a call's arguments see them (host only); not part of the public ABI.
#pragma once

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

// Whether lo < d - i S - t s < hi for some i, t within the given ends, where the inner steps stay within an outer one.
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
    const Steps K = near(r, s);
    for (int64_t t = K.first; t <= K.last; ++t)
      if (lo < r - t * s.step && r - t * s.step < hi) return true;
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

// Whether two arrays of the same size (null: none) share memory; whether they do without being the same.
inline bool shared(const void* a, const void* b, size_t bytes) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return a && b && x < y + bytes && y < x + bytes;
}
inline bool shifted(const void* a, const void* b, size_t bytes) { return a != b && shared(a, b, bytes); }

}  // namespace hg
