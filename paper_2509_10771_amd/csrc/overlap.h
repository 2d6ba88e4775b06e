// Host-side checks shared by the entry points whose matrices have strides: types of the activations, and whether two sets of rows share memory.
// Not part of the public ABI (that is include/rslx.h).
#pragma once

#include <algorithm>

#include "host.h"

namespace rslx {
namespace host {

inline int type_size(int32_t dtype) { return dtype == RSLX_F32 ? 4 : 2; }

inline int32_t check_dtype(int32_t dtype, const char* who) {
  if (dtype != RSLX_F32 && dtype != RSLX_BF16 && dtype != RSLX_F16) return fail(RSLX_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
  return RSLX_OK;
}

// Rows of `bytes` bytes each: row (i, j, ..) lies at p + i stride[0] + j stride[1] + .., strides in bytes.
typedef __int128 wide;                         // (a stride times a count, whatever a caller gives)
struct RowSet {
  const void* p;
  int64_t bytes;
  wide stride[3];
  int64_t count[3];
};

inline RowSet rows_of(const void* p, int64_t ld, int64_t rows, int64_t cols, int size) { return {p, cols * size, {(wide)ld * size}, {rows, 1, 1}}; }

// Whether some x_i of 0..n_i puts the sum of s_i x_i between lo and hi: terms of the largest s first, each tried where the others can
// still reach.  Layouts in use leave one or two values to try at each; where it takes too long to tell, the answer is yes.
struct Term { wide s; wide n; };
inline bool reaches(const Term* t, int count, wide lo, wide hi, int& tries) {
  if (hi < 0) return false;
  if (lo <= 0) return true;
  wide reach = 0;
  for (int i = 1; i < count; ++i) reach += t[i].s * t[i].n;
  if (count == 0 || lo > reach + t[0].s * t[0].n) return false;
  const wide first = lo > reach ? (lo - reach + t[0].s - 1) / t[0].s : 0, last = std::min(hi / t[0].s, t[0].n);
  for (wide x = first; x <= last; ++x)
    if (--tries < 0 || reaches(t + 1, count - 1, lo - x * t[0].s, hi - x * t[0].s, tries)) return true;
  return false;
}

// Whether a row of a and a row of b share a byte.
inline bool share_memory(const RowSet& a, const RowSet& b) {
  struct { wide lo, hi; } range[2];
  const RowSet* set[2] = {&a, &b};
  for (int k = 0; k < 2; ++k) {
    range[k] = {(wide)reinterpret_cast<uintptr_t>(set[k]->p), (wide)reinterpret_cast<uintptr_t>(set[k]->p) + set[k]->bytes};
    for (int i = 0; i < 3; ++i) {
      if (set[k]->count[i] < 1) return false;
      const wide d = set[k]->stride[i] * (set[k]->count[i] - 1);
      (d < 0 ? range[k].lo : range[k].hi) += d;
    }
  }
  if (range[0].hi <= range[1].lo || range[1].hi <= range[0].lo) return false;
  // rows meet where address of a's - address of b's is above -(a's width) and below b's; terms that differ in sign alone are one
  wide lo = (wide)reinterpret_cast<uintptr_t>(b.p) - (wide)reinterpret_cast<uintptr_t>(a.p), hi = lo;
  lo -= a.bytes - 1;
  hi += b.bytes - 1;
  Term t[6];
  int n = 0;
  for (int k = 0; k < 2; ++k)
    for (int i = 0; i < 3; ++i) {
      wide s = k == 0 ? set[k]->stride[i] : -set[k]->stride[i];
      const wide most = set[k]->count[i] - 1;
      if (s == 0 || most == 0) continue;
      if (s < 0) {                             // x counts down from the most
        lo -= s * most;
        hi -= s * most;
        s = -s;
      }
      int j = 0;
      while (j < n && t[j].s != s) ++j;
      if (j == n) t[n++] = {s, 0};
      t[j].n += most;
    }
  std::sort(t, t + n, [](const Term& x, const Term& y) { return x.s > y.s; });
  int tries = 1 << 16;
  return reaches(t, n, lo, hi, tries);
}

// A norm's output may be its input, row by row in place; it must not overlap it otherwise (rows are loaded before earlier ones are stored).
inline int32_t check_in_place(const RowSet& out, const RowSet& in, const char* who, const char* names) {
  const bool same = out.p == in.p && (out.count[0] == 1 || out.stride[0] == in.stride[0]);
  if (!same && share_memory(out, in)) return fail(RSLX_ERR_INVALID_ARG, "%s: %s overlap and are not the same matrix", who, names);
  return RSLX_OK;
}

// Whether two rows of a share a byte.
inline bool overlaps_itself(const RowSet& a) {
  Term t[3];
  int n = 0;
  for (int i = 0; i < 3; ++i) {
    if (a.count[i] < 1) return false;
    if (a.count[i] > 1) t[n++] = {a.stride[i] < 0 ? -a.stride[i] : a.stride[i], a.count[i] - 1};
  }
  std::sort(t, t + n, [](const Term& x, const Term& y) { return x.s > y.s; });
  // rows inside rows: every distance is longer than what all shorter ones together cover
  wide covered = a.bytes;
  bool apart = true;
  for (int i = n - 1; i >= 0; --i) {
    apart = apart && t[i].s >= covered;
    covered += t[i].s * t[i].n;
  }
  if (apart) return false;
  // otherwise two rows whose places differ in dimension i first, upwards: 1 to n there, -n to n in the ones behind it
  int tries = 1 << 16;
  for (int i = 0; i < n; ++i) {
    Term d[3];
    int m = 0;
    wide lo = 1 - a.bytes - t[i].s;
    d[m++] = {t[i].s, t[i].n - 1};
    for (int j = i + 1; j < n; ++j) {
      lo += t[j].s * t[j].n;
      d[m++] = {t[j].s, 2 * t[j].n};
    }
    while (m > 0 && d[m - 1].s == 0) --m;
    if (reaches(d, m, lo, lo + 2 * (a.bytes - 1), tries)) return true;
  }
  return false;
}

// What a call reads or writes, by name; `p` null: not there.
struct Named {
  RowSet rows;
  const char* name;
};
// Outputs (the first of x) must not share memory with inputs or with each other.
template <int COUNT>
int32_t check_apart(const Named (&x)[COUNT], int outputs, const char* who) {
  for (int i = 0; i < outputs; ++i)
    for (int j = i + 1; j < COUNT; ++j)
      if (x[i].rows.p && x[j].rows.p && share_memory(x[i].rows, x[j].rows)) return fail(RSLX_ERR_INVALID_ARG, "%s: %s overlaps %s", who, x[i].name, x[j].name);
  return RSLX_OK;
}

// Whether an output's row lies where an input's row of the same sequence and head begins, and meets no other.
inline bool same_rows(const RowSet& out, const RowSet& in) {
  if (out.p != in.p) return false;
  for (int i = 0; i < 3; ++i)
    if (out.count[i] > 1 && out.stride[i] != in.stride[i]) return false;
  RowSet wider = out;
  wider.bytes = std::max(out.bytes, in.bytes);
  return !overlaps_itself(wider);
}

}  // namespace host
}  // namespace rslx
