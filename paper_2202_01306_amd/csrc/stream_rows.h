// Rows of the residual stream, eight columns at a time: what the kernels of embedding.hip and rows8.hip share.
#pragma once

#include "logit_rows.h"

namespace hmy {

// A row of d columns is worked through as units of eight columns.  The last one, where d is no multiple of eight, begins at column
// d - 8, so that every lane's loads are wide, unconditional and inside of the row (a branch around a load would make the lanes wait for
// it before the next is sent): its first `skip` columns are the unit's before it.  Units behind the row have skip = 8: nothing is
// theirs.  Rows of fewer than eight columns (NARROW) are one unit, read element by element.
struct Unit {
  int c, skip;
};
template <bool NARROW> __device__ __forceinline__ Unit unit_at(int c, int d) {
  if constexpr (NARROW) return {0, c > 0 ? 8 : 0};
  const int over = c - (d - 8);
  return over > 0 ? Unit{d - 8, min(over, 8)} : Unit{c, 0};
}
template <bool NARROW, typename E> __device__ __forceinline__ void load_unit(Eight<E> &v, const E *row, Unit u, int d) {
  if constexpr (!NARROW) {
    load_whole(v, row + u.c);
  } else {
#pragma unroll
    for (int i = 0; i < Eight<E>::WORDS; ++i) v.w[i] = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < d) {
        if constexpr (sizeof(E) == 4) v.w[k] = __float_as_uint(to_f32(row[k]));
        else v.w[k / 2] |= (__float_as_uint(to_f32(row[k])) >> 16) << (16 * (k % 2));
      }
  }
}
template <bool NARROW, typename E> __device__ __forceinline__ void store_unit(E *row, const float (&v)[8], Unit u, int d) {
  if constexpr (!NARROW) {
    if (u.skip == 0) {
      store_whole(row + u.c, v);
    } else if (u.skip < 8) {
#pragma unroll
      for (int k = 1; k < 8; ++k)
        if (k >= u.skip) row[u.c + k] = from_f32<E>(v[k]);
    }
  } else if (u.skip == 0) {
#pragma unroll
    for (int k = 0; k < 7; ++k)
      if (k < d) row[k] = from_f32<E>(v[k]);
  }
}
// zeros in the columns that are not the unit's own
template <bool NARROW> __device__ __forceinline__ void clear_foreign(float (&v)[8], Unit u, int d) {
  if constexpr (NARROW) {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k >= d || u.skip) v[k] = 0.f;
  } else if (u.skip) {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < u.skip) v[k] = 0.f;
  }
}

// ---- on the host ----
inline bool known_prec(int prec) { return prec == HMY_PREC_FP32 || prec == HMY_PREC_BF16; }

// an array of T rows of d elements of `bytes` each at a stride of ld elements
inline int check_array(const char *who, const char *what, const void *p, int bytes, int64_t T, int64_t d, int64_t ld) {
  if (ld < d) return fail(HMY_E_INVALID, "%s: a row stride of %lld does not hold the %lld columns of %s", who, (long long)ld, (long long)d, what);
  if (ld > (int64_t(1) << 46) / T) return fail(HMY_E_INVALID, "%s: row stride of %s out of range", who, what);
  if (misaligned(p, bytes)) return fail(HMY_E_INVALID, "%s: %s not aligned to its elements", who, what);
  return HMY_OK;
}
inline int check_extent(const char *who, int T, int d, int most) {
  if (T < 1 || d < 1 || d > most) return fail(HMY_E_INVALID, "%s: T >= 1 and 1 <= d <= %d wanted, got T = %d, d = %d", who, most, T, d);
  return HMY_OK;
}

// T rows of `cols` bytes at a pitch of `ld` bytes
struct Span {
  const char *name;
  const void *p;
  int64_t cols, ld, T;
  bool written;
};
inline bool spans_clash(const Span &a, const Span &b) {
  if (!a.p || !b.p) return false;
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
  const uintptr_t ea = pa + uintptr_t(a.T - 1) * uintptr_t(a.ld) + uintptr_t(a.cols), eb = pb + uintptr_t(b.T - 1) * uintptr_t(b.ld) + uintptr_t(b.cols);
  if (ea <= pb || eb <= pa) return false;
  if (a.ld == b.ld) {   // rows of one pitch may lie side by side in a wider array
    const uintptr_t ld = uintptr_t(a.ld), off = pb >= pa ? (pb - pa) % ld : (ld - (pa - pb) % ld) % ld;
    return !(off >= uintptr_t(a.cols) && off + uintptr_t(b.cols) <= ld);
  }
  return true;
}
template <int N> inline int check_apart(const char *who, const Span (&spans)[N]) {
  for (int i = 0; i < N; ++i)
    for (int j = i + 1; j < N; ++j)
      if ((spans[i].written || spans[j].written) && spans_clash(spans[i], spans[j]))
        return fail(HMY_E_INVALID, "%s: %s overlaps %s", who, spans[i].name, spans[j].name);
  return HMY_OK;
}

}  // namespace hmy
