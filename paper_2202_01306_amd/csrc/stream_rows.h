// Rows of the residual stream, eight columns at a time: what the kernels of embedding.hip and rows8.hip share.
#pragma once

#include "logit_rows.h"

namespace hmy {

// The first n columns from p on, zeros behind them.  Whole groups take wide accesses at any alignment.
template <typename E> __device__ __forceinline__ void load_columns(float (&v)[8], const E *p, int n) {
  if (n >= 8) {
    Eight<E> e;
    load_whole(e, p);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = e.at(k);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = k < n ? to_f32(p[k]) : 0.f;
  }
}
template <typename E> __device__ __forceinline__ void store_columns(E *p, const float (&v)[8], int n) {
  if (n >= 8) {
    store_whole(p, v);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < n) p[k] = from_f32<E>(v[k]);
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
