// Rows of logits, eight columns at a time: what the kernels of logprob.hip and distill.hip share.
#pragma once

#include <cmath>

#include "dev_common.h"
#include "hmy_internal.h"

namespace hmy {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLog2eLow = 1.9259629911e-8f;   // log2(e) - kLog2e
constexpr float kLn2 = 0.6931471805599453f;
// below this (log2 units) an exponential is 0 and so is its product with its exponent, which may be -inf
constexpr float kNoWeight = -1e4f;

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// exp(s (a - m)) to the last bits, for what whole partial sums are multiplied with: the product with s log2(e) rounds, which
// costs |s (a - m)| 2^-24 relative; here the rounded part is carried along.  a <= m; a = -inf gives 0, and so does the type's
// lowest value beside an ordinary one, whose products here are no longer finite.
__device__ __forceinline__ float rebase(float a, float m, float scale) {
  const float d = (a - m) * scale, hi = d * kLog2e;
  if (a == -INFINITY || d < -200.f) return 0.f;
  const float lo = fmaf(d, kLog2e, -hi) + d * kLog2eLow;
  return fast_exp2(hi) * fmaf(lo, kLn2, 1.f);
}

// Reductions over a wave by moves between neighbouring lanes, without LDS; the result is the same scalar for all lanes.  Lanes
// that a move gives nothing take the operation's neutral element.
template <int CTRL, int ROWS> __device__ __forceinline__ float lane_move(float x, float neutral) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(neutral), __float_as_uint(x), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float last_lane(float x) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), 63)); }
__device__ __forceinline__ float wave_total(float x) {
  x += lane_move<0x111, 0xf>(x, 0.f);   // within rows of sixteen lanes: from 1, 2, 4 and 8 lanes before
  x += lane_move<0x112, 0xf>(x, 0.f);
  x += lane_move<0x114, 0xf>(x, 0.f);
  x += lane_move<0x118, 0xf>(x, 0.f);
  x += lane_move<0x142, 0xa>(x, 0.f);   // a row's last lane to the next row
  x += lane_move<0x143, 0xc>(x, 0.f);   // lane 31 to the upper half
  return last_lane(x);
}
__device__ __forceinline__ float wave_top(float x) {
  x = fmaxf(x, lane_move<0x111, 0xf>(x, -INFINITY));
  x = fmaxf(x, lane_move<0x112, 0xf>(x, -INFINITY));
  x = fmaxf(x, lane_move<0x114, 0xf>(x, -INFINITY));
  x = fmaxf(x, lane_move<0x118, 0xf>(x, -INFINITY));
  x = fmaxf(x, lane_move<0x142, 0xa>(x, -INFINITY));
  x = fmaxf(x, lane_move<0x143, 0xc>(x, -INFINITY));
  return last_lane(x);
}
template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t lane_move(uint32_t x, uint32_t neutral) {
  return __builtin_amdgcn_update_dpp(neutral, x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ uint32_t wave_top(uint32_t x) {
  x = max(x, lane_move<0x111, 0xf>(x, 0u));
  x = max(x, lane_move<0x112, 0xf>(x, 0u));
  x = max(x, lane_move<0x114, 0xf>(x, 0u));
  x = max(x, lane_move<0x118, 0xf>(x, 0u));
  x = max(x, lane_move<0x142, 0xa>(x, 0u));
  x = max(x, lane_move<0x143, 0xc>(x, 0u));
  return __builtin_amdgcn_readlane(x, 63);
}
template <int CTRL, int ROWS> __device__ __forceinline__ double lane_move(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, uint32_t(b), CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, uint32_t(b >> 32), CTRL, ROWS, 0xf, false);
  return __builtin_bit_cast(double, uint64_t(hi) << 32 | lo);
}
__device__ __forceinline__ double wave_total(double x) {
  x += lane_move<0x111, 0xf>(x);
  x += lane_move<0x112, 0xf>(x);
  x += lane_move<0x114, 0xf>(x);
  x += lane_move<0x118, 0xf>(x);
  x += lane_move<0x142, 0xa>(x);
  x += lane_move<0x143, 0xc>(x);
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_readlane(uint32_t(b), 63), hi = __builtin_amdgcn_readlane(uint32_t(b >> 32), 63);
  return __builtin_bit_cast(double, uint64_t(hi) << 32 | lo);
}

// Eight columns as they are stored.  The accesses are 16 bytes wide and aligned to the element only: rows of any stride take
// the same path (the device splits what crosses a cache line).
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_by2 __attribute__((aligned(2)));
typedef u32x4 u32x4_by4 __attribute__((aligned(4)));
template <typename E> struct Unaligned { typedef u32x4_by4 type; };
template <> struct Unaligned<bf16_t> { typedef u32x4_by2 type; };
template <typename E> struct alignas(16) Eight {
  static constexpr int WORDS = 8 * sizeof(E) / 4;
  uint32_t w[WORDS];
  __device__ __forceinline__ float at(int k) const {
    if constexpr (sizeof(E) == 4) return __uint_as_float(w[k]);
    else return __uint_as_float(k & 1 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16);
  }
  // -inf in the columns whose bits are set
  __device__ __forceinline__ void set_no_weight(uint32_t bits) {
    auto all = [&](int k) { return uint32_t(int32_t(bits << (31 - k)) >> 31); };
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if constexpr (sizeof(E) == 4) {
        w[k] = (w[k] & ~all(k)) | (all(k) & 0xff800000u);
      } else if (k % 2 == 0) {
        const uint32_t m = (all(k) & 0xffffu) | (all(k + 1) & 0xffff0000u);
        w[k / 2] = (w[k / 2] & ~m) | (m & 0xff80ff80u);
      }
    }
  }
  // keeps the compiler from holding on to values that were taken apart before this point: a bf16 row fits the registers as loaded,
  // but not as floats
  __device__ __forceinline__ void forget_floats() {
    if constexpr (sizeof(E) == 2) {
#pragma unroll
      for (int i = 0; i < WORDS; ++i) asm volatile("" : "+v"(w[i]));
    }
  }
  __device__ __forceinline__ void all_no_weight() {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) w[i] = sizeof(E) == 4 ? 0xff800000u : 0xff80ff80u;
  }
};
template <typename E> __device__ __forceinline__ void load_whole(Eight<E> &v, const E *p) {
  typedef typename Unaligned<E>::type unaligned;
#pragma unroll
  for (int i = 0; i < Eight<E>::WORDS; i += 4) {
    const u32x4 a = *reinterpret_cast<const unaligned *>(reinterpret_cast<const char *>(p) + 4 * i);
    v.w[i] = a.x; v.w[i + 1] = a.y; v.w[i + 2] = a.z; v.w[i + 3] = a.w;
  }
}
template <typename E> __device__ __forceinline__ void store_whole(E *p, const float (&g)[8]) {
  typedef typename Unaligned<E>::type unaligned;
  Eight<E> o;
  if constexpr (sizeof(E) == 4) {
#pragma unroll
    for (int k = 0; k < 8; ++k) o.w[k] = __float_as_uint(g[k]);
  } else {
    typedef E pair __attribute__((ext_vector_type(2)));
    typedef float floats __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int k = 0; k < 8; k += 2) {   // both halves of a word by one instruction
      floats f;
      f.x = g[k];
      f.y = g[k + 1];
      o.w[k / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, pair));
    }
  }
#pragma unroll
  for (int i = 0; i < Eight<E>::WORDS; i += 4) {
    u32x4 a;
    a.x = o.w[i]; a.y = o.w[i + 1]; a.z = o.w[i + 2]; a.w = o.w[i + 3];
    *reinterpret_cast<unaligned *>(reinterpret_cast<char *>(p) + 4 * i) = a;
  }
}
// A row is its V / 8 whole groups of eight columns, and the V % 8 columns behind them, one thread's each.
template <typename E> __device__ __forceinline__ void zero_padding(E *row, int V, int pad, int tid, int nt) {
  for (int j = V + tid; j < V + pad; j += nt) row[j] = from_f32<E>(0.f);
}

// ---- on the host ----
constexpr int kMaxGrid = 1 << 20;   // workgroups of a launch; rows beyond are taken in further rounds
constexpr int kMaxColumns = 1 << 24;

inline bool misaligned(const void *p, int to) { return (reinterpret_cast<uintptr_t>(p) & uintptr_t(to - 1)) != 0; }
inline int bytes_of(int prec) { return prec == HMY_PREC_BF16 ? 2 : 4; }
inline bool usable_scale(float s) { return s > 0.f && std::isfinite(s * kLog2e); }
inline bool has_workspace(const void *p, uint64_t bytes) { return p && bytes >= uint64_t(HMY_ROWS_WORKSPACE_BYTES); }

inline int check_launch(const char *what) {
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(HMY_E_HIP, "launch of %s failed: %s", what, hipGetErrorString(e));
  return HMY_OK;
}

inline int check_rows(const char *who, int prec, const void *p, int T, int V, int pad, int64_t ld) {
  if (prec != HMY_PREC_FP32 && prec != HMY_PREC_BF16) return fail(HMY_E_INVALID, "%s: unknown precision %d", who, prec);
  if (T < 1 || V < 1 || V > kMaxColumns) return fail(HMY_E_INVALID, "%s: T >= 1 and 1 <= V <= %d wanted, got T = %d, V = %d", who, kMaxColumns, T, V);
  if (pad < 0 || ld < int64_t(V) + pad) return fail(HMY_E_INVALID, "%s: a row stride of %lld does not hold %d columns and a padding of %d", who, (long long)ld, V, pad);
  if (ld > (int64_t(1) << 46) / T) return fail(HMY_E_INVALID, "%s: row stride out of range", who);
  if (pad > (1 << 30)) return fail(HMY_E_INVALID, "%s: padding out of range", who);
  if (misaligned(p, bytes_of(prec))) return fail(HMY_E_INVALID, "%s: rows not aligned to their elements", who);
  return HMY_OK;
}

// Whether rows of `a_cols` and `b_cols` bytes at pitches of `a_ld` and `b_ld` bytes share memory, other than as the same rows of
// the same type (in place).  Rows of one pitch may lie side by side in a wider array.
inline bool rows_clash(const void *a, int64_t a_cols, int64_t a_ld, const void *b, int64_t b_cols, int64_t b_ld, int T, bool same_type) {
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
  if (pa == pb && a_ld == b_ld && same_type) return false;
  const uintptr_t ea = pa + uintptr_t(T - 1) * uintptr_t(a_ld) + uintptr_t(a_cols), eb = pb + uintptr_t(T - 1) * uintptr_t(b_ld) + uintptr_t(b_cols);
  if (ea <= pb || eb <= pa) return false;
  if (a_ld == b_ld) {
    const int64_t off = int64_t((pb >= pa ? pb - pa : a_ld - (pa - pb) % uintptr_t(a_ld)) % uintptr_t(a_ld));
    return !(off >= a_cols && off + b_cols <= a_ld);
  }
  return true;
}

#define DISPATCH_ROWS(lp, ep, ...)                                                                       \
  do {                                                                                                   \
    if ((lp) == HMY_PREC_BF16) {                                                                         \
      typedef bf16_t L;                                                                                  \
      if ((ep) == HMY_PREC_BF16) { typedef bf16_t E; __VA_ARGS__ } else { typedef float E; __VA_ARGS__ } \
    } else {                                                                                             \
      typedef float L;                                                                                   \
      if ((ep) == HMY_PREC_BF16) { typedef bf16_t E; __VA_ARGS__ } else { typedef float E; __VA_ARGS__ } \
    }                                                                                                    \
  } while (0)

}  // namespace hmy
