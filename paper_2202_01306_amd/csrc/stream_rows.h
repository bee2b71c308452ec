// Rows of the residual stream, eight columns at a time: what the kernels of embedding.hip and rows8.hip share.
#pragma once

#include "logit_rows.h"

namespace hmy {

// A row of d columns is worked through as units of N = 4 or 8 neighbouring columns a lane, so many that a lane's widest access takes 16
// bytes: then an instruction of a wave covers a kilobyte without holes (fp32 rows of 134 MB written in units of 8 columns: see k_unpack8).
// The last unit, where d is no multiple of N, begins at column d - N, so that every lane's loads are wide, unconditional and inside of the
// row (a branch around a load would make the lanes wait for it before the next is sent): its first `skip` columns are the unit's before
// it.  Units behind the row have skip = N: nothing is theirs.  Rows of fewer than eight columns (NARROW) are read element by element.
struct Unit {
  int c, skip;
};
template <bool NARROW, int N> __device__ __forceinline__ Unit unit_at(int c, int d) {
  if constexpr (NARROW) return {c, c < d ? 0 : N};
  const int over = c - (d - N);
  return over > 0 ? Unit{d - N, min(over, N)} : Unit{c, 0};
}
template <bool NARROW, int N> __device__ __forceinline__ bool owns(Unit u, int k, int d) { return k >= u.skip && (!NARROW || u.c + k < d); }

// N columns as they are stored.
template <typename E, int N> struct Cols {
  static constexpr int WORDS = N * sizeof(E) / 4;
  uint32_t w[WORDS];
  __device__ __forceinline__ float at(int k) const {
    if constexpr (sizeof(E) == 4) return __uint_as_float(w[k]);
    else return __uint_as_float(k & 1 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16);
  }
};
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_by1 __attribute__((aligned(1)));
typedef u32x2 u32x2_by2 __attribute__((aligned(2)));
typedef uint32_t u32_by1 __attribute__((aligned(1)));
// ONCE: a streaming load, whose data the caches do not keep.  For rows that are read once and are kStreamed bytes or more: a third of the
// memory-side cache of 256 MB, where fewer are found if the last two or three kernels have had them.  What it gives depends on what came before and
// on the width (both sides stand at the kernels): with three sets of rows in turn 3 to 9 % from 84 MB on, -1 % at 328 MB of rows of 5000 columns, 0 at
// 210 MB of 1601 in bf16, -3 to -11 % at 67 MB; with rows that the kernel just before has written, and which the cache still holds, 6 to 43 % from 268
// MB on (0 at the 210 MB of 1601), 0 to -5 % at 84 and 134 MB.
constexpr int64_t kStreamed = int64_t(80) << 20;
template <bool NARROW, bool ONCE = false, typename E, int N> __device__ __forceinline__ void load_unit(Cols<E, N> &v, const E *row, Unit u, int d) {
  const char *p = reinterpret_cast<const char *>(row + u.c);
  if constexpr (NARROW) {
#pragma unroll
    for (int i = 0; i < Cols<E, N>::WORDS; ++i) v.w[i] = 0;
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (u.c + k < d) {
        if constexpr (sizeof(E) == 4) v.w[k] = __float_as_uint(to_f32(row[u.c + k]));
        else v.w[k / 2] |= (__float_as_uint(to_f32(row[u.c + k])) >> 16) << (16 * (k % 2));
      }
  } else if constexpr (Cols<E, N>::WORDS == 2) {
    const u32x2_by2 *from = reinterpret_cast<const u32x2_by2 *>(p);
    const u32x2 a = ONCE ? __builtin_nontemporal_load(from) : *from;
    v.w[0] = a.x; v.w[1] = a.y;
  } else {
    typedef typename Unaligned<E>::type unaligned;
#pragma unroll
    for (int i = 0; i < Cols<E, N>::WORDS; i += 4) {
      const unaligned *from = reinterpret_cast<const unaligned *>(p + 4 * i);
      const u32x4 a = ONCE ? __builtin_nontemporal_load(from) : *from;
      v.w[i] = a.x; v.w[i + 1] = a.y; v.w[i + 2] = a.z; v.w[i + 3] = a.w;
    }
  }
}
template <bool NARROW, typename E, int N> __device__ __forceinline__ void store_unit(E *row, const float (&v)[N], Unit u, int d) {
  if (!NARROW && u.skip == 0) {
    Cols<E, N> o;
    if constexpr (sizeof(E) == 4) {
#pragma unroll
      for (int k = 0; k < N; ++k) o.w[k] = __float_as_uint(v[k]);
    } else {
      typedef E pair __attribute__((ext_vector_type(2)));
      typedef float floats __attribute__((ext_vector_type(2)));
#pragma unroll
      for (int k = 0; k < N; k += 2) {   // both halves of a word by one instruction
        floats f;
        f.x = v[k];
        f.y = v[k + 1];
        o.w[k / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, pair));
      }
    }
    char *p = reinterpret_cast<char *>(row + u.c);
    if constexpr (Cols<E, N>::WORDS == 2) {
      u32x2 a;
      a.x = o.w[0]; a.y = o.w[1];
      *reinterpret_cast<u32x2_by2 *>(p) = a;
    } else {
      typedef typename Unaligned<E>::type unaligned;
#pragma unroll
      for (int i = 0; i < Cols<E, N>::WORDS; i += 4) {
        u32x4 a;
        a.x = o.w[i]; a.y = o.w[i + 1]; a.z = o.w[i + 2]; a.w = o.w[i + 3];
        *reinterpret_cast<unaligned *>(p + 4 * i) = a;
      }
    }
  } else if (u.skip < N) {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (owns<NARROW, N>(u, k, d)) row[u.c + k] = from_f32<E>(v[k]);
  }
}
// zeros in the columns that are not the unit's own
template <bool NARROW, int N> __device__ __forceinline__ void clear_foreign(float (&v)[N], Unit u, int d) {
  if (NARROW || u.skip) {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (!owns<NARROW, N>(u, k, d)) v[k] = 0.f;
  }
}

// ---- the units of rows, shared out over a launch ----
// Wide rows: a wave takes K units a lane of a row, or of two or four rows where it has few, with everything but the column in scalar
// registers; tiles of kWaves waves, one chunk of their rows after the other.  K = 0: rows of less than half a wave's units are numbered through instead,
// unit by unit, and a lane finds its row by one 32-bit division from that of its workgroup's first (a lookup of 32768 x 1024 fp32 took 46 us
// that way, 43 by waves).
constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int per_thread(int K) { return K == 3 ? 3 : 4; }   // units

struct Units {
  int T, d;
  uint32_t per_row;           // K = 0: units in a row
  uint32_t chunks;            // of 64 K N columns in a row
  int64_t tiles;              // times chunks
};
template <int PER> struct Places {
  int64_t row[PER];
  Unit u[PER];
};
// a / b, of which the 64-bit division's hundred instructions are left out where a has 32 bits, as it has nearly always
__device__ __forceinline__ int64_t quotient(int64_t a, uint32_t b) { return a >> 32 ? a / b : int64_t(uint32_t(a) / b); }

// Where the thread's units are; for those behind the last row's another row is read, and nothing of it is theirs.
template <int K, bool NARROW, int N> __device__ __forceinline__ Places<per_thread(K)> places_of(const Units &g, int64_t tile) {
  constexpr int kPerThread = per_thread(K);
  Places<kPerThread> p;
  const int lane = threadIdx.x % kWave;
  if constexpr (K > 0) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t rows = g.chunks == 1 ? tile : quotient(tile, g.chunks);
    const int chunk = int(tile - rows * g.chunks);
    const int64_t row0 = (rows * kWaves + wave) * (kPerThread / K);
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
      const int64_t row = row0 + i / K;
      p.row[i] = min(row, int64_t(g.T) - 1);
      p.u[i] = unit_at<NARROW, N>(((chunk * K + i % K) * kWave + lane) * N, g.d);
      if (row >= g.T) p.u[i].skip = N;
    }
  } else {
    constexpr int kUnits = kThreads * kPerThread;
    const int64_t row0 = quotient(tile * kUnits, g.per_row);
    const uint32_t first = uint32_t(tile * kUnits - row0 * g.per_row);
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
      const uint32_t at = first + threadIdx.x + i * kThreads, down = at / g.per_row;
      const bool there = row0 + down < g.T;
      p.u[i] = unit_at<NARROW, N>(int(at - down * g.per_row) * N, g.d);
      p.row[i] = there ? row0 + down : row0;
      if (!there) p.u[i].skip = N;
    }
  }
  return p;
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

// How rows of d columns in units of N, rounded up to `whole` columns, are shared out: K, and the launch's extent.
struct Shares {
  Units units;
  int K;
  dim3 grid;
};
inline Shares shares_of(int T, int d, int N, int whole) {
  Shares s;
  const int per_row = (d + whole - 1) / whole * (whole / N), waves = (per_row + kWave - 1) / kWave;
  // chunks of up to four waves' units, as even as they go (a lookup of 20000 rows of 1096 fp32 columns, in
  // chunks of 3 and 2 instead of 4 and 1: 37 us instead of 42); a branch around units that are no one's costs more than they do
  const int chunks = (waves + 3) / 4;
  s.K = per_row < kWave / 2 ? 0 : (waves + chunks - 1) / chunks;
  s.units = {T, d, uint32_t(per_row), s.K ? uint32_t(chunks) : 1u, 0};
  const int per = per_thread(s.K);
  const int64_t parts = s.K ? (int64_t(T) + per / s.K - 1) / (per / s.K) : (int64_t(T) * per_row + kWave * per - 1) / (kWave * per);
  s.units.tiles = (parts + kWaves - 1) / kWaves * s.units.chunks;
  s.grid = dim3(uint32_t(s.units.tiles < kMaxGrid ? s.units.tiles : kMaxGrid));
  return s;
}
#define DISPATCH_SHARES(k, d, ...)                                                   \
  do {                                                                               \
    constexpr bool NARROW = false;                                                   \
    if ((d) < 8) { constexpr int K = 0; constexpr bool NARROW = true; __VA_ARGS__ }  \
    else if ((k) == 0) { constexpr int K = 0; __VA_ARGS__ }                          \
    else if ((k) == 1) { constexpr int K = 1; __VA_ARGS__ }                          \
    else if ((k) == 2) { constexpr int K = 2; __VA_ARGS__ }                          \
    else if ((k) == 3) { constexpr int K = 3; __VA_ARGS__ }                          \
    else { constexpr int K = 4; __VA_ARGS__ }                                        \
  } while (0)

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
