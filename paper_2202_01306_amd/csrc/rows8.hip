// Rows of the residual stream held in 8 bits with a power of two for each 32 columns, and the layer norm that reads them.
//
// A power of two as the scale makes every step but the one rounding exact: x 2^-e and q 2^e change no digit, so that what is read is
// the same on every path, an 8-bit integer times a scale is a bf16 number as it stands, and a scale is one byte, which pays for groups
// of 32 columns (3 % more bytes) where 32-bit scales would want 128.  What it costs is up to one bit of an INT8 group's range.
// All kernels here are bound by HBM where there are many rows: 5.03 bytes per element for fp32 rows to or from 8 bits.
#include <algorithm>

#include "stream_rows.h"

namespace hmy {

namespace {

constexpr int kGroup = HMY_ROWS8_GROUP;

struct Rows8 {
  const uint8_t *codes, *scales;
  int64_t ldc, lds;
};

// The largest value of a group's lanes, of which each has N of its columns.
template <int N> __device__ __forceinline__ uint32_t group_top(uint32_t x) {
  x = max(x, uint32_t(__builtin_amdgcn_update_dpp(0, x, 0xb1, 0xf, 0xf, false)));   // from lane ^ 1
  x = max(x, uint32_t(__builtin_amdgcn_update_dpp(0, x, 0x4e, 0xf, 0xf, false)));   // from lane ^ 2
  if constexpr (N == 4) x = max(x, uint32_t(__builtin_amdgcn_update_dpp(0, x, 0x141, 0xf, 0xf, false)));   // from the other four of eight
  return x;
}

// The scale's byte for a group whose largest magnitude has these bits, e + 127 for the least e >= -126 with a <= top 2^e.  The
// exponent's field of a, one more where the mantissa is above top's: an addition that carries into the field says so.
template <int CODE> __device__ __forceinline__ uint32_t scale_byte(uint32_t a) {
  constexpr uint32_t kCarry = CODE == HMY_CODE_INT8 ? 0x01ffffu : 0x1fffffu;   // 0x7fffff less the mantissa of 127, of 448
  constexpr int kTop = CODE == HMY_CODE_INT8 ? 6 : 8;                          // their exponents
  const int e = int((a + kCarry) >> 23) - kTop;
  return a >= 0x7f800000u ? 255u : uint32_t(max(e, 1));
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return byte == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(byte << 23); }

// Four columns to four codes.  INT8: adding 1.5 2^23 leaves the whole number, rounded to nearest even, in the sum's last bits, and the
// multiply-add rounds once.
template <int CODE> __device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d, float inv) {
  if constexpr (CODE == HMY_CODE_INT8) {
    constexpr float kWhole = 12582912.f;
    const uint32_t ia = __float_as_uint(fmaf(a, inv, kWhole)), ib = __float_as_uint(fmaf(b, inv, kWhole));
    const uint32_t ic = __float_as_uint(fmaf(c, inv, kWhole)), id = __float_as_uint(fmaf(d, inv, kWhole));
    const uint32_t lo = __builtin_amdgcn_perm(ib, ia, 0x0c0c0400u), hi = __builtin_amdgcn_perm(id, ic, 0x04000c0cu);
    return lo | hi;
  } else {
    uint32_t w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, w, true);
  }
}
template <int CODE> __device__ __forceinline__ void decode4(uint32_t w, float s, float *v) {
  if constexpr (CODE == HMY_CODE_INT8) {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = float(int8_t(w >> (8 * k))) * s;
  } else {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    v[0] = lo[0] * s;
    v[1] = lo[1] * s;
    v[2] = hi[0] * s;
    v[3] = hi[1] * s;
  }
}

// A unit's codes.
template <bool NARROW, int N> __device__ __forceinline__ void load_codes(uint32_t (&w)[N / 4], const uint8_t *row, Unit u, int d) {
  if constexpr (NARROW) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) w[i] = 0;
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (u.c + k < d) w[k / 4] |= uint32_t(row[u.c + k]) << (8 * (k % 4));
  } else if constexpr (N == 8) {
    const u32x2 a = *reinterpret_cast<const u32x2_by1 *>(row + u.c);
    w[0] = a.x; w[1] = a.y;
  } else {
    w[0] = *reinterpret_cast<const u32_by1 *>(row + u.c);
  }
}
template <bool NARROW, int N> __device__ __forceinline__ void store_codes(uint8_t *row, const uint32_t (&w)[N / 4], Unit u, int d) {
  if (!NARROW && u.skip == 0) {
    if constexpr (N == 8) {
      u32x2 a;
      a.x = w[0]; a.y = w[1];
      *reinterpret_cast<u32x2_by1 *>(row + u.c) = a;
    } else {
      *reinterpret_cast<u32_by1 *>(row + u.c) = w[0];
    }
  } else if (u.skip < N) {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (owns<NARROW, N>(u, k, d)) row[u.c + k] = uint8_t(w[k / 4] >> (8 * (k % 4)));
  }
}
// Its scale is that of the group that its own columns are in: the last column's, whichever of them are its own.
template <bool NARROW, int N> __device__ __forceinline__ int group_of(Unit u) { return NARROW ? 0 : (u.c + N - 1) / kGroup; }
template <int CODE, int N> __device__ __forceinline__ void decode(const uint32_t (&w)[N / 4], uint32_t byte, float (&v)[N]) {
  const float s = scale_of(byte);
#pragma unroll
  for (int i = 0; i < N / 4; ++i) decode4<CODE>(w[i], s, v + 4 * i);
}

// 32768 x 4096 fp32, 537 MB read and 138 written: 111 us (6.1 TB/s); with a row's four chunks in four sweeps over all rows 14 more.
// ONCE, from kStreamed bytes on, calls with three sets of rows in turn: 114 us instead of 120, 65536 x 1024 59 and 62, 32768 x 1024 32 and 34, 20480 x
// 1024 22 and 24, but 16384 x 1024 18 and 16; bf16 20480 x 2048 25 and 27; it does not pay at bf16 65536 x 1601: 61 and 61.  With x written by the
// kernel just before: 109 us instead of 156, 65536 x 1024 53 and 68, but 32768 x 1024 29 and 28, 20480 x 1024 20.3 and 20.0, bf16 23.8 and 23.3.
template <typename E, int CODE, int K, bool NARROW, bool ONCE>
__global__ __launch_bounds__(kThreads) void k_pack8(const E *x, int64_t ldx, uint8_t *codes, int64_t ldc, uint8_t *scales, int64_t lds, Units g) {
  constexpr int N = 16 / sizeof(E);
  for (int64_t tile = blockIdx.x; tile < g.tiles; tile += gridDim.x) {
    constexpr int kPer = per_thread(K);
    const Places<kPer> p = places_of<K, NARROW, N>(g, tile);
    Cols<E, N> raw[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) load_unit<NARROW, ONCE>(raw[i], x + p.row[i] * ldx, p.u[i], g.d);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      float v[N];
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] = raw[i].at(k);
      clear_foreign<NARROW>(v, p.u[i], g.d);
      uint32_t a = 0;
#pragma unroll
      for (int k = 0; k < N; ++k) a = max(a, __float_as_uint(v[k]) & 0x7fffffffu);
      a = group_top<N>(a);
      const uint32_t byte = scale_byte<CODE>(a);
      const float inv = __uint_as_float((254u - byte) << 23);
      uint32_t w[N / 4];
#pragma unroll
      for (int k = 0; k < N; k += 4) w[k / 4] = byte == 255u ? 0u : encode4<CODE>(v[k], v[k + 1], v[k + 2], v[k + 3], inv);
      store_codes<NARROW, N>(codes + p.row[i] * ldc, w, p.u[i], g.d);
      if (p.u[i].skip < N && threadIdx.x % (kGroup / N) == 0) scales[p.row[i] * lds + group_of<NARROW, N>(p.u[i])] = uint8_t(byte);
    }
  }
}

// 32768 x 1024 to fp32, 35 MB read and 134 written: 31 us (5.4 TB/s).  In units of eight fp32 columns, whose two stores a lane leave holes
// of 16 bytes between neighbouring lanes, it took 36 to 39; marking the stores as streaming changes nothing.
template <typename E, int CODE, int K, bool NARROW>
__global__ __launch_bounds__(kThreads) void k_unpack8(Rows8 r, E *x, int64_t ldx, Units g) {
  constexpr int N = 16 / sizeof(E);
  for (int64_t tile = blockIdx.x; tile < g.tiles; tile += gridDim.x) {
    constexpr int kPer = per_thread(K);
    const Places<kPer> p = places_of<K, NARROW, N>(g, tile);
    uint32_t w[kPer][N / 4], byte[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      load_codes<NARROW, N>(w[i], r.codes + p.row[i] * r.ldc, p.u[i], g.d);
      byte[i] = r.scales[p.row[i] * r.lds + group_of<NARROW, N>(p.u[i])];
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      float v[N];
      decode<CODE>(w[i], byte[i], v);
      store_unit<NARROW>(x + p.row[i] * ldx, v, p.u[i], g.d);
    }
  }
}

// ---- layer norm of rows in 8 bits -------------------------------------------------------------

// A row is LPR lanes' of a wave (8, 16, 32 or 64: narrow rows lie side by side in one), or W waves', NJ units of kN columns a lane: wave w of
// a row has the units 64 NJ w + lane + 64 j.  Sums over a row: between lanes by moves, between waves through LDS, added in the same order
// by each of them.
constexpr int kN = 4;

template <int LPR> __device__ __forceinline__ float lanes_total(float x) {
  if constexpr (LPR == 64) return wave_total(x);
  x += lane_move<0xb1, 0xf>(x, 0.f);                            // from lane ^ 1
  x += lane_move<0x4e, 0xf>(x, 0.f);                            // from lane ^ 2
  x += lane_move<0x141, 0xf>(x, 0.f);                           // from the other four of eight
  if constexpr (LPR >= 16) x += lane_move<0x140, 0xf>(x, 0.f);  // from the other eight of sixteen
  if constexpr (LPR >= 32) x += __shfl_xor(x, 16, kWave);
  return x;
}
template <int LPR, int W, int M> __device__ __forceinline__ void row_sums(float (&s)[M], float (*xch)[M], int wave) {
#pragma unroll
  for (int i = 0; i < M; ++i) s[i] = lanes_total<LPR>(s[i]);
  if constexpr (W > 1) {
    if (threadIdx.x % kWave == 0)
#pragma unroll
      for (int i = 0; i < M; ++i) xch[wave][i] = s[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < M; ++i) {
      s[i] = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) s[i] += xch[wave / W * W + w][i];
    }
  }
}

struct Norm8 {
  Rows8 r;
  int T, d;
  int64_t ldy, ldx;
  float *mean, *rstd;
  float eps;
};

// A wave has ROWS rows (times 64 / LPR) on their way at a time; gamma and beta stay in registers.  One pass over the codes: the row is held
// in registers through mean, variance and output.  4096 x 1024 to bf16 with the rows themselves, 29.5 MB: 7.4 us (8 in a trace), of which 3 are a launch
// that does next to nothing; 16384 rows 25.6 (4.6 TB/s; 27.7 with one row on its way, which is 2 % faster at 4096).  Narrow rows: 131072 x
// 128 take 27 us side by side, 50 with a wave each.  As many units a lane as the row needs: 20000 x 1096 take 41 us with five, 52 with eight.
// Seven and eight units take 184 to 209 registers, two waves per SIMD, and one row is on its way: 4000 x 2048 to bf16 with the rows 12.5 us (4.6
// TB/s), to fp32 without them 10.8 (3.8), 4000 x 8192 51 (4.5) and 44 (3.7); 4000 x 4096 with four units 27.6 (4.2) and 16.8 (4.9).
template <typename E, int CODE, int LPR, int W, int NJ, int ROWS, bool NARROW>
__global__ __launch_bounds__(256) void k_layernorm8_fwd(Norm8 g, const E *gamma, const E *beta, E *y, float *x) {
  static_assert(LPR == 64 || (W == 1 && NJ == 1), "narrow rows are one unit a lane");
  constexpr int kAbreast = kWave / LPR, kSlot = ROWS * kAbreast, kSlots = 4 / W * kSlot;
  __shared__ float xch[2][2][4][ROWS];   // of a round's two sums, and of the round before, which a wave may still read
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  Unit u[NJ];
  Cols<E, kN> ga[NJ], be[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    u[j] = unit_at<NARROW, kN>(kN * (kWave * (NJ * (wave % W) + j) + lane % LPR), g.d);
    load_unit<NARROW>(ga[j], gamma, u[j], g.d);
    load_unit<NARROW>(be[j], beta, u[j], g.d);
  }
  int parity = 0;
  for (int64_t base = int64_t(blockIdx.x) * kSlots; base < g.T; base += int64_t(gridDim.x) * kSlots, parity ^= 1) {
    const int64_t first = base + wave / W * kSlot + (LPR < kWave ? lane / LPR : 0);
    float v[ROWS][NJ][kN], s[ROWS], mu[ROWS];
    uint32_t w[ROWS][NJ][kN / 4], byte[ROWS][NJ];
    int64_t row[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      row[r] = min(first + r * kAbreast, int64_t(g.T) - 1);   // one behind the last row does that row again, and stores nothing
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        load_codes<NARROW, kN>(w[r][j], g.r.codes + row[r] * g.r.ldc, u[j], g.d);
        byte[r][j] = g.r.scales[row[r] * g.r.lds + group_of<NARROW, kN>(u[j])];
      }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      s[r] = 0.f;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        decode<CODE>(w[r][j], byte[r][j], v[r][j]);
        clear_foreign<NARROW>(v[r][j], u[j], g.d);
#pragma unroll
        for (int k = 0; k < kN; ++k) s[r] += v[r][j][k];
      }
    }
    row_sums<LPR, W>(s, xch[parity][0], wave);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      mu[r] = s[r] / float(g.d);
      s[r] = 0.f;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        float t[kN];
#pragma unroll
        for (int k = 0; k < kN; ++k) t[k] = v[r][j][k] - mu[r];
        clear_foreign<NARROW>(t, u[j], g.d);
#pragma unroll
        for (int k = 0; k < kN; ++k) s[r] = fmaf(t[k], t[k], s[r]);
      }
    }
    row_sums<LPR, W>(s, xch[parity][1], wave);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (first + r * kAbreast >= g.T) continue;
      const float rs = 1.f / sqrtf(s[r] / float(g.d) + g.eps);
      if (lane % LPR == 0 && wave % W == 0) {
        if (g.mean) g.mean[row[r]] = mu[r];
        if (g.rstd) g.rstd[row[r]] = rs;
      }
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        float o[kN];
#pragma unroll
        for (int k = 0; k < kN; ++k) o[k] = fmaf(ga[j].at(k), (v[r][j][k] - mu[r]) * rs, be[j].at(k));
        store_unit<NARROW>(y + row[r] * g.ldy, o, u[j], g.d);
        if (x) store_unit<NARROW>(x + row[r] * g.ldx, v[r][j], u[j], g.d);
      }
    }
  }
}

struct Norm8Grad {
  Rows8 r;
  int T, d;
  int64_t ldy, ldr, ldx, lde;
  const float *mean, *rstd;
  const float *res;
  float *dx;
  float *sums[3];   // dgamma, dbeta, dres_sum
  float *partial;
  int accumulate;
};

constexpr int kStretch = 256;   // rows that a lane adds up one after the other

// What a wave reads of a row, on its way while the row before is worked on.
template <typename E, int NJ> struct Row8 {
  uint32_t codes[NJ][kN / 4];
  uint32_t byte[NJ];
  Cols<E, kN> dy[NJ];
  Cols<float, kN> res[NJ];
  float mean, rstd;
};

// The rows of a workgroup's slots leave their column sums in registers; at the end the slots' meet in LDS and one row of sums per
// workgroup goes to the workspace: 256 workgroups, one per compute unit, of eight waves with up to 256 registers, seven bytes per column
// of the row at hand and of the next one among them.  4096 x 1024 bf16 with res, dx_e and all sums, 54.7 MB: 13.4 us (the rows beyond the first
// 2048 at 7 TB/s; the rest is launch, the first loads and the slots' joining) and 3.9 for the sums; 32768 rows 81 (5.4 TB/s); 4095 x 4096 40.
// Sixteen waves of half the registers are 1 to 5 % faster there, 3 % slower at 16384 x 1024 and 19 % at 2000 x 8000.
// Registers take kStretch rows' sums, which then go to those that the slot has in LDS (a workgroup of one slot: in the workspace), so that a term
// goes through 256 additions and one for each 256 of its rows: in one chain 2^28 rows of 8 equal columns were off by up to 2e-4 of their sum.
template <typename E, int CODE, int LPR, int W, int NJ, bool NARROW>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(1, 2))) void k_layernorm8_bwd(Norm8Grad g, const E *dy, const E *gamma, E *dx_e) {
  static_assert(LPR == 64 || (W == 1 && NJ == 1), "narrow rows are one unit a lane");
  constexpr int kWaves = 8, kSlots = kWaves / W, kAbreast = kWave / LPR;
  extern __shared__ __align__(16) float lds[];   // kSlots > 1: per slot its sums' ns rows of d floats
  __shared__ float xch[2][kWaves][2];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), slot = wave / W;
  const int ns = g.sums[2] ? 3 : 2;
  Unit u[NJ];
  float dg[NJ][kN], db[NJ][kN], dr[NJ][kN];
  Cols<E, kN> ga[NJ];
  Row8<E, NJ> now, next;
  auto fetch = [&](Row8<E, NJ> &r, int64_t base) {
    // a slot behind the last row does that row again, and nothing comes of it
    const int64_t row = min(base + slot * kAbreast + (LPR < kWave ? lane / LPR : 0), int64_t(g.T) - 1);
    r.mean = g.mean[row];
    r.rstd = g.rstd[row];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      load_codes<NARROW, kN>(r.codes[j], g.r.codes + row * g.r.ldc, u[j], g.d);
      r.byte[j] = g.r.scales[row * g.r.lds + group_of<NARROW, kN>(u[j])];
      load_unit<NARROW>(r.dy[j], dy + row * g.ldy, u[j], g.d);
      if (g.res) load_unit<NARROW>(r.res[j], g.res + row * g.ldr, u[j], g.d);
    }
  };
  // a unit's sums to the slot's, where only this lane has its columns; of lanes whose rows lie side by side the first ones
  auto leave = [&](float *to, float (&t)[kN], Unit at, bool more) {
    if (LPR < kWave && lane >= LPR) return;
    if (more) {
      Cols<float, kN> before;
      load_unit<NARROW>(before, to, at, g.d);
#pragma unroll
      for (int k = 0; k < kN; ++k) t[k] += before.at(k);
    }
    store_unit<NARROW>(to, t, at, g.d);
  };
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    u[j] = unit_at<NARROW, kN>(kN * (kWave * (NJ * (wave % W) + j) + lane % LPR), g.d);
    load_unit<NARROW>(ga[j], gamma, u[j], g.d);
  }
  float *out = g.partial + int64_t(blockIdx.x) * ns * g.d;
  float *mine = kSlots > 1 ? lds + int64_t(slot) * ns * g.d : out;
  const int64_t begin = int64_t(blockIdx.x) * kSlots * kAbreast, step = int64_t(gridDim.x) * kSlots * kAbreast;
  int parity = 0;
  fetch(now, begin);
  for (int64_t base = begin; base < g.T;) {
    const int64_t until = min(int64_t(g.T), base + kStretch * step);
    const bool more = base != begin;   // sums of rows before are in place already
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int k = 0; k < kN; ++k) dg[j][k] = db[j][k] = dr[j][k] = 0.f;
    for (; base < until; base += step, parity ^= 1) {
      if (base + step < g.T) fetch(next, base + step);
      const int64_t row = base + slot * kAbreast + (LPR < kWave ? lane / LPR : 0);
      const bool live = row < g.T;
      float xh[NJ][kN], gy[NJ][kN], s[2] = {0.f, 0.f};
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        decode<CODE>(now.codes[j], now.byte[j], xh[j]);
#pragma unroll
        for (int k = 0; k < kN; ++k) {
          xh[j][k] = (xh[j][k] - now.mean) * now.rstd;
          gy[j][k] = now.dy[j].at(k);
        }
        clear_foreign<NARROW>(xh[j], u[j], g.d);
        clear_foreign<NARROW>(gy[j], u[j], g.d);
#pragma unroll
        for (int k = 0; k < kN; ++k) {
          const float t = gy[j][k] * ga[j].at(k);
          s[0] += t;
          s[1] = fmaf(t, xh[j][k], s[1]);
        }
      }
      row_sums<LPR, W>(s, xch[parity], wave);
      const float m1 = s[0] / float(g.d), m2 = s[1] / float(g.d);
      if (live) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          float o[kN];
#pragma unroll
          for (int k = 0; k < kN; ++k) {
            o[k] = (gy[j][k] * ga[j].at(k) - m1 - xh[j][k] * m2) * now.rstd;
            dg[j][k] = fmaf(gy[j][k], xh[j][k], dg[j][k]);
            db[j][k] += gy[j][k];
            if (g.res) {
              o[k] += now.res[j].at(k);
              dr[j][k] += now.res[j].at(k);
            }
          }
          store_unit<NARROW>(g.dx + row * g.ldx, o, u[j], g.d);
          if (dx_e) store_unit<NARROW>(dx_e + row * g.lde, o, u[j], g.d);
        }
      }
      now = next;
    }
    if constexpr (LPR < kWave) {   // rows side by side in the wave: their sums, left in each of them
#pragma unroll
      for (int k = 0; k < kN; ++k)
#pragma unroll
        for (int o = LPR; o < kWave; o *= 2) {
          dg[0][k] += __shfl_xor(dg[0][k], o, kWave);
          db[0][k] += __shfl_xor(db[0][k], o, kWave);
          dr[0][k] += __shfl_xor(dr[0][k], o, kWave);
        }
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      leave(mine, dg[j], u[j], more);
      leave(mine + g.d, db[j], u[j], more);
      if (ns == 3) leave(mine + 2 * g.d, dr[j], u[j], more);
    }
  }
  if constexpr (kSlots > 1) {
    __syncthreads();
    for (int c = threadIdx.x; c < ns * g.d; c += 512) {
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < kSlots; ++i) t += lds[int64_t(i) * ns * g.d + c];
      out[c] = t;
    }
  }
}

// Sums of the workgroups' rows: 64 columns a workgroup, its 16 waves taking every 16th row, joined in one order.
__global__ __launch_bounds__(1024) void k_layernorm8_sums(Norm8Grad g, int rows) {
  __shared__ float part[16][64];
  const int ns = g.sums[2] ? 3 : 2, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int c = blockIdx.x * 64 + lane, width = ns * g.d;
  float t = 0.f;
  if (c < width) {
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = g.partial[int64_t(min(wave + 16 * i, rows - 1)) * width + c];
#pragma unroll
    for (int i = 0; i < 16; ++i) t += wave + 16 * i < rows ? v[i] : 0.f;
  }
  part[wave][lane] = t;
  __syncthreads();
  if (wave == 0 && c < width) {
    t = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) t += part[w][lane];
    float *out = g.sums[c / g.d] + c % g.d;
    *out = g.accumulate ? *out + t : t;
  }
}

constexpr int kGradGroups = 256;   // workgroups of a backward pass: rows of the workspace

int check_rows8(const char *who, int prec, int code, int T, int d, int most, const void *codes, int64_t ldc, const void *scales, int64_t lds) {
  if (!known_prec(prec)) return fail(HMY_E_INVALID, "%s: unknown precision %d", who, prec);
  if (code != HMY_CODE_INT8 && code != HMY_CODE_E4M3) return fail(HMY_E_INVALID, "%s: unknown code %d", who, code);
  int rc = check_extent(who, T, d, most);
  if (!rc) rc = check_array(who, "codes", codes, 1, T, d, ldc);
  if (!rc) rc = check_array(who, "scales", scales, 1, T, (d + kGroup - 1) / kGroup, lds);
  return rc;
}
Span span(const char *name, const void *p, int64_t bytes, int64_t T, int64_t d, int64_t ld, bool written) { return {name, p, d * bytes, ld * bytes, T, written}; }

}  // namespace

#define DISPATCH_ROWS8(prec, code, ...)                                                                            \
  do {                                                                                                             \
    if ((prec) == HMY_PREC_BF16) {                                                                                 \
      typedef bf16_t E;                                                                                            \
      if ((code) == HMY_CODE_INT8) { constexpr int CODE = HMY_CODE_INT8; __VA_ARGS__ } else { constexpr int CODE = HMY_CODE_E4M3; __VA_ARGS__ } \
    } else {                                                                                                       \
      typedef float E;                                                                                             \
      if ((code) == HMY_CODE_INT8) { constexpr int CODE = HMY_CODE_INT8; __VA_ARGS__ } else { constexpr int CODE = HMY_CODE_E4M3; __VA_ARGS__ } \
    }                                                                                                              \
  } while (0)

static int check_move8(const char *who, const hmy_rows8_desc &g, bool pack) {
  int rc = check_rows8(who, g.prec, g.code, g.T, g.d, kMaxColumns, g.codes, g.ldc, g.scales, g.lds);
  const int e = bytes_of(g.prec);
  if (!rc) rc = check_array(who, "x", g.x, e, g.T, g.d, g.ldx);
  if (rc) return rc;
  const Span spans[] = {span("x", g.x, e, g.T, g.d, g.ldx, !pack), span("codes", g.codes, 1, g.T, g.d, g.ldc, pack),
                        span("scales", g.scales, 1, g.T, (g.d + kGroup - 1) / kGroup, g.lds, pack)};
  return check_apart(who, spans);
}

int launch_pack8(const hmy_rows8_desc &g, stream_t st) {
  const int rc = check_move8("pack8", g, true);
  if (rc) return rc;
  const Shares h = shares_of(g.T, g.d, 16 / bytes_of(g.prec), kGroup);
  const bool once = int64_t(g.T) * g.d * bytes_of(g.prec) >= kStreamed;
  DISPATCH_ROWS8(g.prec, g.code, {
    DISPATCH_SHARES(h.K, g.d, {
      hipLaunchKernelGGL((once ? k_pack8<E, CODE, K, NARROW, true> : k_pack8<E, CODE, K, NARROW, false>), h.grid, dim3(kThreads), 0,
                         (hipStream_t)st, (const E *)g.x, g.ldx, (uint8_t *)g.codes, g.ldc, (uint8_t *)g.scales, g.lds, h.units);
    });
  });
  return check_launch("pack8");
}

int launch_unpack8(const hmy_rows8_desc &g, stream_t st) {
  const int rc = check_move8("unpack8", g, false);
  if (rc) return rc;
  const Shares h = shares_of(g.T, g.d, 16 / bytes_of(g.prec), kGroup);
  const Rows8 r = {(const uint8_t *)g.codes, (const uint8_t *)g.scales, g.ldc, g.lds};
  DISPATCH_ROWS8(g.prec, g.code, {
    DISPATCH_SHARES(h.K, g.d, {
      hipLaunchKernelGGL((k_unpack8<E, CODE, K, NARROW>), h.grid, dim3(kThreads), 0, (hipStream_t)st, r, (E *)g.x, g.ldx, h.units);
    });
  });
  return check_launch("unpack8");
}

int launch_layernorm8_fwd(const hmy_layernorm8_desc &g, stream_t st) {
  const char *who = "layernorm8_fwd";
  int rc = check_rows8(who, g.prec, g.code, g.T, g.d, HMY_MAX_NORM8_COLUMNS, g.codes, g.ldc, g.scales, g.lds);
  const int e = bytes_of(g.prec);
  if (!rc) rc = check_array(who, "y", g.y, e, g.T, g.d, g.ldy);
  if (!rc && g.x) rc = check_array(who, "x", g.x, 4, g.T, g.d, g.ldx);
  if (rc) return rc;
  if (!(g.eps > 0.f) || !std::isfinite(g.eps)) return fail(HMY_E_INVALID, "%s: eps must be positive and finite", who);
  if (misaligned(g.gamma, e) || misaligned(g.beta, e) || misaligned(g.mean, 4) || misaligned(g.rstd, 4))
    return fail(HMY_E_INVALID, "%s: misaligned array", who);
  const Span spans[] = {span("codes", g.codes, 1, g.T, g.d, g.ldc, false), span("scales", g.scales, 1, g.T, (g.d + kGroup - 1) / kGroup, g.lds, false),
                        span("gamma", g.gamma, e, 1, g.d, g.d, false), span("beta", g.beta, e, 1, g.d, g.d, false), span("y", g.y, e, g.T, g.d, g.ldy, true),
                        span("x", g.x, 4, g.T, g.d, g.ldx, true), span("mean", g.mean, 4, 1, g.T, g.T, true), span("rstd", g.rstd, 4, 1, g.T, g.T, true)};
  rc = check_apart(who, spans);
  if (rc) return rc;
  const Norm8 a = {{(const uint8_t *)g.codes, (const uint8_t *)g.scales, g.ldc, g.lds}, g.T, g.d, g.ldy, g.ldx, g.mean, g.rstd, g.eps};
  const hipStream_t s = (hipStream_t)st;
#define NORM8_FWD(LPR, W, NJ, ROWS, NARROW)                                                                                             \
  do {                                                                                                                                  \
    constexpr int kRows = 4 / W * ROWS * (kWave / LPR);                                                                                 \
    const dim3 grid(uint32_t(std::min<int64_t>((int64_t(g.T) + kRows - 1) / kRows, kMaxGrid)));                                          \
    hipLaunchKernelGGL((k_layernorm8_fwd<E, CODE, LPR, W, NJ, ROWS, NARROW>), grid, dim3(256), 0, s, a, (const E *)g.gamma, (const E *)g.beta, \
                       (E *)g.y, g.x);                                                                                                  \
  } while (0)
  DISPATCH_ROWS8(g.prec, g.code, {
    if (g.d < 8) NORM8_FWD(8, 1, 1, 2, true);
    else if (g.d <= 32) NORM8_FWD(8, 1, 1, 2, false);
    else if (g.d <= 64) NORM8_FWD(16, 1, 1, 2, false);
    else if (g.d <= 128) NORM8_FWD(32, 1, 1, 2, false);
    else if (g.d <= 256) NORM8_FWD(64, 1, 1, 2, false);
    else if (g.d <= 512) NORM8_FWD(64, 1, 2, 1, false);
    else if (g.d <= 1024 && g.T >= 8192) NORM8_FWD(64, 1, 4, 2, false);
    else if (g.d <= 1024) NORM8_FWD(64, 1, 4, 1, false);
    else if (g.d <= 1280) NORM8_FWD(64, 1, 5, 1, false);
    else if (g.d <= 1536) NORM8_FWD(64, 1, 6, 1, false);
    else if (g.d <= 1792) NORM8_FWD(64, 1, 7, 1, false);
    else if (g.d <= 2048) NORM8_FWD(64, 1, 8, 1, false);
    else if (g.d <= 3 * 1024) NORM8_FWD(64, 4, 3, 1, false);
    else if (g.d <= 4096) NORM8_FWD(64, 4, 4, 1, false);
    else if (g.d <= 5120) NORM8_FWD(64, 4, 5, 1, false);
    else if (g.d <= 6144) NORM8_FWD(64, 4, 6, 1, false);
    else if (g.d <= 7168) NORM8_FWD(64, 4, 7, 1, false);
    else NORM8_FWD(64, 4, 8, 1, false);
  });
#undef NORM8_FWD
  return check_launch(who);
}

int launch_layernorm8_bwd(const hmy_layernorm8_grad_desc &g, stream_t st) {
  const char *who = "layernorm8_bwd";
  int rc = check_rows8(who, g.prec, g.code, g.T, g.d, HMY_MAX_NORM8_COLUMNS, g.codes, g.ldc, g.scales, g.lds);
  const int e = bytes_of(g.prec);
  if (!rc) rc = check_array(who, "dy", g.dy, e, g.T, g.d, g.ldy);
  if (!rc) rc = check_array(who, "dx", g.dx, 4, g.T, g.d, g.ldx);
  if (!rc && g.res) rc = check_array(who, "res", g.res, 4, g.T, g.d, g.ldr);
  if (!rc && g.dx_e) rc = check_array(who, "dx_e", g.dx_e, e, g.T, g.d, g.lde);
  if (rc) return rc;
  if (g.accumulate != 0 && g.accumulate != 1) return fail(HMY_E_INVALID, "%s: accumulate must be 0 or 1", who);
  if (g.dres_sum && !g.res) return fail(HMY_E_INVALID, "%s: column sums of a residual gradient that is not given", who);
  if (g.workspace_bytes < HMY_NORM8_WORKSPACE_BYTES(g.d) || misaligned(g.workspace, 16))
    return fail(HMY_E_INVALID, "%s: a workspace of %llu bytes, aligned to 16, wanted", who, (unsigned long long)HMY_NORM8_WORKSPACE_BYTES(g.d));
  const void *words[] = {g.mean, g.rstd, g.dgamma, g.dbeta, g.dres_sum};
  for (const void *p : words)
    if (misaligned(p, 4)) return fail(HMY_E_INVALID, "%s: misaligned array", who);
  if (misaligned(g.gamma, e)) return fail(HMY_E_INVALID, "%s: misaligned array", who);
  const bool in_place = g.res == g.dx && g.ldr == g.ldx;
  const Span spans[] = {span("codes", g.codes, 1, g.T, g.d, g.ldc, false), span("scales", g.scales, 1, g.T, (g.d + kGroup - 1) / kGroup, g.lds, false),
                        span("gamma", g.gamma, e, 1, g.d, g.d, false), span("mean", g.mean, 4, 1, g.T, g.T, false), span("rstd", g.rstd, 4, 1, g.T, g.T, false),
                        span("dy", g.dy, e, g.T, g.d, g.ldy, false), span("res", in_place ? nullptr : g.res, 4, g.T, g.d, g.ldr, false),
                        span("dx", g.dx, 4, g.T, g.d, g.ldx, true), span("dx_e", g.dx_e, e, g.T, g.d, g.lde, true), span("dgamma", g.dgamma, 4, 1, g.d, g.d, true),
                        span("dbeta", g.dbeta, 4, 1, g.d, g.d, true), span("dres_sum", g.dres_sum, 4, 1, g.d, g.d, true),
                        span("workspace", g.workspace, 1, 1, int64_t(HMY_NORM8_WORKSPACE_BYTES(g.d)), int64_t(HMY_NORM8_WORKSPACE_BYTES(g.d)), true)};
  rc = check_apart(who, spans);
  if (rc) return rc;
  const Norm8Grad a = {{(const uint8_t *)g.codes, (const uint8_t *)g.scales, g.ldc, g.lds}, g.T, g.d, g.ldy, g.ldr, g.ldx, g.lde, g.mean, g.rstd, g.res, g.dx,
                       {g.dgamma, g.dbeta, g.dres_sum}, (float *)g.workspace, g.accumulate};
  const int W = g.d <= 1024 ? 1 : g.d <= 2048 ? 2 : g.d <= 4096 ? 4 : 8, slots = 8 / W, ns = g.dres_sum ? 3 : 2;
  const int abreast = g.d <= 32 ? 8 : g.d <= 64 ? 4 : g.d <= 128 ? 2 : 1, rows = slots * abreast;
  const int groups = int(std::min<int64_t>((int64_t(g.T) + rows - 1) / rows, kGradGroups));
  const size_t lds = slots > 1 ? size_t(slots) * ns * g.d * 4 : 0;
  const hipStream_t s = (hipStream_t)st;
#define NORM8_BWD(LPR, W, NJ, NARROW) \
  hipLaunchKernelGGL((k_layernorm8_bwd<E, CODE, LPR, W, NJ, NARROW>), dim3(groups), dim3(512), lds, s, a, (const E *)g.dy, (const E *)g.gamma, (E *)g.dx_e)
  DISPATCH_ROWS8(g.prec, g.code, {
    if (g.d < 8) NORM8_BWD(8, 1, 1, true);
    else if (g.d <= 32) NORM8_BWD(8, 1, 1, false);
    else if (g.d <= 64) NORM8_BWD(16, 1, 1, false);
    else if (g.d <= 128) NORM8_BWD(32, 1, 1, false);
    else if (g.d <= 256) NORM8_BWD(64, 1, 1, false);
    else if (g.d <= 512) NORM8_BWD(64, 1, 2, false);
    else if (g.d <= 768) NORM8_BWD(64, 1, 3, false);
    else if (g.d <= 1024) NORM8_BWD(64, 1, 4, false);
    else if (g.d <= 1536) NORM8_BWD(64, 2, 3, false);
    else if (g.d <= 2048) NORM8_BWD(64, 2, 4, false);
    else if (g.d <= 3 * 1024) NORM8_BWD(64, 4, 3, false);
    else if (g.d <= 4096) NORM8_BWD(64, 4, 4, false);
    else if (g.d <= 6144) NORM8_BWD(64, 8, 3, false);
    else NORM8_BWD(64, 8, 4, false);
  });
#undef NORM8_BWD
  hipLaunchKernelGGL(k_layernorm8_sums, dim3((ns * g.d + 63) / 64), dim3(1024), 0, s, a, groups);
  return check_launch(who);
}

}  // namespace hmy
