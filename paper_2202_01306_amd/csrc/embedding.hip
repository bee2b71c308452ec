// Rows of a table by token, and the table's gradient by sorted tokens.
//
// The gradient of a lookup adds up rows that share a token.  Sorted by token (and, for one token, in their own order) those rows are
// neighbours, a sum is a run of the sorted list, and no row of the table is written by two workgroups: no atomics, one order.
// Three steps: the sort (keys only: 8 bytes per token), the sums of runs inside pieces of the list, and the joining of those runs that
// cross from one piece into the next.  Bound by HBM: every row of dx is read once, every row of the table written once.
#include <algorithm>

#include "stream_rows.h"

namespace hmy {

namespace {

// ---- lookup -------------------------------------------------------------------------------------

constexpr int kThreads = 256, kPerThread = 2, kUnits = kThreads * kPerThread;

struct Lookup {
  const int32_t *ids, *positions;
  int T, d, V, P;
  uint32_t per_row;           // units of eight columns in a row
  int64_t ldw, ldp, ldx, total, tiles;
  float scale;
};

template <typename E, typename O>
__global__ __launch_bounds__(kThreads) void k_embed_lookup(Lookup g, const E *table, const E *pos_table, O *x) {
  for (int64_t tile = blockIdx.x; tile < g.tiles; tile += gridDim.x) {
    const int64_t row0 = tile * kUnits / g.per_row;
    const uint32_t first = uint32_t(tile * kUnits - row0 * g.per_row);
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
      const uint32_t at = first + threadIdx.x + i * kThreads, down = at / g.per_row;
      if (tile * kUnits + threadIdx.x + i * kThreads >= g.total) continue;
      const int64_t t = row0 + down;
      const int c = int(at - down * g.per_row) * 8, n = g.d - c;
      const int id = g.ids[t];
      float v[8] = {}, p[8] = {};
      if (uint32_t(id) < uint32_t(g.V)) load_columns(v, table + id * g.ldw + c, n);
      if (g.P) {
        const int place = g.positions ? g.positions[t] : int(t % g.P);
        if (uint32_t(place) < uint32_t(g.P)) load_columns(p, pos_table + place * g.ldp + c, n);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = fmaf(v[k], g.scale, p[k]);
      store_columns(x + t * g.ldx + c, v, n);
    }
  }
}

// ---- sort -----------------------------------------------------------------------------------------
// Stable sorting by eight bits of the key at a time, least ones first.  A wave takes 64 tokens at a time: the lanes that share a digit
// find each other by eight ballots, which gives each its rank among them, and the first of them advances the digit's counter, so that
// counters are a wave's own and need no atomics.  Tokens that name no row have the key V and end up last.

constexpr int kDigits = 256;

__device__ __forceinline__ uint32_t key_of(int32_t id, int V) { return uint32_t(id) < uint32_t(V) ? uint32_t(id) : uint32_t(V); }

// lanes of the wave with the same digit, among those that are active
__device__ __forceinline__ uint64_t lanes_alike(uint32_t digit, bool active) {
  uint64_t m = __ballot(active);
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    const uint64_t set = __ballot(digit >> b & 1);
    m &= digit >> b & 1 ? set : ~set;
  }
  return m;
}
// what the wave's lanes wrote to LDS before is what its lanes read after
__device__ __forceinline__ void wave_sees_lds() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
// sum of x over the lanes before this one
__device__ __forceinline__ uint32_t lanes_before(uint32_t x, int lane) {
  uint32_t s = x;
#pragma unroll
  for (int o = 1; o < kWave; o *= 2) {
    const uint32_t y = __shfl_up(s, o, kWave);
    if (lane >= o) s += y;
  }
  return s - x;
}
// Exclusive sum over the first kDigits threads of a workgroup; all of its threads call it.
__device__ __forceinline__ uint32_t digits_before(uint32_t x, uint32_t *scratch) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  uint32_t s = 0;
  if (threadIdx.x < kDigits) {
    s = lanes_before(x, lane);
    if (lane == kWave - 1) scratch[wave] = s + x;
  }
  __syncthreads();
  if (threadIdx.x < kDigits)
    for (int w = 0; w < wave; ++w) s += scratch[w];
  __syncthreads();
  return s;
}

// All of it in one workgroup's LDS: up to kOneGroup tokens.
constexpr int kOneGroup = 16384, kSortWaves = 16;

__global__ __launch_bounds__(kSortWaves *kWave) void k_sort_tokens(const int32_t *ids, int T, int V, int passes, uint32_t *keys, uint32_t *order) {
  extern __shared__ uint32_t lds[];   // keys[T], and two lists of T tokens in 16 bits
  __shared__ uint16_t at[kSortWaves][kDigits];
  __shared__ uint32_t scratch[kDigits / kWave];
  uint32_t *key = lds;
  uint16_t *from = reinterpret_cast<uint16_t *>(lds + T), *to = from + T;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  for (int i = tid; i < T; i += kSortWaves * kWave) key[i] = key_of(ids[i], V);
  const int per = (T + kSortWaves * kWave - 1) / (kSortWaves * kWave) * kWave, begin = wave * per, end = min(T, begin + per);
  const uint64_t before = (uint64_t(1) << lane) - 1;
  __syncthreads();
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = 8 * pass;
    for (int b = lane; b < kDigits; b += kWave) at[wave][b] = 0;
    wave_sees_lds();
    for (int i0 = begin; i0 < end; i0 += kWave) {
      const bool active = i0 + lane < end;
      const int t = active ? (pass ? from[i0 + lane] : i0 + lane) : 0;
      const uint32_t digit = key[t] >> shift & 255;
      const uint64_t alike = lanes_alike(digit, active);
      if (active && !(alike & before)) at[wave][digit] += uint16_t(__popcll(alike));
      wave_sees_lds();
    }
    __syncthreads();
    uint32_t total = 0;
    if (tid < kDigits)
      for (int w = 0; w < kSortWaves; ++w) total += at[w][tid];
    uint32_t run = digits_before(total, scratch);
    if (tid < kDigits)
      for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t n = at[w][tid];
        at[w][tid] = uint16_t(run);
        run += n;
      }
    __syncthreads();
    for (int i0 = begin; i0 < end; i0 += kWave) {
      const bool active = i0 + lane < end;
      const int t = active ? (pass ? from[i0 + lane] : i0 + lane) : 0;
      const uint32_t k = key[t], digit = k >> shift & 255;
      const uint64_t alike = lanes_alike(digit, active);
      const uint32_t pos = at[wave][digit] + __popcll(alike & before);
      wave_sees_lds();
      if (active && !(alike & before)) at[wave][digit] += uint16_t(__popcll(alike));
      wave_sees_lds();
      if (active) {
        if (pass == passes - 1) {
          keys[pos] = k;
          order[pos] = uint32_t(t);
        } else {
          to[pos] = uint16_t(t);
        }
      }
    }
    __syncthreads();
    uint16_t *s = from;
    from = to;
    to = s;
  }
}

// The same over workgroups, a pass in two launches: counts[tile][digit] of tiles of kTile tokens, then each tile's tokens to their
// places, which are those of the digits before, of the tiles before, and of the waves before.
constexpr int kTile = 2048, kTileWaves = 4, kTilePerWave = kTile / kTileWaves;

__global__ __launch_bounds__(kTileWaves *kWave) void k_sort_count(const int32_t *ids, const uint32_t *keys, int T, int V, int shift, uint32_t *counts) {
  __shared__ uint32_t at[kTileWaves][kDigits];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const uint64_t before = (uint64_t(1) << lane) - 1;
  const int64_t begin = int64_t(blockIdx.x) * kTile + wave * kTilePerWave;
  for (int b = lane; b < kDigits; b += kWave) at[wave][b] = 0;
  wave_sees_lds();
#pragma unroll
  for (int i = 0; i < kTilePerWave; i += kWave) {
    const int64_t p = begin + i + lane;
    const bool active = p < T;
    const uint32_t k = active ? (ids ? key_of(ids[p], V) : keys[p]) : 0, digit = k >> shift & 255;
    const uint64_t alike = lanes_alike(digit, active);
    if (active && !(alike & before)) at[wave][digit] += __popcll(alike);
    wave_sees_lds();
  }
  __syncthreads();
  if (tid < kDigits) {
    uint32_t n = 0;
#pragma unroll
    for (int w = 0; w < kTileWaves; ++w) n += at[w][tid];
    counts[int64_t(blockIdx.x) * kDigits + tid] = n;
  }
}

// `ids`: the first pass, whose keys are made of them and whose order is their own
__global__ __launch_bounds__(kTileWaves *kWave) void k_sort_place(const int32_t *ids, const uint32_t *keys, const uint32_t *order, int T, int V, int shift,
                                                               const uint32_t *counts, int tiles, uint32_t *to_keys, uint32_t *to_order) {
  static_assert(kTileWaves * kWave == kDigits, "a thread per digit");
  __shared__ uint32_t at[kTileWaves][kDigits];
  __shared__ uint32_t scratch[kDigits / kWave];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const uint64_t before = (uint64_t(1) << lane) - 1;
  const int64_t begin = int64_t(blockIdx.x) * kTile + wave * kTilePerWave;
  for (int b = lane; b < kDigits; b += kWave) at[wave][b] = 0;
  wave_sees_lds();
  uint32_t key[kTilePerWave / kWave];
#pragma unroll
  for (int i = 0; i < kTilePerWave / kWave; ++i) {
    const int64_t p = begin + kWave * i + lane;
    const bool active = p < T;
    key[i] = active ? (ids ? key_of(ids[p], V) : keys[p]) : 0;
    const uint32_t digit = key[i] >> shift & 255;
    const uint64_t alike = lanes_alike(digit, active);
    if (active && !(alike & before)) at[wave][digit] += __popcll(alike);
    wave_sees_lds();
  }
  uint32_t total = 0, mine = 0;   // of this thread's digit: in all tiles, in those before
#pragma unroll 8
  for (int i = 0; i < tiles; ++i) {
    const uint32_t n = counts[int64_t(i) * kDigits + tid];
    total += n;
    mine += i < int(blockIdx.x) ? n : 0;
  }
  uint32_t run = digits_before(total, scratch) + mine;
#pragma unroll
  for (int w = 0; w < kTileWaves; ++w) {
    const uint32_t n = at[w][tid];
    at[w][tid] = run;
    run += n;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kTilePerWave / kWave; ++i) {
    const int64_t p = begin + kWave * i + lane;
    const bool active = p < T;
    const uint32_t digit = key[i] >> shift & 255;
    const uint64_t alike = lanes_alike(digit, active);
    const uint32_t pos = at[wave][digit] + __popcll(alike & before);
    wave_sees_lds();
    if (active && !(alike & before)) at[wave][digit] += __popcll(alike);
    wave_sees_lds();
    if (active) {
      to_keys[pos] = key[i];
      to_order[pos] = ids ? uint32_t(p) : order[p];
    }
  }
}

// ---- sums of runs -----------------------------------------------------------------------------------

struct Runs {
  const uint32_t *keys, *order;   // sorted
  int T, d, V;
  int piece, pieces, slabs;       // tokens of a piece; pieces of the list; slabs of columns
  int64_t ldx, ldt;
  float *dtable;
  float *partial;                 // per piece: the sum of the run that it begins within, of the one that it ends within
  float scale;
  int accumulate;
};

constexpr int kAhead = 16, kFillRows = 16;

template <int N> __device__ __forceinline__ void load_some(float (&v)[N], const float *p, int n) {
  if (n >= N) {
    typedef u32x4 u32x4_u __attribute__((aligned(4)));
#pragma unroll
    for (int k = 0; k < N; k += 4) {
      const u32x4 a = *reinterpret_cast<const u32x4_u *>(p + k);
      v[k] = __uint_as_float(a.x); v[k + 1] = __uint_as_float(a.y); v[k + 2] = __uint_as_float(a.z); v[k + 3] = __uint_as_float(a.w);
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = k < n ? p[k] : 0.f;
  }
}
__device__ __forceinline__ void load_some(float (&v)[8], const bf16_t *p, int n) { load_columns(v, p, n); }
template <int N> __device__ __forceinline__ void store_some(float *p, const float (&v)[N], int n) {
  if (n >= N) {
    typedef u32x4 u32x4_u __attribute__((aligned(4)));
#pragma unroll
    for (int k = 0; k < N; k += 4) {
      u32x4 a;
      a.x = __float_as_uint(v[k]); a.y = __float_as_uint(v[k + 1]); a.z = __float_as_uint(v[k + 2]); a.w = __float_as_uint(v[k + 3]);
      *reinterpret_cast<u32x4_u *>(p + k) = a;
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (k < n) p[k] = v[k];
  }
}
template <int N> __device__ __forceinline__ void write_row(const Runs &g, uint32_t key, int c, int n, const float (&sum)[N]) {
  float *out = g.dtable + int64_t(key) * g.ldt + c;
  float o[N];
  if (g.accumulate) {
    load_some(o, out, n);
#pragma unroll
    for (int k = 0; k < N; ++k) o[k] = fmaf(sum[k], g.scale, o[k]);
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) o[k] = sum[k] * g.scale;
  }
  store_some(out, o, n);
}

// A wave sums a piece of the sorted list over a slab of columns; the workgroups behind those write the rows that no token names.
template <typename E>
__global__ __launch_bounds__(256) void k_embed_grad_runs(Runs g, const E *dx, int run_groups) {
  constexpr int N = ElemTraits<E>::VEC, kSlab = kWave * N;   // columns of a lane, of a wave
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if (int(blockIdx.x) >= run_groups) {
    // kFillRows rows: a lane looks for one of them in the list
    const int64_t row0 = (int64_t(int(blockIdx.x) - run_groups) * 4 + wave) * kFillRows;
    const int64_t row = row0 + lane % kFillRows;
    int lo = 0, hi = g.T;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (int64_t(g.keys[mid]) < row) lo = mid + 1;
      else hi = mid;
    }
    const bool named = row >= g.V || (lo < g.T && int64_t(g.keys[lo]) == row);
    uint64_t empty = __ballot(!named && lane < kFillRows);
    const float zero[4] = {0.f, 0.f, 0.f, 0.f};
    while (empty) {
      const int i = __builtin_ctzll(empty);
      empty &= empty - 1;
      float *out = g.dtable + (row0 + i) * g.ldt;
      for (int c = 4 * lane; c < g.d; c += 4 * kWave) store_some(out + c, zero, g.d - c);
    }
    return;
  }
  const int64_t job = int64_t(blockIdx.x) * 4 + wave;
  const int piece = int(job / g.slabs), c = int(job % g.slabs) * kSlab + lane * N, n = g.d - c;
  if (piece >= g.pieces) return;
  const int p0 = piece * g.piece, p1 = min(g.T, p0 + g.piece);
  uint32_t key = g.keys[p0];
  const uint32_t after = p1 < g.T ? g.keys[p1] : 0xffffffffu;
  bool begun = p0 > 0 && g.keys[p0 - 1] == key;   // in a piece before
  float sum[N];
#pragma unroll
  for (int k = 0; k < N; ++k) sum[k] = 0.f;
  auto end_run = [&](bool goes_on) {
    if (key >= uint32_t(g.V)) return;
    if (begun) store_some(g.partial + int64_t(2 * piece) * g.d + c, sum, n);
    else if (goes_on) store_some(g.partial + int64_t(2 * piece + 1) * g.d + c, sum, n);
    else write_row(g, key, c, n, sum);
  };
  for (int p = p0; p < p1; p += kAhead) {
    const int at = min(p + lane % kAhead, g.T - 1);
    const uint32_t keys = g.keys[at], order = g.order[at];
    float v[kAhead][N];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const uint32_t t = __builtin_amdgcn_readlane(order, i), k = __builtin_amdgcn_readlane(keys, i);
      load_some(v[i], dx + int64_t(t) * g.ldx + c, p + i < p1 && k < uint32_t(g.V) ? n : 0);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const uint32_t k = __builtin_amdgcn_readlane(keys, i);
      if (p + i < p1) {
        if (k != key) {
          end_run(false);
          key = k;
          begun = false;
#pragma unroll
          for (int q = 0; q < N; ++q) sum[q] = 0.f;
        }
#pragma unroll
        for (int q = 0; q < N; ++q) sum[q] += v[i][q];
      }
    }
  }
  end_run(key == after);
}

// The runs that cross pieces: the piece that one starts in joins its end with the beginnings of the pieces that follow.  Four waves take
// a fourth of them each, joined in one order.
__global__ __launch_bounds__(256) void k_embed_grad_join(Runs g) {
  constexpr int N = 4;
  __shared__ float part[4][kWave * N];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int64_t slabs = (g.d + kWave * N - 1) / (kWave * N);
  const int piece = int(blockIdx.x / slabs), c = int(blockIdx.x % slabs) * kWave * N + lane * N, n = g.d - c;
  const int p0 = piece * g.piece, p1 = p0 + g.piece;
  if (p1 >= g.T) return;
  const uint32_t key = g.keys[p1];
  if (key >= uint32_t(g.V) || g.keys[p1 - 1] != key || (p0 > 0 && g.keys[p0 - 1] == key)) return;
  int last = piece;   // the last piece that begins within the run
  for (int q = piece + 1;; q += kWave) {
    const bool in = q + lane < g.pieces && g.keys[min(int64_t(q + lane) * g.piece, int64_t(g.T) - 1)] == key;
    const int more = __popcll(__ballot(in));
    last += more;
    if (more < kWave) break;
  }
  const int count = last - piece, per = (count + 3) / 4;   // wave w: pieces piece + 1 + w per ..
  float sum[N] = {0.f, 0.f, 0.f, 0.f};
  if (wave == 0) load_some(sum, g.partial + int64_t(2 * piece + 1) * g.d + c, n);
  const int q1 = min(count, (wave + 1) * per);
  for (int q = wave * per; q < q1; q += 8) {
    float v[8][N];
#pragma unroll
    for (int i = 0; i < 8; ++i) load_some(v[i], g.partial + int64_t(2 * (piece + 1 + min(q + i, q1 - 1))) * g.d + c, q + i < q1 ? n : 0);
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int k = 0; k < N; ++k) sum[k] += v[i][k];
  }
#pragma unroll
  for (int k = 0; k < N; ++k) part[wave][lane * N + k] = sum[k];
  __syncthreads();
  if (wave == 0) {
#pragma unroll
    for (int w = 1; w < 4; ++w)
#pragma unroll
      for (int k = 0; k < N; ++k) sum[k] += part[w][lane * N + k];
    write_row(g, key, c, n, sum);
  }
}

}  // namespace

int launch_embed_lookup(const hmy_embed_lookup_desc &g, stream_t st) {
  const char *who = "embed_lookup";
  if (!known_prec(g.prec) || !known_prec(g.out_prec)) return fail(HMY_E_INVALID, "%s: unknown precision %d or %d", who, g.prec, g.out_prec);
  int rc = check_extent(who, g.T, g.d, kMaxColumns);
  if (rc) return rc;
  if (g.V < 1 || g.P < 0) return fail(HMY_E_INVALID, "%s: V >= 1 and P >= 0 wanted, got V = %d, P = %d", who, g.V, g.P);
  if (!g.pos_table != !g.P) return fail(HMY_E_INVALID, "%s: a table of positions and its number of rows come together", who);
  if (g.positions && !g.P) return fail(HMY_E_INVALID, "%s: positions without a table of them", who);
  if (!std::isfinite(g.scale)) return fail(HMY_E_INVALID, "%s: the scale must be finite", who);
  const int e = bytes_of(g.prec), o = bytes_of(g.out_prec);
  rc = check_array(who, "table", g.table, e, g.V, g.d, g.ldw);
  if (!rc && g.P) rc = check_array(who, "pos_table", g.pos_table, e, g.P, g.d, g.ldp);
  if (!rc) rc = check_array(who, "x", g.x, o, g.T, g.d, g.ldx);
  if (rc) return rc;
  if (misaligned(g.ids, 4) || misaligned(g.positions, 4)) return fail(HMY_E_INVALID, "%s: misaligned array", who);
  const Span spans[] = {{"x", g.x, int64_t(g.d) * o, g.ldx * o, g.T, true},
                        {"table", g.table, int64_t(g.d) * e, g.ldw * e, g.V, false},
                        {"pos_table", g.pos_table, int64_t(g.d) * e, g.ldp * e, g.P, false},
                        {"ids", g.ids, int64_t(g.T) * 4, int64_t(g.T) * 4, 1, false},
                        {"positions", g.positions, int64_t(g.T) * 4, int64_t(g.T) * 4, 1, false}};
  rc = check_apart(who, spans);
  if (rc) return rc;
  Lookup a = {g.ids, g.positions, g.T, g.d, g.V, g.P, uint32_t((g.d + 7) / 8), g.ldw, g.ldp, g.ldx, 0, 0, g.scale};
  a.total = int64_t(g.T) * a.per_row;
  a.tiles = (a.total + kUnits - 1) / kUnits;
  const dim3 grid(uint32_t(std::min<int64_t>(a.tiles, kMaxGrid)));
  DISPATCH_ROWS(g.prec, g.out_prec, {
    hipLaunchKernelGGL((k_embed_lookup<L, E>), grid, dim3(kThreads), 0, (hipStream_t)st, a, (const L *)g.table, (const L *)g.pos_table, (E *)g.x);
  });
  return check_launch(who);
}

int launch_embed_grad(const hmy_embed_grad_desc &g, stream_t st) {
  const char *who = "embed_grad";
  if (!known_prec(g.prec)) return fail(HMY_E_INVALID, "%s: unknown precision %d", who, g.prec);
  int rc = check_extent(who, g.T, g.d, kMaxColumns);
  if (rc) return rc;
  if (g.T > HMY_MAX_SORTED) return fail(HMY_E_INVALID, "%s: T = %d is beyond %d", who, g.T, HMY_MAX_SORTED);
  if (g.V < 1 || g.V == INT32_MAX) return fail(HMY_E_INVALID, "%s: 1 <= V < 2^31 - 1 wanted, got V = %d", who, g.V);
  if (g.accumulate != 0 && g.accumulate != 1) return fail(HMY_E_INVALID, "%s: accumulate must be 0 or 1", who);
  if (!std::isfinite(g.scale)) return fail(HMY_E_INVALID, "%s: the scale must be finite", who);
  const int e = bytes_of(g.prec);
  rc = check_array(who, "dx", g.dx, e, g.T, g.d, g.ldx);
  if (!rc) rc = check_array(who, "dtable", g.dtable, 4, g.V, g.d, g.ldt);
  if (rc) return rc;
  if (misaligned(g.ids, 4)) return fail(HMY_E_INVALID, "%s: misaligned array", who);
  const uint64_t wanted = HMY_EMBED_GRAD_WORKSPACE_BYTES(g.T, g.d);
  if (g.workspace_bytes < wanted || misaligned(g.workspace, 16))
    return fail(HMY_E_INVALID, "%s: a workspace of %llu bytes, aligned to 16, wanted", who, (unsigned long long)wanted);
  const Span spans[] = {{"dtable", g.dtable, int64_t(g.d) * 4, g.ldt * 4, g.V, true},
                        {"dx", g.dx, int64_t(g.d) * e, g.ldx * e, g.T, false},
                        {"ids", g.ids, int64_t(g.T) * 4, int64_t(g.T) * 4, 1, false},
                        {"workspace", g.workspace, int64_t(wanted), int64_t(wanted), 1, true}};
  rc = check_apart(who, spans);
  if (rc) return rc;
  const hipStream_t s = (hipStream_t)st;
  const int T = g.T;
  Runs a = {nullptr, nullptr, T, g.d, g.V, T <= kOneGroup ? 16 : 64, 0, 0, g.ldx, g.ldt, g.dtable, nullptr, g.scale, g.accumulate};
  a.pieces = (T + a.piece - 1) / a.piece;
  a.partial = (float *)g.workspace + (int64_t(wanted) / 4 - 2 * int64_t(g.d) * a.pieces) / 4 * 4;   // at the workspace's end
  const int slab = kWave * (g.prec == HMY_PREC_BF16 ? 8 : 4);
  a.slabs = (g.d + slab - 1) / slab;
  const int64_t run_groups = (int64_t(a.pieces) * a.slabs + 3) / 4, fill_groups = g.accumulate ? 0 : (int64_t(g.V) + 4 * kFillRows - 1) / (4 * kFillRows);
  const int64_t join_groups = int64_t(a.pieces) * ((g.d + 255) / 256);
  constexpr int64_t kMostGroups = (1 << 24) - 1;   // of 256 threads: a launch has fewer than 2^32
  if (run_groups + fill_groups > kMostGroups || join_groups > kMostGroups) return fail(HMY_E_INVALID, "%s: T, d and V are too large together", who);
  const int64_t Ta = (int64_t(T) + 3) / 4 * 4;
  uint32_t *base = (uint32_t *)g.workspace;
  uint32_t *keys[2] = {base, base + 2 * Ta}, *order[2] = {base + Ta, base + 3 * Ta}, *counts = base + 4 * Ta;
  int passes = 1;
  while (passes < 4 && (uint64_t(g.V) >> (8 * passes))) ++passes;
  int sorted = 0;
  if (T <= kOneGroup) {
    hipLaunchKernelGGL(k_sort_tokens, dim3(1), dim3(kSortWaves * kWave), size_t(T) * 8, s, g.ids, T, g.V, passes, keys[0], order[0]);
  } else {
    const int tiles = (T + kTile - 1) / kTile;
    for (int pass = 0; pass < passes; ++pass) {
      const int32_t *ids = pass ? nullptr : g.ids;
      const int to = pass ? 1 - sorted : 0;
      hipLaunchKernelGGL(k_sort_count, dim3(tiles), dim3(kTileWaves * kWave), 0, s, ids, keys[sorted], T, g.V, 8 * pass, counts);
      hipLaunchKernelGGL(k_sort_place, dim3(tiles), dim3(kTileWaves * kWave), 0, s, ids, keys[sorted], order[sorted], T, g.V, 8 * pass, counts, tiles,
                         keys[to], order[to]);
      sorted = to;
    }
  }
  a.keys = keys[sorted];
  a.order = order[sorted];
  const dim3 grid{uint32_t(run_groups + fill_groups)};
  if (g.prec == HMY_PREC_BF16) hipLaunchKernelGGL(k_embed_grad_runs<bf16_t>, grid, dim3(256), 0, s, a, (const bf16_t *)g.dx, int(run_groups));
  else hipLaunchKernelGGL(k_embed_grad_runs<float>, grid, dim3(256), 0, s, a, (const float *)g.dx, int(run_groups));
  if (a.pieces > 1) hipLaunchKernelGGL(k_embed_grad_join, dim3(uint32_t(join_groups)), dim3(256), 0, s, a);
  return check_launch(who);
}

}  // namespace hmy
