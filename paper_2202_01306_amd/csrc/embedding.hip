// Rows of a table by token, and the table's gradient by sorted tokens.
//
// The gradient of a lookup adds up rows that share a token.  Sorted by token (and, for one token, in their own order) those rows are
// neighbours, a sum is a run of the sorted list, and no row of the table is written by two workgroups: no atomics, one order.
// Three steps: the order (keys only: 8 bytes per token), the sums of runs inside pieces of the list, and the joining of those runs that
// go through whole pieces.  Bound by HBM where there are many tokens: every row of dx is read once, every row of the table written once.
// 131072 tokens of 1024 fp32 columns, 30522 rows, 662 MB: 164 us a call; one by one, in a trace, which adds some 0.6 us to a kernel, 24 for the
// order (two passes, four launches), 134 for the sums (4.9 TB/s) and 10 for the joining; 4096 tokens, 50257 rows of which most are empty, 222 MB:
// 5, 42 (5.3 TB/s) and 4.7.  Far from HBM, by the order's launches and by lanes without columns: 131072 x 24 41 us (3 at a copy's rate), x 128
// 45 (17), x 256 63 (35); and by the joining of a few very long runs on a workgroup each: 131072 x 1024 in 2 rows 142 (112), 2^24 x 4 in one row
// 18.9 ms (0.07).
#include <algorithm>

#include "stream_rows.h"

namespace hmy {

namespace {

// ---- lookup -------------------------------------------------------------------------------------

struct Lookup {
  const int32_t *ids, *positions;
  int V, P;
  int64_t ldw, ldp, ldx;
  float scale;
};

// A token's row is found through its id, so that a lane waits twice for memory before it stores: all of its ids are on their way together,
// and then all of its rows.  Bound by HBM, with what the eight L2s each fetch of popular rows: 32768 tokens of 1024 columns, bf16 to fp32
// with positions, 134 MB written and 42 read (23 of them what the call cannot do without): 43 us (4.1 TB/s; from a table of 512 rows,
// which the L2s hold, 29).  Workgroups that stay and fetch their next rows ahead take 47 to 49.
template <typename E, typename O, int K, bool NARROW>
__global__ __launch_bounds__(kThreads) void k_embed_lookup(Lookup g, const E *table, const E *pos_table, O *x, Units units) {
  constexpr int N = 16 / sizeof(O), kPerThread = per_thread(K);
  for (int64_t tile = blockIdx.x; tile < units.tiles; tile += gridDim.x) {
    const Places<kPerThread> at = places_of<K, NARROW, N>(units, tile);
    int id[kPerThread], place[kPerThread];
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
      if (K && i % (K ? K : 1)) {   // the same row
        id[i] = id[i - 1];
        place[i] = place[i - 1];
        continue;
      }
      id[i] = g.ids[at.row[i]];
      place[i] = -1;
      if (g.positions) place[i] = g.positions[at.row[i]];
      else if (g.P) place[i] = int(uint32_t(at.row[i]) % uint32_t(g.P));
    }
    if constexpr (K > 0) {
#pragma unroll
      for (int i = 0; i < kPerThread; ++i) {
        id[i] = __builtin_amdgcn_readfirstlane(id[i]);
        place[i] = __builtin_amdgcn_readfirstlane(place[i]);
      }
    }
    Cols<E, N> v[kPerThread], p[kPerThread];
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {   // what names no row reads the first one and drops it
      load_unit<NARROW>(v[i], table + (uint32_t(id[i]) < uint32_t(g.V) ? id[i] : 0) * g.ldw, at.u[i], units.d);
      if (g.P) load_unit<NARROW>(p[i], pos_table + (uint32_t(place[i]) < uint32_t(g.P) ? place[i] : 0) * g.ldp, at.u[i], units.d);
    }
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
      const bool named = uint32_t(id[i]) < uint32_t(g.V), placed = uint32_t(place[i]) < uint32_t(g.P);
      float o[N];
#pragma unroll
      for (int k = 0; k < N; ++k) o[k] = fmaf(named ? v[i].at(k) : 0.f, g.scale, placed ? p[i].at(k) : 0.f);
      store_unit<NARROW>(x + at.row[i] * g.ldx, o, at.u[i], units.d);
    }
  }
}

// ---- sort -----------------------------------------------------------------------------------------
// Tokens that name no row have the key V and end up last.

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

// Up to kMostRanked tokens: a token's place is the number of tokens before it in the order, counted by comparing it with all of them.  A
// workgroup places kRankTokens tokens against a copy of all keys in LDS; each sixteen lanes of its waves compare them with a 64th of the
// keys, four at a time: for 4096 tokens a comparison and an addition for each of 64 keys a lane.  4096 tokens: 5.8 us in one launch; 16384
// take 34, the radix sort's four launches 21.
constexpr int kMostRanked = 8192, kRankThreads = 1024, kRankTokens = 16, kRankParts = kRankThreads / kRankTokens;

__global__ __launch_bounds__(kRankThreads) void k_rank_tokens(const int32_t *ids, int T, int V, uint32_t *keys, uint32_t *order) {
  extern __shared__ __align__(16) uint32_t all[];   // keys, up to the next multiple of 4 kRankParts
  __shared__ uint32_t counts[kRankParts][kRankTokens + 1];
  const int tid = threadIdx.x, token = tid % kRankTokens, part = tid / kRankTokens;
  const int t0 = blockIdx.x * kRankTokens, rounds = (T + 4 * kRankParts - 1) / (4 * kRankParts);
  for (int i = tid; i < rounds * 4 * kRankParts; i += kRankThreads) all[i] = i < T ? key_of(ids[i], V) : 0xffffffffu;
  __syncthreads();
  const uint32_t key = all[min(t0 + token, T - 1)];
  uint32_t n = 0;
  const uint4 *p = reinterpret_cast<const uint4 *>(all) + part;
  auto compare = [&](int round, uint32_t below) {
    const uint4 k = p[round * kRankParts];
    n += (k.x < below) + (k.y < below) + (k.z < below) + (k.w < below);
  };
  // equal keys keep their order: those of tokens before these count; among these themselves below
  const int own = t0 / (4 * kRankParts), at = 4 * (own * kRankParts + part);
#pragma unroll 4
  for (int i = 0; i < own; ++i) compare(i, key + 1);
  compare(own, at < t0 ? key + 1 : at < t0 + kRankTokens ? 0 : key);
#pragma unroll 4
  for (int i = own + 1; i < rounds; ++i) compare(i, key);
  counts[part][token] = n;
  __syncthreads();
  if (tid < kRankTokens && t0 + tid < T) {
    n = 0;
#pragma unroll
    for (int p = 0; p < kRankParts; ++p) n += counts[p][tid];
#pragma unroll
    for (int i = 0; i < kRankTokens; ++i) n += all[min(t0 + i, rounds * 4 * kRankParts - 1)] < key + (i < tid ? 1u : 0u);
    keys[n] = key;
    order[n] = uint32_t(t0 + tid);
  }
}

// More tokens: stable sorting by eight bits of the key at a time, least ones first, a pass in two launches: counts[tile][digit] of tiles of
// kTile tokens, then each tile's tokens to their places, which are behind those of the digits before, of the tiles before, and of the waves
// before.  A wave takes 64 tokens at a time: the lanes that share a digit find each other by eight ballots, which gives each its rank among
// them, and the first of them advances the digit's counter, so that counters are a wave's own and need no atomics.  Bound by latency: a
// pass of 131072 tokens takes 4 and 8 us with eight waves a tile (4 and 10 with four).
constexpr int kTile = 1024, kTileWaves = 8, kSteps = kTile / kTileWaves / kWave;
constexpr int kTilesRead = 256;   // tiles whose counts a tile adds up by itself; of more, a launch in between has added them up

struct Sort {
  const int32_t *ids;             // the first pass, whose keys are made of them and whose order is their own; later ones: NULL
  const uint32_t *keys, *order;
  int T, V, shift, tiles;
  uint32_t *counts;               // [tiles + 1][kDigits]
};

__device__ __forceinline__ void load_keys(const Sort &g, uint32_t (&key)[kSteps], int64_t begin) {
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int64_t p = min(begin + kWave * i, int64_t(g.T) - 1);
    key[i] = g.ids ? key_of(g.ids[p], g.V) : g.keys[p];
  }
}
// counts the digits of a wave's keys
__device__ __forceinline__ void count_digits(const Sort &g, const uint32_t (&key)[kSteps], int64_t begin, uint32_t *at, uint64_t before, int lane) {
  for (int b = lane; b < kDigits; b += kWave) at[b] = 0;
  wave_sees_lds();
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const bool active = begin + kWave * i < g.T;
    const uint32_t digit = key[i] >> g.shift & 255;
    const uint64_t alike = lanes_alike(digit, active);
    if (active && !(alike & before)) at[digit] += __popcll(alike);
    wave_sees_lds();
  }
}

__global__ __launch_bounds__(kTileWaves *kWave) void k_sort_count(Sort g) {
  __shared__ uint32_t at[kTileWaves][kDigits];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int64_t begin = int64_t(blockIdx.x) * kTile + wave * (kSteps * kWave) + lane;
  uint32_t key[kSteps];
  load_keys(g, key, begin);
  count_digits(g, key, begin, at[wave], (uint64_t(1) << lane) - 1, lane);
  __syncthreads();
  if (tid < kDigits) {
    uint32_t n = 0;
#pragma unroll
    for (int w = 0; w < kTileWaves; ++w) n += at[w][tid];
    g.counts[int64_t(blockIdx.x) * kDigits + tid] = n;
  }
}

// Many tiles: counts become those of the tiles before, with the totals behind the last.  64 digits a workgroup, whose waves take a
// sixteenth of the tiles each.
__global__ __launch_bounds__(1024) void k_sort_scan(uint32_t *counts, int tiles) {
  __shared__ uint32_t part[16][kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, per = (tiles + 15) / 16;
  const int t0 = min(tiles, wave * per), t1 = min(tiles, t0 + per);
  uint32_t *p = counts + blockIdx.x * kWave + lane;
  uint32_t n = 0;
#pragma unroll 8
  for (int t = t0; t < t1; ++t) n += p[int64_t(t) * kDigits];
  part[wave][lane] = n;
  __syncthreads();
  uint32_t run = 0, total = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    run += w < wave ? part[w][lane] : 0;
    total += part[w][lane];
  }
#pragma unroll 8
  for (int t = t0; t < t1; ++t) {
    const uint32_t m = p[int64_t(t) * kDigits];
    p[int64_t(t) * kDigits] = run;
    run += m;
  }
  if (wave == 0) p[int64_t(tiles) * kDigits] = total;
}

__global__ __launch_bounds__(kTileWaves *kWave) void k_sort_place(Sort g, uint32_t *to_keys, uint32_t *to_order) {
  static_assert(kTileWaves * kWave >= kDigits, "a thread per digit");
  __shared__ uint32_t at[kTileWaves][kDigits];
  __shared__ uint4 sums[2][kTileWaves][kWave];   // per wave and digit: counts of its tiles, of those before this one
  __shared__ uint32_t scratch[kDigits / kWave];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, tile = blockIdx.x;
  const uint64_t before = (uint64_t(1) << lane) - 1;
  const int64_t begin = int64_t(tile) * kTile + wave * (kSteps * kWave) + lane;
  uint32_t key[kSteps], order[kSteps];
  load_keys(g, key, begin);
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int64_t p = min(begin + kWave * i, int64_t(g.T) - 1);
    order[i] = g.ids ? uint32_t(p) : g.order[p];
  }
  uint32_t total = 0, mine = 0;   // of this thread's digit: in all tiles, in those before
  if (g.tiles <= kTilesRead) {
    // the waves take turns at the tiles, four digits a lane
    uint4 all = make_uint4(0, 0, 0, 0), some = all;
    const uint4 *p = reinterpret_cast<const uint4 *>(g.counts) + lane;
#pragma unroll 16
    for (int t = wave; t < g.tiles; t += kTileWaves) {
      const uint4 n = p[int64_t(t) * (kDigits / 4)];
      all.x += n.x; all.y += n.y; all.z += n.z; all.w += n.w;
      if (t < tile) { some.x += n.x; some.y += n.y; some.z += n.z; some.w += n.w; }
    }
    sums[0][wave][lane] = all;
    sums[1][wave][lane] = some;
  } else if (tid < kDigits) {
    total = g.counts[int64_t(g.tiles) * kDigits + tid];
    mine = g.counts[int64_t(tile) * kDigits + tid];
  }
  count_digits(g, key, begin, at[wave], before, lane);
  __syncthreads();
  if (g.tiles <= kTilesRead && tid < kDigits) {
#pragma unroll
    for (int w = 0; w < kTileWaves; ++w) {
      total += reinterpret_cast<const uint32_t *>(sums[0][w])[tid];
      mine += reinterpret_cast<const uint32_t *>(sums[1][w])[tid];
    }
  }
  uint32_t run = digits_before(total, scratch) + mine;
  if (tid < kDigits)
#pragma unroll
    for (int w = 0; w < kTileWaves; ++w) {
      const uint32_t n = at[w][tid];
      at[w][tid] = run;
      run += n;
    }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const bool active = begin + kWave * i < g.T;
    const uint32_t digit = key[i] >> g.shift & 255;
    const uint64_t alike = lanes_alike(digit, active);
    const uint32_t pos = at[wave][digit] + __popcll(alike & before);
    wave_sees_lds();
    if (active && !(alike & before)) at[wave][digit] += __popcll(alike);
    wave_sees_lds();
    if (active) {
      to_keys[pos] = key[i];
      to_order[pos] = order[i];
    }
  }
}

// ---- sums of runs -----------------------------------------------------------------------------------

struct Runs {
  const uint32_t *keys, *order;   // sorted
  const int32_t *ids;             // as they are
  int T, d, V;
  int piece, pieces, slabs;       // tokens of a piece; pieces of the list; slabs of columns
  int64_t ldx, ldt;
  float *dtable;
  float *partial;                 // per piece: the sum of a run's tokens in a piece that it goes through, of those in the piece that it starts in
  float scale;
  int fill_rows;                  // rows that a wave looks after
};

constexpr int kAhead = 16;        // rows on their way at a time
constexpr int kPieceRanked = 16, kPieceSorted = 32;
// A wave that may have to write rows with zeros looks after up to kMostFilled rows and kFillColumns columns of them, some 16 KB.
constexpr int kMostFilled = 64, kFillColumns = 1024;

// A wave's columns of a row: a slab of kWave * N of them, a unit a lane.
template <typename E, bool NARROW> struct Slab {
  static constexpr int N = ElemTraits<E>::VEC;
  typedef Cols<E, N> Raw;
  Unit u;
  int d;
  __device__ __forceinline__ Slab(int slab, int lane, int d_) : u(unit_at<NARROW, N>((slab * kWave + lane) * N, d_)), d(d_) {}
  template <bool ONCE = false> __device__ __forceinline__ void load(Raw &v, const E *row) const { load_unit<NARROW, ONCE>(v, row, u, d); }
  __device__ __forceinline__ void load(float (&v)[N], const float *row) const {
    Cols<float, N> c;
    load_unit<NARROW>(c, row, u, d);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = c.at(k);
  }
  __device__ __forceinline__ void store(float *row, const float (&v)[N]) const { store_unit<NARROW>(row, v, u, d); }
};

// sum to row `key`, whose present content is `old` if that is added to
template <bool ADD, int N, typename S> __device__ __forceinline__ void write_row(const Runs &g, const S &s, uint32_t key, const float (&sum)[N], const float (&old)[N]) {
  float o[N];
#pragma unroll
  for (int k = 0; k < N; ++k) o[k] = ADD ? fmaf(sum[k], g.scale, old[k]) : sum[k] * g.scale;
  s.store(g.dtable + int64_t(key) * g.ldt, o);
}

// Zeros to kFillColumns columns from c0 on of the rows row0 + i for which bit i is set.  They are streaming stores, which leave the caches to
// the rows of dx: with ordinary ones 16384 tokens of 1024 columns, 30522 rows or more, take 73 us instead of 66, 1000 of them 41 instead of 42.
__device__ __forceinline__ void zero_rows(const Runs &g, int64_t row0, uint64_t empty, int c0, int lane) {
  const int c1 = min(g.d, c0 + kFillColumns), whole = c0 + (c1 - c0) / 4 * 4;
  while (empty) {
    const int i = __builtin_ctzll(empty);
    empty &= empty - 1;
    float *out = g.dtable + (row0 + i) * g.ldt;
    const u32x4 zero = {0, 0, 0, 0};
    for (int c = c0 + 4 * lane; c < whole; c += 4 * kWave) __builtin_nontemporal_store(zero, reinterpret_cast<u32x4_by4 *>(out + c));
    if (whole + lane < c1) out[whole + lane] = 0.f;
  }
}

// The number of keys below `key`, by the whole wave: 64 places at a time.
__device__ __forceinline__ int keys_below(const Runs &g, int64_t key, int lane) {
  int lo = 0, n = g.T;   // it is in lo .. lo + n
  while (n > 0) {
    const int step = (n + kWave) / (kWave + 1);   // probes at lo + step - 1, lo + 2 step - 1, ..
    const int64_t at = int64_t(lo) + int64_t(lane + 1) * step - 1;
    const int m = __popcll(__ballot(at < int64_t(lo) + n && int64_t(g.keys[min(at, int64_t(g.T) - 1)]) < key));
    const int end = lo + n;
    lo += m * step;
    n = min(m < kWave ? step - 1 : step, end - lo);
  }
  return lo;
}

// A wave sums a piece of the sorted list over a slab of columns.  A run that ends in the piece behind the one that it starts in, or behind
// one that it goes through, is taken along to its end; so only runs that go through a whole piece leave parts of their sum to be joined.
// Pieces of 16 tokens up to kMostRanked, for the waves' number, of 32 beyond (16384 x 1024 fp32: 78 us with 16, 79 with 32, 81 with 64; 131072
// x 1024: 190, 184, 184; all before any loads were streaming ones).  kAhead rows are on their way before the first is added (8 instead of 16: 90
// instead of 81 us at 16384 x 1024).
// What the wave has to know of the list it reads in one go, a place a lane: the piece, the one behind, and a key at either end.
// ONCE, from kStreamed bytes on: the caches are left to the table and to sums of parts of runs.  Calls with three sets of inputs in turn: fp32 rows of
// 1024 columns, 131072 tokens 167 us instead of 178, 65536 105 and 115, 32768 74 and 79, 20480 63 and 65, but 16384 57 and 55; bf16 x 2048, 20480
// tokens 84 and 90; it does not pay at fp32 x 5000, 16384 tokens: 226 and 224.  With dx written by the kernel just before: 131072 tokens 158 us
// instead of 198, 65536 96 and 102, 16384 x 5000 210 and 227, but 32768 69 and 65, 20480 58 and 56 (16384 54 and 54).
// ADD: what is in the table is on its way for every token, though only the last one of a run needs it; bf16 rows, eight columns a lane, take 218 to
// 223 registers for it, two waves per SIMD, fp32 rows 150 to 155: 4096 x 1024 18 us for either, 20480 x 2048 75 (fp32) and 66 (bf16).
template <typename E, int PIECE, bool NARROW, bool ADD, bool ONCE>
__device__ __forceinline__ void sum_piece(const Runs &g, const E *dx, int piece, int slab, int lane) {
  static_assert(2 * PIECE <= kWave, "a place a lane");
  constexpr int N = ElemTraits<E>::VEC;
  constexpr uint32_t kNone = 0xffffffffu, kBefore = 0xfffffffeu;   // no token's key: behind the list, before it
  const Slab<E, NARROW> s(slab, lane, g.d);
  const int p0 = piece * PIECE, at = p0 + lane, len = min(PIECE, g.T - p0);
  uint32_t keys = g.keys[min(at, g.T - 1)], next = g.keys[min(p0 + 2 * PIECE, g.T - 1)], before = g.keys[max(p0 - 1, 0)];
  const uint32_t order = g.order[min(at, g.T - 1)];
  if (at >= g.T) keys = kNone;
  if (p0 + 2 * PIECE >= g.T) next = kNone;
  if (p0 == 0) before = kBefore;
  const uint32_t key = __builtin_amdgcn_readlane(keys, 0), last = __builtin_amdgcn_readlane(keys, len - 1), after = __builtin_amdgcn_readlane(keys, PIECE);
  if (key >= uint32_t(g.V)) return;
  int begin = 0, end = len;
  bool through = false;                               // all of the piece, and what is behind, is a run that has begun before
  if (before == key) {
    through = after == key;
    if (!through) {                                   // the run ends here: its end was taken along
      if (last == key) return;
      begin = __popcll(__ballot(keys == key && lane < PIECE));
      if (uint32_t(__builtin_amdgcn_readlane(keys, begin)) >= uint32_t(g.V)) return;
    }
  }
  bool goes_on = false;                               // the last run goes through all of the next piece
  if (after == last && last < uint32_t(g.V)) {
    if (next == last) goes_on = true;
    else end = PIECE + __popcll(__ballot(keys == last && lane >= PIECE && lane < 2 * PIECE));
  }
  const uint32_t first = __builtin_amdgcn_readlane(order, begin);
  float sum[N];
#pragma unroll
  for (int k = 0; k < N; ++k) sum[k] = 0.f;
  for (int p = begin; p < end; p += kAhead) {
    const int from = p + lane % kAhead;
    uint32_t k16 = __shfl(keys, from, kWave), o16 = __shfl(order, from, kWave);
    if (from >= end || k16 >= uint32_t(g.V)) {        // read in place of nothing, and not added
      k16 = kNone;
      o16 = first;
    }
    typename Slab<E, NARROW>::Raw v[kAhead];
    float old[ADD ? kAhead : 1][N];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) s.template load<ONCE>(v[i], dx + int64_t(__builtin_amdgcn_readlane(o16, i)) * g.ldx);
    if constexpr (ADD) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) s.load(old[i], g.dtable + int64_t(min(uint32_t(__builtin_amdgcn_readlane(k16, i)), uint32_t(g.V - 1))) * g.ldt);
    }
    const uint32_t behind = p + kAhead < end ? __builtin_amdgcn_readlane(keys, p + kAhead) : kBefore;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const uint32_t k = __builtin_amdgcn_readlane(k16, i), following = i + 1 < kAhead ? __builtin_amdgcn_readlane(k16, (i + 1) % kAhead) : behind;
      if (k != kNone) {
#pragma unroll
        for (int q = 0; q < N; ++q) sum[q] += v[i].at(q);
        if (following != k) {
          const bool at_end = p + i + 1 >= end;
          if (through && at_end) s.store(g.partial + int64_t(2 * piece) * g.d, sum);
          else if (goes_on && at_end) s.store(g.partial + int64_t(2 * piece + 1) * g.d, sum);
          else write_row<ADD>(g, s, k, sum, old[ADD ? i : 0]);
#pragma unroll
          for (int q = 0; q < N; ++q) sum[q] = 0.f;
        }
      }
    }
  }
}

// The workgroups behind those of the sums write the rows that no token names.
template <typename E, bool NARROW, bool ADD, bool ONCE>
__global__ __launch_bounds__(256) void k_embed_grad_runs(Runs g, const E *dx, int run_groups) {
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if (int(blockIdx.x) >= run_groups) {
    const int job = int(blockIdx.x) - run_groups, slabs = (g.d + kFillColumns - 1) / kFillColumns;
    const int64_t row0 = (int64_t(job / slabs) * 4 + wave) * g.fill_rows, row = row0 + lane;
    int lo = keys_below(g, row0, lane), hi = g.T;
    // a lane looks for one of the rows behind that
    if (lane >= g.fill_rows) hi = lo;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (int64_t(g.keys[mid]) < row) lo = mid + 1;
      else hi = mid;
    }
    const bool named = row >= g.V || (lo < g.T && int64_t(g.keys[lo]) == row);
    zero_rows(g, row0, __ballot(!named && lane < g.fill_rows), job % slabs * kFillColumns, lane);
    return;
  }
  const int64_t job = int64_t(blockIdx.x) * 4 + wave;
  const int piece = int(job / g.slabs), slab = int(job % g.slabs);
  if (piece >= g.pieces) return;
  if (g.piece == kPieceRanked) sum_piece<E, kPieceRanked, NARROW, ADD, ONCE>(g, dx, piece, slab, lane);
  else sum_piece<E, kPieceSorted, NARROW, ADD, ONCE>(g, dx, piece, slab, lane);
}

// The runs that go through whole pieces: the sum of the piece that one starts in, and of those that follow.  A workgroup looks at
// kJoinPieces pieces (1841 tokens of 203 rows, twice: 28 us with 4 pieces, 30 with 16; 131072 tokens of 30522, without streaming loads:
// 179 and 178).  Runs of up to kShortRun parts are a wave's each; of a longer one each of the four waves takes a fourth of the parts, joined
// in one order (eight or sixteen waves are slower: most runs are short).  Bound by latency: keys, their count, the parts, the row.
// A wave adds up kStretch parts one after the other, then as many of these sums, then those: a term goes through 63 additions in its piece and
// 165 here at most, where one chain over a run of 2^24 tokens has 131072 (equal terms of 0.1: off by 1.0e-3 of the sum, 9e-7 this way).
constexpr int kJoinPieces = 4, kShortRun = 8, kStretch = 64;

// parts q0 .. q1 - 1 of the run that starts in `piece`, added to sum
template <bool NARROW, int DEEP> __device__ __forceinline__ void add_parts(const Runs &g, const Slab<float, NARROW> &s, int piece, int q0, int q1, float (&sum)[4]) {
  for (int q = q0; q < q1; q += DEEP) {
    float v[DEEP][4];
#pragma unroll
    for (int i = 0; i < DEEP; ++i) s.load(v[i], g.partial + int64_t(2 * (piece + 1 + min(q + i, q1 - 1))) * g.d);
#pragma unroll
    for (int i = 0; i < DEEP; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) sum[k] += q + i < q1 ? v[i][k] : 0.f;
  }
}
// pieces that the run of `key` goes through behind the one that it starts in: all but the end of the last one
__device__ __forceinline__ int parts_of(const Runs &g, int piece, uint32_t key, int lane) {
  int parts = 0;
  for (int q = piece + 1;; q += kWave) {
    const int64_t next = int64_t(q + lane + 1) * g.piece;
    const int more = __popcll(__ballot(next < g.T && g.keys[min(next, int64_t(g.T) - 1)] == key));
    parts += more;
    if (more < kWave) return parts;
  }
}
template <bool NARROW, bool ADD> __device__ __forceinline__ void join_runs(const Runs &g, uint64_t shorts, uint64_t longs, uint32_t keys, int piece0, int slab, int lane, int wave, float (&part)[4][kWave * 4]) {
  const Slab<float, NARROW> s(slab, lane, g.d);
  float sum[4], old[4];
  for (int turn = 0; shorts; ++turn, shorts &= shorts - 1) {
    if (turn % 4 != wave) continue;
    const int piece = piece0 + __builtin_ctzll(shorts);
    const uint32_t key = __builtin_amdgcn_readlane(keys, __builtin_ctzll(shorts));
    s.load(sum, g.partial + int64_t(2 * piece + 1) * g.d);
    if (ADD) s.load(old, g.dtable + int64_t(key) * g.ldt);
    add_parts<NARROW, kShortRun>(g, s, piece, 0, parts_of(g, piece, key, lane), sum);
    write_row<ADD>(g, s, key, sum, old);
  }
  for (; longs; longs &= longs - 1) {
    const int piece = piece0 + __builtin_ctzll(longs);
    const uint32_t key = __builtin_amdgcn_readlane(keys, __builtin_ctzll(longs));
    const int parts = parts_of(g, piece, key, lane), per = (parts + 3) / 4;
#pragma unroll
    for (int k = 0; k < 4; ++k) sum[k] = 0.f;
    if (wave == 0) s.load(sum, g.partial + int64_t(2 * piece + 1) * g.d);
    if (ADD && wave == 0) s.load(old, g.dtable + int64_t(key) * g.ldt);
    float some[4] = {0.f, 0.f, 0.f, 0.f}, all[4] = {0.f, 0.f, 0.f, 0.f};
    const int q1 = min(parts, (wave + 1) * per);
    for (int q = wave * per, turn = 1; q < q1; q += kStretch, ++turn) {
      add_parts<NARROW, 16>(g, s, piece, q, min(q1, q + kStretch), sum);
      if (q + kStretch >= q1) break;
      const bool far = turn % kStretch == 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        some[k] += sum[k];
        sum[k] = 0.f;
        if (far) {
          all[k] += some[k];
          some[k] = 0.f;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) sum[k] = all[k] + (some[k] + sum[k]);
    __syncthreads();              // of the run before, whose parts wave 0 has read
#pragma unroll
    for (int k = 0; k < 4; ++k) part[wave][lane * 4 + k] = sum[k];
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int w = 1; w < 4; ++w)
#pragma unroll
        for (int k = 0; k < 4; ++k) sum[k] += part[w][lane * 4 + k];
      write_row<ADD>(g, s, key, sum, old);
    }
  }
}

template <bool NARROW, bool ADD>
__global__ __launch_bounds__(256) void k_embed_grad_join(Runs g, int slabs) {
  __shared__ float part[4][kWave * 4];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int piece0 = int(blockIdx.x / slabs) * kJoinPieces, slab = int(blockIdx.x % slabs);
  bool starts = false, is_long = false;
  uint32_t key = 0;
  const int64_t p0 = int64_t(piece0 + lane) * g.piece, p1 = p0 + g.piece, p2 = p1 + g.piece, far = p1 + int64_t(kShortRun + 1) * g.piece;
  if (lane < kJoinPieces && p2 < g.T) {
    key = g.keys[p1];
    const uint32_t next = g.keys[p2], last = g.keys[p1 - 1], before = g.keys[max(p0 - 1, int64_t(0))], beyond = g.keys[min(far, int64_t(g.T) - 1)];
    starts = key < uint32_t(g.V) && last == key && next == key && !(p0 > 0 && before == key);
    is_long = far < g.T && beyond == key;
  }
  const uint64_t shorts = __ballot(starts && !is_long), longs = __ballot(starts && is_long);
  if (!(shorts | longs)) return;
  join_runs<NARROW, ADD>(g, shorts, longs, key, piece0, slab, lane, wave, part);
}

// Few tokens, in one launch: a workgroup for each token and slab looks through all ids, kFewEach a lane, for those that equal its token's; the
// workgroup of the first of them adds up their rows, by one wave up to kAhead rows, by all of its waves beyond.  One wave for up to 256
// tokens, four for up to 1024, while there are no more than kFewGroups workgroups.  Bound by the launch: 512 x 1024 take 5.3 us, 12 by the
// three steps; 1024 x 2048 (8192 workgroups) 11.2 and 13, 1024 x 4096 18.7 and 14.7; 256 x 4096 6.4 with one wave and 8.4 with four.
constexpr int kFewEach = 4, kFewGroups = 8192;

template <typename E, bool NARROW, bool ADD, int WAVES>
__global__ __launch_bounds__(WAVES *kWave) void k_embed_grad_few(Runs g, const E *dx, int run_groups) {
  constexpr int N = ElemTraits<E>::VEC, kFew = WAVES * kWave * kFewEach;
  __shared__ uint16_t list[kFew];
  __shared__ uint32_t named[WAVES * kMostFilled];
  __shared__ int found[WAVES], earlier[WAVES];
  __shared__ float part[WAVES][kWave * N];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if (int(blockIdx.x) >= run_groups) {
    const int job = int(blockIdx.x) - run_groups, slabs = (g.d + kFillColumns - 1) / kFillColumns;
    const int n = WAVES * g.fill_rows;
    const int64_t row0 = int64_t(job / slabs) * n;
    named[threadIdx.x] = row0 + threadIdx.x >= g.V;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kFewEach; ++i) {
      const int t = i * (WAVES * kWave) + threadIdx.x;
      const int64_t at = t < g.T ? int64_t(g.ids[min(t, g.T - 1)]) - row0 : -1;
      if (at >= 0 && at < n) named[at] = 1;
    }
    __syncthreads();
    zero_rows(g, row0 + wave * g.fill_rows, __ballot(lane < g.fill_rows && !named[wave * g.fill_rows + lane]), job % slabs * kFillColumns, lane);
    return;
  }
  const int t = int(blockIdx.x) / g.slabs, slab = int(blockIdx.x) % g.slabs;
  const int id = g.ids[t];
  int v[kFewEach];
#pragma unroll
  for (int i = 0; i < kFewEach; ++i) v[i] = g.ids[min((wave * kFewEach + i) * kWave + lane, g.T - 1)];
  if (uint32_t(id) >= uint32_t(g.V)) return;
  uint64_t hits[kFewEach];
  int n = 0, before = 0;
#pragma unroll
  for (int i = 0; i < kFewEach; ++i) {
    const int at = (wave * kFewEach + i) * kWave + lane;
    hits[i] = __ballot(at < g.T && v[i] == id);
    before += __popcll(__ballot(at < t && v[i] == id));
    n += __popcll(hits[i]);
  }
  if (lane == 0) {
    found[wave] = n;
    earlier[wave] = before;
  }
  __syncthreads();
  int total = 0, mine = 0, first = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    mine += w < wave ? found[w] : 0;
    total += found[w];
    first += earlier[w];
  }
  if (__builtin_amdgcn_readfirstlane(first)) return;   // another workgroup's
  n = __builtin_amdgcn_readfirstlane(total);
#pragma unroll
  for (int i = 0; i < kFewEach; ++i) {
    if (hits[i] >> lane & 1) list[mine + __popcll(hits[i] & ((uint64_t(1) << lane) - 1))] = uint16_t((wave * kFewEach + i) * kWave + lane);
    mine += __popcll(hits[i]);
  }
  __syncthreads();
  const Slab<E, NARROW> s(slab, lane, g.d);
  const bool shared = n > kAhead;
  if (!shared && wave) return;
  const int per = shared ? (n + WAVES - 1) / WAVES : n, p1 = min(n, (wave + 1) * per);
  float sum[N], old[N];
#pragma unroll
  for (int k = 0; k < N; ++k) sum[k] = 0.f;
  if (ADD && wave == 0) s.load(old, g.dtable + int64_t(id) * g.ldt);
  for (int p = wave * per; p < p1; p += kAhead) {
    const uint32_t order = list[min(p + lane % kAhead, p1 - 1)];
    typename Slab<E, NARROW>::Raw v[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) s.load(v[i], dx + int64_t(__builtin_amdgcn_readlane(order, i)) * g.ldx);
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (p + i < p1)
#pragma unroll
        for (int q = 0; q < N; ++q) sum[q] += v[i].at(q);
  }
  if (shared) {
#pragma unroll
    for (int k = 0; k < N; ++k) part[wave][lane * N + k] = sum[k];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w)
#pragma unroll
      for (int k = 0; k < N; ++k) sum[k] += part[w][lane * N + k];
  }
  write_row<ADD>(g, s, uint32_t(id), sum, old);
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
  const Lookup a = {g.ids, g.positions, g.V, g.P, g.ldw, g.ldp, g.ldx, g.scale};
  const Shares h = shares_of(g.T, g.d, 16 / o, 16 / o);
  DISPATCH_ROWS(g.prec, g.out_prec, {
    DISPATCH_SHARES(h.K, g.d, {
      hipLaunchKernelGGL((k_embed_lookup<L, E, K, NARROW>), h.grid, dim3(kThreads), 0, (hipStream_t)st, a, (const L *)g.table, (const L *)g.pos_table, (E *)g.x,
                         h.units);
    });
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
  const int slab = kWave * (g.prec == HMY_PREC_BF16 ? 8 : 4), slabs = (g.d + slab - 1) / slab, join_slabs = (g.d + 255) / 256;
  const int few = int64_t(T) * slabs > kFewGroups ? 0 : T <= kWave * kFewEach ? 1 : T <= 4 * kWave * kFewEach ? 4 : 0;   // waves of a workgroup
  Runs a = {nullptr, nullptr, g.ids, T, g.d, g.V, T <= kMostRanked ? kPieceRanked : kPieceSorted, 0, 0, g.ldx, g.ldt, g.dtable, nullptr, g.scale, std::max(4, std::min(kMostFilled, 4096 / std::min(g.d, kFillColumns)))};
  a.pieces = (T + a.piece - 1) / a.piece;
  a.partial = (float *)g.workspace + (int64_t(wanted) / 4 - 2 * int64_t(g.d) * a.pieces) / 4 * 4;   // at the workspace's end
  a.slabs = slabs;
  const int64_t run_groups = few ? int64_t(T) * slabs : (int64_t(a.pieces) * slabs + 3) / 4;
  const int filled = (few ? few : 4) * a.fill_rows;   // rows of a workgroup
  const int64_t fill_groups = g.accumulate ? 0 : (int64_t(g.V) + filled - 1) / filled * ((g.d + kFillColumns - 1) / kFillColumns);
  const int64_t join_groups = (int64_t(a.pieces) + kJoinPieces - 1) / kJoinPieces * join_slabs;
  // a launch has fewer than 2^32 threads, of which a workgroup has one wave's or four waves'
  const auto most_groups = [](int64_t threads) { return (int64_t(1) << 32) / threads - 1; };
  if (run_groups + fill_groups > most_groups(kWave * (few ? few : 4)) || join_groups > most_groups(4 * kWave))
    return fail(HMY_E_INVALID, "%s: T, d and V are too large together", who);
  const dim3 grid{uint32_t(run_groups + fill_groups)};
#define GRAD_AS(N, KERNEL, E, NARROW, ...)                                                                                                       \
  hipLaunchKernelGGL((g.accumulate ? KERNEL<E, NARROW, true, ##__VA_ARGS__> : KERNEL<E, NARROW, false, ##__VA_ARGS__>), grid, dim3(N), 0, s, a, \
                     (const E *)g.dx, int(run_groups))
#define GRAD(N, KERNEL, ...)                                             \
  do {                                                                   \
    if (g.prec == HMY_PREC_BF16) {                                       \
      if (g.d < 8) GRAD_AS(N, KERNEL, bf16_t, true, ##__VA_ARGS__);      \
      else GRAD_AS(N, KERNEL, bf16_t, false, ##__VA_ARGS__);             \
    } else {                                                             \
      if (g.d < 8) GRAD_AS(N, KERNEL, float, true, ##__VA_ARGS__);       \
      else GRAD_AS(N, KERNEL, float, false, ##__VA_ARGS__);              \
    }                                                                    \
  } while (0)
  if (few) {
    if (few == 1) GRAD(64, k_embed_grad_few, 1);
    else GRAD(256, k_embed_grad_few, 4);
    return check_launch(who);
  }
  const int64_t Ta = (int64_t(T) + 3) / 4 * 4;
  uint32_t *base = (uint32_t *)g.workspace;
  uint32_t *keys[2] = {base, base + 2 * Ta}, *order[2] = {base + Ta, base + 3 * Ta}, *counts = base + 4 * Ta;
  int sorted = 0;
  if (T <= kMostRanked) {
    hipLaunchKernelGGL(k_rank_tokens, dim3((T + kRankTokens - 1) / kRankTokens), dim3(kRankThreads),
                       size_t(T + 4 * kRankParts - 1) / (4 * kRankParts) * (4 * kRankParts) * 4, s, g.ids, T, g.V, keys[0], order[0]);
  } else {
    const int tiles = (T + kTile - 1) / kTile;
    int passes = 1;
    while (passes < 4 && (uint64_t(g.V) >> (8 * passes))) ++passes;
    for (int pass = 0; pass < passes; ++pass) {
      const int to = pass ? 1 - sorted : 0;
      const Sort q = {pass ? nullptr : g.ids, keys[sorted], order[sorted], T, g.V, 8 * pass, tiles, counts};
      hipLaunchKernelGGL(k_sort_count, dim3(tiles), dim3(kTileWaves * kWave), 0, s, q);
      if (tiles > kTilesRead) hipLaunchKernelGGL(k_sort_scan, dim3(kDigits / kWave), dim3(1024), 0, s, counts, tiles);
      hipLaunchKernelGGL(k_sort_place, dim3(tiles), dim3(kTileWaves * kWave), 0, s, q, keys[to], order[to]);
      sorted = to;
    }
  }
  a.keys = keys[sorted];
  a.order = order[sorted];
  if (int64_t(T) * g.d * e >= kStreamed) GRAD(256, k_embed_grad_runs, true);
  else GRAD(256, k_embed_grad_runs, false);
#undef GRAD
#undef GRAD_AS
  auto *join = g.d < 8 ? (g.accumulate ? k_embed_grad_join<true, true> : k_embed_grad_join<true, false>)
                       : (g.accumulate ? k_embed_grad_join<false, true> : k_embed_grad_join<false, false>);
  hipLaunchKernelGGL(join, dim3(uint32_t(join_groups)), dim3(256), 0, s, a, join_slabs);
  return check_launch(who);
}

}  // namespace hmy
