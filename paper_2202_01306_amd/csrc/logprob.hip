// Operators on rows of logits x[T,V]: log probabilities of given tokens with entropy and the most likely tokens, and their
// gradient.
//
// With the scale s, m = max x, u_j = s (x_j - m), S = sum exp u_j:  log p_j = u_j - log S,
//   H = log S - (sum u_j exp u_j) / S.
// u is taken from the difference to the maximum, so rows of the type's lowest value, or of very large values, lose nothing; a
// token at -inf has no weight (0 times its u counts as 0), a row of nothing else has m = -inf and S = 0.
#include <algorithm>

#include "logit_rows.h"

namespace hmy {

namespace {

// ---- the most likely tokens -------------------------------------------------------------------------------------------
// A token's rank as one number: the larger logit first, of equal ones the lower column.  +0 and -0 are equal.  Keys are unique
// and never 0, which stands for "none".
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ uint64_t rank_key(float x, int col) { return (uint64_t(ordered(x)) << 32) | uint32_t(~col); }
__device__ __forceinline__ int key_column(uint64_t key) { return int(~uint32_t(key)); }
constexpr uint32_t kLowestOrdered = 0x00800000u;   // of the lowest finite value: -inf and "none" are below

// What a workgroup finds a list with, in LDS: `keys` candidates at most; as many as `ranked` are ranked by comparing all with all;
// the segments of a row fall into `slots` slots, of which each thread knows its largest logit.
template <int NT_, int KEYS, int RANKED, int SLOTS, int HITS> struct Candidates {
  static constexpr int NT = NT_, keys = KEYS, ranked = RANKED, slots = SLOTS, hits = HITS;
  uint64_t key[KEYS];
  uint32_t rank[RANKED + kWave];
  float top[SLOTS * NT];           // a thread's largest logit in a slot
  uint32_t hit[HITS];              // slot * NT + thread of those that reach the floor
  uint32_t n, n_hits, floor, count[2];
};
// For rows (and parts of rows) of one slot, which are many at a time, and for longer ones.  On 64 threads for lists of up to
// kList64 entries only: there are but as many maxima to take the floor from as threads, and the floor has to be far above the
// lowest of them for few columns to pass.
template <int NT, bool ONE_SLOT> struct CandidatesOf { typedef Candidates<NT, 2048, 512, 8, 1024> type; };
template <int NT> struct CandidatesOf<NT, true> { typedef Candidates<NT, 1024, 512, 1, NT> type; };
template <> struct CandidatesOf<64, true> { typedef Candidates<64, 512, 256, 1, 64> type; };
constexpr int kList64 = 24, kList128 = 64;

// by one wave: some t with at least k of its values at or above it, and not many more if it can be had: the bisection ends at
// k + k / 8 + 2.  kLowestOrdered if fewer than k are at or above that.  count(t): how many are; each lane's smallest (of those
// from kLowestOrdered on) and largest in lo and hi.
template <typename F>
__device__ __forceinline__ uint32_t threshold(uint32_t lo, uint32_t hi, int k, F count) {
  if (count(kLowestOrdered) < k) return kLowestOrdered;
  hi = wave_top(hi);   // at or above lo: at least k; above hi: none
  lo = ~wave_top(~lo);
#pragma unroll 1
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo + 1) / 2;
    const int c = count(mid);
    if (c < k) {
      hi = mid - 1;
    } else {
      lo = mid;
      if (c <= k + k / 8 + 2) break;
    }
  }
  return lo;
}

// by the workgroup: the number of its threads' hits, all together
template <typename C>
__device__ __forceinline__ int hits(C &c, int mine, int &turn) {
  // two counters in turn: the next is cleared while this one is read
  const int total = int(wave_total(float(mine)));   // below 2^24: exact
  if (threadIdx.x % kWave == 0 && total) atomicAdd(&c.count[turn], uint32_t(total));
  __syncthreads();
  const int r = int(c.count[turn]);
  if (threadIdx.x == 0) c.count[turn ^ 1] = 0;
  __syncthreads();
  turn ^= 1;
  return r;
}

// by the workgroup: leaves only those of n > k candidates that the k largest can be among, at most `most` of them, and says how
// many.  Wants a barrier in front.  The first wave does it: there is little to do, and the others keep their registers.
template <typename C>
__device__ __forceinline__ int thin_out(C &c, int n, int k, int most) {
  const int lane = threadIdx.x;
  if (lane < kWave) {
    uint32_t lo = ~0u, hi = 0;
#pragma unroll 1
    for (int i = lane; i < n; i += kWave) {
      const uint32_t v = uint32_t(c.key[i] >> 32);   // at or above kLowestOrdered: -inf is no candidate
      lo = min(lo, v);
      hi = max(hi, v);
    }
    auto count = [&](uint64_t t) {
      int r = 0;
#pragma unroll 1
      for (int i = lane; i - lane < n; i += 4 * kWave) {
        bool in[4];
#pragma unroll
        for (int o = 0; o < 4; ++o) in[o] = c.key[min(i + o * kWave, n - 1)] >= t && i + o * kWave < n;
#pragma unroll
        for (int o = 0; o < 4; ++o) r += __popcll(__ballot(in[o]));
      }
      return r;
    };
    uint64_t least = uint64_t(threshold(lo, hi, k, [&](uint32_t t) { return count(uint64_t(t) << 32); })) << 32;
    if (count(least) > most) {   // many equal logits: the k-th largest key itself, bit by bit
      least = 0;
#pragma unroll 1
      for (int bit = 63; bit >= 0; --bit)
        if (count(least | uint64_t(1) << bit) >= k) least |= uint64_t(1) << bit;
    }
    int kept = 0;
#pragma unroll 1
    for (int i = 0; i < n; i += kWave) {   // to places that have been read already
      const uint64_t key = i + lane < n ? c.key[i + lane] : 0;
      const uint64_t keep = __ballot(key >= least && key != 0);
      if (key >= least && key != 0) c.key[kept + __popcll(keep & ((uint64_t(1) << lane) - 1))] = key;
      kept += __popcll(keep);
    }
    if (lane == 0) c.n = kept;
  }
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(c.n);
}

// by the workgroup, where more than there is room for reach a floor that at least k of the columns x[0 .. cols-1] (numbered from
// `first` on) reach: very many are equal, as in the rows of an untrained model or under masks of a finite value, or the largest
// logits are those of few threads.  All columns are read again: those above the floor, and while there is no room for them
// either, for what the k-th of an arbitrary part of them gives as a floor; then the lowest columns that equal it.  Says how many
// candidates there are.  Wants a barrier in front.
template <typename C, typename L>
__device__ __forceinline__ int list_ties(C &c, const L *x, int first, int cols, int k, float floor) {
  constexpr int NT = C::NT, kRoom = C::keys - 8;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  int n;
#pragma unroll 1
  while (true) {
    if (tid == 0) c.n = 0;
    __syncthreads();
#pragma unroll 1
    for (int j0 = 0; j0 < cols; j0 += NT) {
      const int j = j0 + tid;
      const float v = j < cols ? to_f32(x[j]) : -INFINITY;
      const uint64_t above = __ballot(v > floor);
      if (above) {
        int at = 0;
        if (lane == 0) at = int(atomicAdd(&c.n, uint32_t(__popcll(above))));
        at = __builtin_amdgcn_readfirstlane(at) + __popcll(above & ((uint64_t(1) << lane) - 1));
        if (v > floor && at < kRoom) c.key[at] = rank_key(v, first + j);
      }
    }
    __syncthreads();
    n = __builtin_amdgcn_readfirstlane(c.n);
    if (n <= kRoom) break;
    if (tid < kWave) {
      uint32_t lo = ~0u, hi = 0;
      for (int i = lane; i < kRoom; i += kWave) {
        const uint32_t v = uint32_t(c.key[i] >> 32);
        lo = min(lo, v);
        hi = max(hi, v);
      }
      const uint32_t t = threshold(lo, hi, k, [&](uint32_t to) {
        int r = 0;
        for (int i = 0; i < kRoom; i += kWave) r += __popcll(__ballot(i + lane < kRoom && uint32_t(c.key[min(i + lane, kRoom - 1)] >> 32) >= to));
        return r;
      });
      if (lane == 0) c.floor = t;
    }
    __syncthreads();
    floor = unordered(__builtin_amdgcn_readfirstlane(c.floor));   // above the one before
  }
  __syncthreads();   // all have read c.n, which thin_out writes: no column that equals the floor may be wanted
  const int wanted = k - n;   // of those that equal the floor, the lowest columns first
  int taken = 0;
#pragma unroll 1
  for (int j0 = 0; j0 < cols && taken < wanted; j0 += NT) {
    const int j = j0 + tid;
    const bool equal = j < cols && to_f32(x[j]) == floor;
    const uint64_t equals = __ballot(equal);
    if (lane == 0) c.rank[wave] = uint32_t(__popcll(equals));
    __syncthreads();
    int before = taken;
    for (int w = 0; w < NT / kWave; ++w) {
      if (w < wave) before += int(c.rank[w]);
      taken += int(c.rank[w]);
    }
    before += __popcll(equals & ((uint64_t(1) << lane) - 1));
    if (equal && before < wanted) c.key[n + before] = rank_key(floor, first + j);
    __syncthreads();
  }
  return n + max(0, min(taken, wanted));
}

// by the workgroup: the k first of n candidates, `put(rank, key)` for each.  Wants a barrier in front.
template <typename C, typename F>
__device__ __forceinline__ void rank_candidates(C &c, int n, int k, F put) {
  constexpr int NT = C::NT;
  const int tid = threadIdx.x;
  if (n > min(2 * k + 64, C::ranked)) n = thin_out(c, n, k, C::ranked);
  // n is at most C::ranked now.  All compared with all: `parts` threads share the comparisons of one candidate.
  const int wide = (n + kWave - 1) / kWave * kWave, parts = max(1, NT / max(wide, 1)), share = ((n + parts - 1) / parts + 7) / 8 * 8;
  for (int i = tid; i < wide; i += NT) c.rank[i] = 0;
  if (tid < 8) c.key[n + tid] = 0;
  __syncthreads();
  for (int i = tid; i < wide * parts; i += NT) {
    const int own = i % wide, first = i / wide * share;
    const uint64_t mine = own < n ? c.key[own] : ~uint64_t(0);
    int above = 0;
    for (int j = first; j < min(first + share, n); j += 8) {
#pragma unroll
      for (int o = 0; o < 8; ++o) above += c.key[j + o] > mine;
    }
    if (above) atomicAdd(&c.rank[own], uint32_t(above));
  }
  __syncthreads();
  for (int i = tid; i < n; i += NT)
    if (int(c.rank[i]) < k) put(int(c.rank[i]), c.key[i]);
  for (int i = n + tid; i < k; i += NT) put(i, uint64_t(0));
}

// ---- forward ------------------------------------------------------------------------------------------------------------
struct LogprobArgs {
  const int32_t *targets;
  float *logp, *row_max, *log_sum, *entropy;
  int32_t *top_ids;
  float *top_logp;
  int V, k;
  int64_t ldl;
  float scale;
};

// m, sum exp(s (x - m)) and sum exp(u) u (u = s (x - m) in log2 units) of some of a row's tokens
struct Sums { float m, S, A; };
__device__ __forceinline__ Sums no_sums() { return {-INFINITY, 0.f, 0.f}; }
// the same two sums relative to `to` >= m
__device__ __forceinline__ Sums relative_to(const Sums &z, float to, float scale) {
  Sums r = {to, 0.f, 0.f};
  if (z.S == 0.f) return r;
  const float f = rebase(z.m, to, scale), u = fmaxf((z.m - to) * (scale * kLog2e), kNoWeight);
  r.S = z.S * f;
  r.A = f * fmaf(u, z.S, z.A);
  return r;
}
__device__ __forceinline__ Sums wave_sums(const Sums &z, float scale) {
  Sums r = relative_to(z, wave_top(z.m), scale);
  r.S = wave_total(r.S);
  r.A = wave_total(r.A);
  return r;
}
// A thread's sums while it reads.  Exponents in log2 units, u = c x - R with R near c m, take one instruction, and one rounding;
// what R is beside c m, d = c m - R, is taken out at the end.  Where c m itself is beyond kLargest, d is no small number: a thread's
// tokens that are that far down have no weight beside a row's maximum that is not, and for a row whose maximum is, the sums are
// taken once more, from c (x - m).  bf16 is bound by what it computes, too: us, with c (x - m) throughout / as it is, 1027 x 30522,
// k = 20, 22.3 / 21.7; 2048 x 131072, k = 128, 123.8 / 121.4.
constexpr float kLargest = 1 << 20;
struct Running {
  float m, R, S, A;
  __device__ __forceinline__ static float reference(float mc) { return fminf(fmaxf(mc, -kLargest), kLargest); }
  __device__ __forceinline__ void raise(float to, float c) {   // to > m
    const float next = reference(to * c), by = R - next, f = fast_exp2(by);
    A = f * fmaf(by, S, A);
    S *= f;
    m = to;
    R = next;
  }
  __device__ __forceinline__ void add(float u) {
    const float e = fast_exp2(u);
    S += e;
    A = fmaf(e, fmaxf(u, kNoWeight), A);
  }
  __device__ __forceinline__ Sums sums(float c) const {
    const float d = fmaf(m, c, -R), down = d > -126.f ? d : 0.f, f = d > -126.f ? fast_exp2(-d) : 0.f;
    return {m, f * S, fmaf(-down, f * S, f * A)};
  }
};
// Few, long rows: per_row <= 64 workgroups each take `cols` (a multiple of eight) of a row's columns.
struct RowParts {
  Sums *sums;          // [rows * per_row]
  uint64_t *keys;      // [rows * per_row, k]
  int per_row, cols;
};
// one entry of a row's list
struct PutEntry {
  int32_t *ids;
  float *logp;
  float m, scale, log_sum;
  __device__ __forceinline__ PutEntry(const LogprobArgs &a, int row, const Sums &z)
      : ids(a.top_ids + int64_t(row) * a.k), logp(a.top_logp + int64_t(row) * a.k), m(z.m), scale(a.scale), log_sum(logf(z.S)) {}
  __device__ __forceinline__ void operator()(int rank, uint64_t key) const {
    ids[rank] = key ? key_column(key) : -1;
    logp[rank] = key ? (unordered(uint32_t(key >> 32)) - m) * scale - log_sum : -INFINITY;
  }
};
__device__ __forceinline__ void put_row(const LogprobArgs &a, int row, const Sums &z, float target_logit, bool has_target) {
  const float log_sum = logf(z.S), ref = z.m == -INFINITY ? 0.f : z.m;
  if (a.logp) a.logp[row] = !has_target ? 0.f : z.S == 0.f ? -INFINITY : (target_logit - ref) * a.scale - log_sum;
  if (a.row_max) a.row_max[row] = z.m;
  if (a.log_sum) a.log_sum[row] = log_sum;
  if (a.entropy) a.entropy[row] = z.S == 0.f ? 0.f : log_sum - z.A * kLn2 / z.S;
}

// by the workgroup: the k first of the columns x[0 .. cols-1], numbered from `first` on, `put(rank, key)` for each.  `mine`: this thread's largest logit, c.top its
// largest per slot of `per_slot` segments; xb: the logit of column `behind`, -inf where the thread has none.
// A floor that at least k logits reach: the k-th largest, or a little less, of the maxima of 256 groups of threads (FINE = 4: `fine`
// holds this thread's largest of each fourth of its columns, and there are 512 groups, at a cost of 0.6 us; 2048 rows of 512 columns
// in fp32, us on one maximum / four: k = 64 on 128 threads 21.3 / 12.9, k = 128 on 256 31.1 / 21.7, but k = 32 of 4000 13.6 / 14.5).  What reaches
// it is in the slots of few threads (k of 256 groups at least; as many as the row's largest logits fall into), and those columns
// are read again: a second reading of a small part of the row (counted: 7 % of 512 x 50257 fp32 at k = 64, 30 % of 2048 x 131072
// bf16 at k = 128, whose 128 entries are in 128 of 4096 slots), where looking for candidates in the first one costs every segment a
// comparison and a barrier.  us, with the floor's columns read again / looked for in the one reading: 2048 x 131072 bf16, k = 128,
// 119 / 192; 512 x 50257 fp32, k = 64, 24.2 / 39; without a list 98 and 18.5.
template <int NG, int FINE, typename C, typename L, typename F>
__device__ __forceinline__ void list_row(C &c, const L *x, int first, int groups, int cols, int per_slot, int k, const float (&fine)[FINE], float mine, float xb, int behind, F put) {
  constexpr int NT = C::NT, kSegment = NT * NG, kGroups = FINE == 1 ? 4 : 8;   // a lane's
  const int tid = threadIdx.x, lane = tid % kWave;
  const int slots = ((groups + kSegment - 1) / kSegment + per_slot - 1) / per_slot;
  uint32_t *group = reinterpret_cast<uint32_t *>(c.key);   // free until there are candidates
  static_assert(FINE * NT * sizeof(uint32_t) <= sizeof(c.key), "the maxima fit");
#pragma unroll
  for (int f = 0; f < FINE; ++f) group[f * NT + tid] = ordered(f == 0 ? fmaxf(fine[f], xb) : fine[f]);
  if (tid == 0) c.n = c.n_hits = 0;
  __syncthreads();
  if (tid < kWave) {
    uint32_t g[kGroups] = {}, lo = ~0u, hi = 0;
#pragma unroll
    for (int f = 0; f < FINE; ++f)
#pragma unroll
      for (int w = 0; w < NT / kWave; ++w) {
        uint32_t &to = g[f * (kGroups / FINE) + w % (kGroups / FINE)];
        to = max(to, group[f * NT + w * kWave + lane]);
      }
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      hi = max(hi, g[i]);
      if (g[i] >= kLowestOrdered) lo = min(lo, g[i]);
    }
    const uint32_t t = threshold(lo, hi, k, [&](uint32_t to) {
      int r = 0;
#pragma unroll
      for (int i = 0; i < kGroups; ++i) r += __popcll(__ballot(g[i] >= to));
      return r;
    });
    if (lane == 0) c.floor = t;
  }
  __syncthreads();
  const float floor = unordered(__builtin_amdgcn_readfirstlane(c.floor));
  if (mine >= floor) {
    for (int s = 0; s < slots; ++s)
      if (c.top[s * NT + tid] >= floor) {
        const uint32_t at = atomicAdd(&c.n_hits, 1u);
        if (at < C::hits) c.hit[at] = s * NT + tid;
      }
  }
  __syncthreads();
  if (xb >= floor) {   // other waves may be counting what they find below by now: there may be no room left
    const uint32_t at = atomicAdd(&c.n, 1u);
    if (at < C::keys) c.key[at] = rank_key(xb, first + behind);
  }
  const int n_hits = int(c.n_hits);
  if (n_hits <= C::hits) {
    for (int s = 0; s < per_slot; ++s)
      for (int i = tid; i < n_hits * NG; i += NT) {
        const uint32_t h = c.hit[i / NG];
        const int g = ((h / NT) * per_slot + s) * kSegment + (i % NG) * NT + h % NT;
        if (g < groups) {
          Eight<L> v;
          load_whole(v, x + uint32_t(g) * 8);
          int above = 0;
#pragma unroll
          for (int o = 0; o < 8; ++o) above += v.at(o) >= floor;
          if (above) {
            uint32_t at = atomicAdd(&c.n, uint32_t(above));
#pragma unroll
            for (int o = 0; o < 8; ++o)
              if (v.at(o) >= floor) {
                if (at < C::keys) c.key[at] = rank_key(v.at(o), first + g * 8 + o);
                ++at;
              }
          }
        }
      }
  }
  __syncthreads();
  int n = __builtin_amdgcn_readfirstlane(c.n);
  __syncthreads();   // all have read c.n, which is written again
  if (n > C::keys - 8 || n_hits > C::hits) n = list_ties(c, x, first, cols, k, floor);   // (eight keys more are written behind n)
  rank_candidates(c, n, k, put);
}

// One workgroup per row (PARTS: per part of a row, of which the workspace gets the sums and the list), NT * NG groups of eight
// columns at a time, the next ones' loads on their way meanwhile.  One reading: each thread keeps a running maximum and sums
// relative to it, and its largest logit per slot for the list (LIST = 4: of each fourth of its columns, in rows of one slot, where
// a long list is to be taken from few threads' maxima; LIST = 0: no list).  Bound by HBM where there are rows for all compute units: 512 x
// 50257 fp32 18.5 us (5.5 TB/s), 2048 x 131072 bf16 98 (5.5); a large copy runs at 5.06, a reading sum at 3.97.  Few or short
// rows are a chain of latencies: launch, ids, one round of loads, one barrier, and with a list four more (6 us for 64 rows of 512
// columns, 9.5 for one of 50257, with a list each).
template <typename L, int NT, int NG, int LIST, bool ONE_SLOT, bool PARTS>
__global__ __launch_bounds__(NT) void k_logprob(const L *logits, LogprobArgs a, RowParts p) {
  constexpr int kWaves = NT / kWave, kSegment = NT * NG;
  typedef typename CandidatesOf<NT, ONE_SLOT>::type Cands;
  __shared__ Sums part[kWaves];
  __shared__ __attribute__((aligned(16))) char cand_[LIST ? sizeof(Cands) : 1];
  Cands &cand = *reinterpret_cast<Cands *>(cand_);
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int row = PARTS ? blockIdx.x / p.per_row : blockIdx.x, piece = PARTS ? blockIdx.x % p.per_row : 0;
  const float c = a.scale * kLog2e;
  // columns first .. first+cols-1
  const int first = PARTS ? piece * p.cols : 0, cols = PARTS ? min(p.cols, a.V - first) : a.V;
  const L *x = logits + int64_t(row) * a.ldl + first;
  const int groups = cols / 8, segments = (groups + kSegment - 1) / kSegment;
  const int per_slot = max(1, (segments + Cands::slots - 1) / Cands::slots);   // list_row divides by it, also for rows of no group
  // the column behind the groups, if there is one for this thread
  const int behind = groups * 8 + tid;
  const float xb = behind < cols ? to_f32(x[behind]) : -INFINITY;
  auto load = [&](Eight<L> (&v)[NG], int seg) {
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const int g = seg * kSegment + i * NT + tid;
      if (g < groups) load_whole(v[i], x + uint32_t(g) * 8);
      else v[i].all_no_weight();
    }
  };
  Eight<L> v[NG], next[NG];
  if (segments > 0) load(v, 0);
  // behind the columns' loads: the first of these two is waited for before the second is issued
  const int tgt = !PARTS && a.targets ? a.targets[row] : -1;
  const bool has_target = tgt >= 0 && tgt < a.V;
  const float target_logit = has_target ? to_f32(x[tgt]) : 0.f;
  Running z = {fmaxf(xb, -INFINITY), Running::reference(xb * c), 0.f, 0.f};
  z.add(fmaf(xb, c, -z.R));   // nothing for -inf, NaN for what is no number
  constexpr int kFine = LIST ? LIST : 1;
  static_assert(LIST <= 1 || ONE_SLOT, "several maxima a thread in one slot");
  float in_slot = -INFINITY, fine[kFine];
#pragma unroll
  for (int f = 0; f < kFine; ++f) fine[f] = -INFINITY;
  for (int seg = 0, of_slot = 0; seg < segments; ++seg) {
    if (seg + 1 < segments) load(next, seg + 1);
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < NG; ++i) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if constexpr (kFine > 1) fine[k / 2] = fmaxf(fine[k / 2], v[i].at(k));
        else top = fmaxf(top, v[i].at(k));
      }
      v[i].forget_floats();
    }
    if constexpr (kFine > 1) {
      top = fmaxf(fmaxf(fine[0], fine[1]), fmaxf(fine[2], fine[3]));   // of all segments so far
      if (seg + 1 == segments) cand.top[tid] = top;
    } else if constexpr (LIST) {
      in_slot = fmaxf(in_slot, top);
      if (++of_slot == per_slot || seg + 1 == segments) {
        cand.top[(seg / per_slot) * NT + tid] = in_slot;
        in_slot = -INFINITY;
        of_slot = 0;
      }
    }
    if (top > z.m) z.raise(top, c);
#pragma unroll
    for (int i = 0; i < NG; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) z.add(fmaf(v[i].at(k), c, -z.R));
#pragma unroll
    for (int i = 0; i < NG; ++i) v[i] = next[i];
  }
  if constexpr (kFine == 1) fine[0] = z.m;
  const Sums ws = wave_sums(z.sums(c), a.scale);
  if (lane == 0) part[wave] = ws;
  __syncthreads();
  Sums all = lane < kWaves ? part[lane] : no_sums();
  all = wave_sums(all, a.scale);
  if (all.m != -INFINITY && !(fabsf(all.m * c) <= kLargest)) {
    Running r = {all.m, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int g = tid; g < groups; g += NT) {
      Eight<L> w;
      load_whole(w, x + uint32_t(g) * 8);
#pragma unroll
      for (int k = 0; k < 8; ++k) r.add((w.at(k) - all.m) * c);
    }
    if (behind < cols) r.add((xb - all.m) * c);
    __syncthreads();   // all have read the waves' sums
    const Sums again = wave_sums({all.m, r.S, r.A}, a.scale);
    if (lane == 0) part[wave] = again;
    __syncthreads();
    all = wave_sums(lane < kWaves ? part[lane] : no_sums(), a.scale);
  }
  if constexpr (PARTS) {
    if (tid == 0) p.sums[blockIdx.x] = all;
    if constexpr (LIST)
      list_row<NG>(cand, x, first, groups, cols, per_slot, a.k, fine, z.m, xb, behind, [&](int rank, uint64_t key) { p.keys[int64_t(blockIdx.x) * a.k + rank] = key; });
  } else {
    if (tid == 0) put_row(a, row, all, target_logit, has_target);
    if constexpr (LIST) list_row<NG>(cand, x, 0, groups, cols, per_slot, a.k, fine, z.m, xb, behind, PutEntry(a, row, all));
  }
}

// The rows of few, long rows whose parts have been taken by a workgroup each: sums of the parts' sums, and the first of the
// parts' lists.
constexpr int kJoinThreads = 256;
template <typename L>
__global__ __launch_bounds__(kJoinThreads) void k_logprob_join(const L *logits, LogprobArgs a, RowParts p) {
  typedef Candidates<kJoinThreads, 2048, 512, 1, 1> Cands;
  __shared__ __attribute__((aligned(16))) Cands cand;
  const int tid = threadIdx.x, lane = tid % kWave, row = blockIdx.x;
  const Sums all = wave_sums(lane < p.per_row ? p.sums[row * p.per_row + lane] : no_sums(), a.scale);   // per_row <= 64
  if (tid == 0) {
    const int tgt = a.targets ? a.targets[row] : -1;
    const bool has_target = tgt >= 0 && tgt < a.V;
    put_row(a, row, all, has_target ? to_f32(logits[int64_t(row) * a.ldl + tgt]) : 0.f, has_target);
  }
  if (!a.k) return;
  // What at least k of the parts' keys reach: each part's j-th with j parts >= k, or the k-th of one part.  0: none
  const uint64_t *keys = p.keys + int64_t(row) * p.per_row * a.k;
  const int total = p.per_row * a.k, j = (a.k + p.per_row - 1) / p.per_row;
  uint64_t each = lane < p.per_row ? keys[lane * a.k + j - 1] : ~uint64_t(0), one = lane < p.per_row ? keys[lane * a.k + a.k - 1] : 0;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    each = min(each, uint64_t(__shfl_xor((unsigned long long)each, o, kWave)));
    one = max(one, uint64_t(__shfl_xor((unsigned long long)one, o, kWave)));
  }
  uint64_t least = max(max(each, one), uint64_t(1));
  if (tid == 0) cand.n = cand.count[0] = cand.count[1] = 0;
  __syncthreads();
  int turn = 0;
  auto reach = [&](uint64_t t) {
    int r = 0;
    for (int i = tid; i < total; i += kJoinThreads) r += keys[i] >= t;
    return hits(cand, r, turn);
  };
  if (reach(least) > Cands::keys - 8) {   // most of the list in one or two parts: the k-th largest key itself, bit by bit
    least = 0;
#pragma unroll 1
    for (int bit = 63; bit >= 0; --bit)
      if (reach(least | uint64_t(1) << bit) >= a.k) least |= uint64_t(1) << bit;
  }
  for (int i = tid; i < total; i += kJoinThreads)
    if (keys[i] >= least) cand.key[atomicAdd(&cand.n, 1u)] = keys[i];
  __syncthreads();
  const int n = __builtin_amdgcn_readfirstlane(cand.n);
  __syncthreads();
  rank_candidates(cand, n, a.k, PutEntry(a, row, all));
}

struct LogprobGradArgs {
  const float *row_max, *log_sum;
  const int32_t *targets;
  const float *d_logp, *entropy, *d_entropy;
  int T, V, pad;
  int64_t ldl, ldd;
  float scale;
};

// g_j = s (a (1[j = target] - p_j) - h p_j (log p_j + H)) with a = dL/dlogp, h = dL/dH.  Every column on its own: a stream over
// the logits and the gradient, bound by HBM.  A workgroup takes NT * U * 8 columns of one row, all of a thread's loads in flight
// before its first store.  us (TB/s), rows x columns, U = 2: fp32 into bf16, 512 x 50257 30.0 (5.1); bf16, 1111 x 131071 99.5
// (5.9), x 131072 102.6 (5.7): rows that start off any alignment cost nothing.  A large copy runs at 5.06.  U = 1 took 2 % and 19 %
// more, U = 4 6 % and 2 %.
template <typename L, typename E, int NT, int U>
__global__ __launch_bounds__(NT) void k_logprob_bwd(const L *logits, E *dlogits, LogprobGradArgs g, int tiles) {
  const int64_t n = int64_t(g.T) * tiles;
  const uint32_t whole = uint32_t(g.V) & ~7u;
  for (int64_t wg = blockIdx.x; wg < n; wg += gridDim.x) {
    const int row = int(wg / tiles), tile = int(wg % tiles);
    const uint32_t c0 = (uint32_t(tile) * NT * U + threadIdx.x) * 8;
    const L *x = logits + int64_t(row) * g.ldl;
    E *d = dlogits + int64_t(row) * g.ldd;
    Eight<L> v[U];
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (c0 + i * NT * 8 < whole) load_whole(v[i], x + (c0 + i * NT * 8));
    const float m = g.row_max[row], z = g.log_sum[row];
    const int tgt = g.targets ? g.targets[row] : -1;
    const float a = g.d_logp && tgt >= 0 && tgt < g.V ? g.d_logp[row] : 0.f;
    const float h = g.d_entropy ? g.d_entropy[row] : 0.f, H = g.d_entropy ? g.entropy[row] : 0.f;
    const float na = -g.scale * fmaf(h, H, a), nh = -g.scale * h;
    const bool empty = z == -INFINITY;   // no token has any weight: p = 0 throughout
    auto grad = [&](float xj) {
      const float l = fmaf(xj - m, g.scale, -z);
      return empty ? 0.f : fast_exp2(l * kLog2e) * fmaf(nh, fmaxf(l, kNoWeight), na);
    };
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const uint32_t col = c0 + i * NT * 8;
      if (col < whole) {
        float o[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) o[k] = grad(v[i].at(k));
        if (uint32_t(tgt) - col < 8u) {
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (int(col) + k == tgt) o[k] = fmaf(g.scale, a, o[k]);
        }
        store_whole(d + col, o);
      }
    }
    if (tile == tiles - 1) {
      const int col = int(whole) + int(threadIdx.x);
      if (col < g.V) d[col] = from_f32<E>(fmaf(g.scale, col == tgt ? a : 0.f, grad(to_f32(x[col]))));
      zero_padding(d, g.V, g.pad, threadIdx.x, NT);
    }
  }
}

template <typename L, int NT, int NG, bool ONE_SLOT>
void launch_rows(const L *x, LogprobArgs a, int rows, hipStream_t s) {
  const RowParts none = {};
  for (; rows > 0; rows -= kMaxGrid) {   // a launch has a limited number of workgroups
    const dim3 grid(rows < kMaxGrid ? rows : kMaxGrid);
    constexpr int kFine = ONE_SLOT && NT > 64 ? 4 : 1;   // 64 threads have no such lists
    if (a.k > NT / 4 && kFine > 1) hipLaunchKernelGGL((k_logprob<L, NT, NG, kFine, ONE_SLOT, false>), grid, dim3(NT), 0, s, x, a, none);
    else if (a.k) hipLaunchKernelGGL((k_logprob<L, NT, NG, 1, ONE_SLOT, false>), grid, dim3(NT), 0, s, x, a, none);
    else hipLaunchKernelGGL((k_logprob<L, NT, NG, 0, true, false>), grid, dim3(NT), 0, s, x, a, none);
    x += int64_t(kMaxGrid) * a.ldl;
    for (float **p : {&a.logp, &a.row_max, &a.log_sum, &a.entropy})
      if (*p) *p += kMaxGrid;
    if (a.targets) a.targets += kMaxGrid;
    if (a.k) {
      a.top_ids += int64_t(kMaxGrid) * a.k;
      a.top_logp += int64_t(kMaxGrid) * a.k;
    }
  }
}

constexpr int kPartLaunch = 512, kPartMinCols = 16384, kPartMaxCols = 65536, kPartsMax = 64;
static_assert(kPartLaunch * (sizeof(Sums) + 4 + HMY_MAX_TOP * 8) <= HMY_ROWS_WORKSPACE_BYTES, "the parts' sums and lists fit the workspace");

template <typename L>
void launch_rows(const L *x, const LogprobArgs &a, int rows, void *workspace, hipStream_t s) {
  // Parts: two launches, the second of which waits for the first and ranks the parts' lists, so a row has to be long enough for
  // six parts, rows few, fewer with long lists, and parts short, for their list is ranked on one slot.  us by parts / by rows, fp32:
  // one row of 131072, k = 10, 11.6 / 16.3; of 80000 (four parts) 12.5 / 12.4; 32 rows of 131072, k = 128, 21.8 / 20.5.
  const int room = rows <= (a.k > kList64 ? 16 : 64) ? kPartLaunch / rows : 1;
  const int parts = std::min(std::min(room, kPartsMax), a.V / kPartMinCols);
  // Short rows are bound by what a workgroup does once, not by the columns: fewer threads, more workgroups at a time.  us on 64 /
  // 128 / 256 threads, bf16, 8192 rows: 2000 columns, k = 20, 21.7 / - / 40.4, 4000 columns, k = 0, 17.3 / 16.8 / 25.2, k = 20, 31.2 /
  // 29.4 / 40.3, 8000 columns, k = 20, 51.5 / 44.5 / 41.9.  Where rows are few a long list is quicker on more threads: 1000 columns,
  // k = 64, on 64 / 128, one row 11.8 / 9.1, 2048 rows 15.1 / 13.7; k = 128 on 128 / 256 (fp32), 512 rows 16.0 / 11.9, 1024 15.9 /
  // 14.1, 2048 19.9 / 24.9, 8192 62 / 78.
  // One slot while a thread has but one: 8000 columns, k = 20, 42.6, with eight (twice the LDS) 51.8.  256 against 512 threads:
  // 4096 rows of 20000 columns, k = 20, 51.1 / 64.0, of 12000 36.9 / 47.2; 1024 rows of 131072, k = 128, 75.8 / 70.2 (fp32 117 / 104).
  if (workspace && parts >= 6 && a.V / parts <= kPartMaxCols) {
    RowParts p;
    p.cols = (a.V + parts - 1) / parts + 7 & ~7;
    p.per_row = (a.V + p.cols - 1) / p.cols;
    p.keys = static_cast<uint64_t *>(workspace);
    p.sums = reinterpret_cast<Sums *>(p.keys + int64_t(rows) * p.per_row * a.k);
    const dim3 grid(rows * p.per_row);
    if (a.k) hipLaunchKernelGGL((k_logprob<L, 512, sizeof(L) == 4 ? 2 : 4, 1, true, true>), grid, dim3(512), 0, s, x, a, p);
    else hipLaunchKernelGGL((k_logprob<L, 512, sizeof(L) == 4 ? 2 : 4, 0, true, true>), grid, dim3(512), 0, s, x, a, p);
    hipLaunchKernelGGL(k_logprob_join<L>, dim3(rows), dim3(kJoinThreads), 0, s, x, a, p);
  } else if (a.V <= 2048 && a.k <= kList64) {
    launch_rows<L, 64, 4, true>(x, a, rows, s);
  } else if (a.V <= 4096 && (a.k <= kList128 || rows >= 2048)) {
    launch_rows<L, 128, 4, true>(x, a, rows, s);
  } else if (a.V <= 8192) {
    launch_rows<L, 256, 4, true>(x, a, rows, s);
  } else if (a.V <= 32768) {
    launch_rows<L, 256, 4, false>(x, a, rows, s);
  } else {
    launch_rows<L, 512, sizeof(L) == 4 ? 2 : 4, false>(x, a, rows, s);
  }
}

}  // namespace

int launch_logprob(const hmy_logprob_desc &g, stream_t st) {
  int rc = check_rows("logprob", g.logits_prec, g.logits, g.T, g.V, 0, g.ldl);
  if (rc) return rc;
  if (!usable_scale(g.scale)) return fail(HMY_E_INVALID, "logprob: the scale must be positive and finite");
  if (g.k < 0 || g.k > HMY_MAX_TOP) return fail(HMY_E_INVALID, "logprob: k = %d is not in 0..%d", g.k, HMY_MAX_TOP);
  if (g.k > 0 && (!g.top_ids || !g.top_logp)) return fail(HMY_E_INVALID, "logprob: k > 0 needs top_ids and top_logp");
  if (!g.targets != !g.logp) return fail(HMY_E_INVALID, "logprob: targets and logp come together");
  if (!g.logp && !g.row_max && !g.log_sum && !g.entropy && !g.k) return fail(HMY_E_INVALID, "logprob: no output asked for");
  const void *words[] = {g.targets, g.logp, g.row_max, g.log_sum, g.entropy, g.top_ids, g.top_logp};
  for (const void *p : words)
    if (misaligned(p, 4)) return fail(HMY_E_INVALID, "logprob: misaligned array");
  const LogprobArgs a = {g.targets, g.logp, g.row_max, g.log_sum, g.entropy, g.top_ids, g.top_logp, g.V, g.k, g.ldl, g.scale};
  const hipStream_t s = (hipStream_t)st;
  void *ws = has_workspace(g.workspace, g.workspace_bytes) ? g.workspace : nullptr;
  if (misaligned(ws, 16)) return fail(HMY_E_INVALID, "logprob: workspace not aligned to 16 bytes");
  if (g.logits_prec == HMY_PREC_BF16) launch_rows((const bf16_t *)g.logits, a, g.T, ws, s);
  else launch_rows((const float *)g.logits, a, g.T, ws, s);
  return check_launch("logprob");
}

int launch_logprob_bwd(const hmy_logprob_grad_desc &g, stream_t st) {
  int rc = check_rows("logprob_bwd", g.logits_prec, g.logits, g.T, g.V, 0, g.ldl);
  if (!rc) rc = check_rows("logprob_bwd", g.prec, g.dlogits, g.T, g.V, g.pad, g.ldd);
  if (rc) return rc;
  if (!usable_scale(g.scale)) return fail(HMY_E_INVALID, "logprob_bwd: the scale must be positive and finite");
  if (!g.d_logp && !g.d_entropy) return fail(HMY_E_INVALID, "logprob_bwd: d_logp, d_entropy or both wanted");
  if (g.d_logp && !g.targets) return fail(HMY_E_INVALID, "logprob_bwd: d_logp needs targets");
  if (g.d_entropy && !g.entropy) return fail(HMY_E_INVALID, "logprob_bwd: d_entropy needs the rows' entropy");
  const void *words[] = {g.row_max, g.log_sum, g.targets, g.d_logp, g.entropy, g.d_entropy};
  for (const void *p : words)
    if (misaligned(p, 4)) return fail(HMY_E_INVALID, "logprob_bwd: misaligned array");
  const int el = bytes_of(g.logits_prec), ee = bytes_of(g.prec);
  if (rows_clash(g.logits, int64_t(g.V) * el, g.ldl * el, g.dlogits, (int64_t(g.V) + g.pad) * ee, g.ldd * ee, g.T, g.logits_prec == g.prec))
    return fail(HMY_E_INVALID, "logprob_bwd: dlogits overlaps logits other than in place");
  const LogprobGradArgs a = {g.row_max, g.log_sum, g.targets, g.d_logp, g.entropy, g.d_entropy, g.T, g.V, g.pad, g.ldl, g.ldd, g.scale};
  // one group of eight columns per thread while the row gives a workgroup of 64, 128 or 256 threads no more, two beyond: us, 8192
  // rows of 300 columns 5.3 on 64 threads, 9.0 on 256; of 1000 in bf16 8.5 on 128, 10.0 on 256
  const int nt = g.V <= 512 ? 64 : g.V <= 1024 ? 128 : 256, per_wg = 8 * nt * (g.V <= 2048 ? 1 : 2);
  const int tiles = (g.V + per_wg - 1) / per_wg;
  const int64_t n = int64_t(g.T) * tiles;
  const dim3 grid(uint32_t(n < kMaxGrid ? n : kMaxGrid));
  const hipStream_t s = (hipStream_t)st;
  DISPATCH_ROWS(g.logits_prec, g.prec, {
    const L *x = (const L *)g.logits;
    E *d = (E *)g.dlogits;
    if (nt == 64) hipLaunchKernelGGL((k_logprob_bwd<L, E, 64, 1>), grid, dim3(64), 0, s, x, d, a, tiles);
    else if (nt == 128) hipLaunchKernelGGL((k_logprob_bwd<L, E, 128, 1>), grid, dim3(128), 0, s, x, d, a, tiles);
    else if (g.V <= 2048) hipLaunchKernelGGL((k_logprob_bwd<L, E, 256, 1>), grid, dim3(256), 0, s, x, d, a, tiles);
    else hipLaunchKernelGGL((k_logprob_bwd<L, E, 256, 2>), grid, dim3(256), 0, s, x, d, a, tiles);
  });
  return check_launch("logprob_bwd");
}

}  // namespace hmy
