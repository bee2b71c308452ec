// Operators on rows of logits x[T,V]: log probabilities of given tokens with entropy and the most likely tokens, and their
// gradient.
//
// With the scale s, m = max x, u_j = s (x_j - m), S = sum exp u_j:  log p_j = u_j - log S,
//   H = log S - (sum u_j exp u_j) / S.
// u is taken from the difference to the maximum, so rows of the type's lowest value, or of very large values, lose nothing; a
// token at -inf has no weight (0 times its u counts as 0), a row of nothing else has m = -inf and S = 0.
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

// Candidates for a row's list, in LDS.  What is not among them is outranked by at least k that are.
constexpr int kCandidates = 2048;
constexpr int kRanked = 512;       // as many are ranked by comparing all with all
template <int NT> struct Candidates {
  uint64_t key[kCandidates];
  uint32_t group[NT];              // maxima of the threads' columns
  uint32_t n, floor, count[2];     // floor: `ordered` of the least logit that can still be among the k
};

// by one wave: some t with at least k of the values at or above it, and not many more if it can be had: the bisection ends at
// k + k / 8 + 2.  kLowestOrdered if fewer than k are at or above that.
template <int P>
__device__ __forceinline__ uint32_t threshold(const uint32_t (&v)[P], int k) {
  auto count = [&](uint32_t t) {
    int c = 0;
#pragma unroll
    for (int i = 0; i < P; ++i) c += __popcll(__ballot(v[i] >= t));
    return c;
  };
  if (count(kLowestOrdered) < k) return kLowestOrdered;
  uint32_t lo = ~0u, hi = 0;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    hi = max(hi, v[i]);
    if (v[i] >= kLowestOrdered) lo = min(lo, v[i]);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    hi = max(hi, uint32_t(__shfl_xor(int(hi), o, kWave)));
    lo = min(lo, uint32_t(__shfl_xor(int(lo), o, kWave)));
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);   // at or above lo: at least k; above hi: none
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
template <int NT>
__device__ __forceinline__ int hits(Candidates<NT> &c, int mine, int &turn) {
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

// by the workgroup: leaves only candidates that the k largest can be among, at most `most` of them.  Barriers on both sides.
template <int NT>
__device__ __forceinline__ void thin_out(Candidates<NT> &c, int k, int most, int &turn) {
  constexpr int P = kCandidates / 2 / kWave, PT = (kCandidates + NT - 1) / NT;
  const int tid = threadIdx.x, n = min(int(c.n), kCandidates);
  if (n <= k) return;
  uint64_t mine[PT], least = 0;
#pragma unroll
  for (int i = 0; i < PT; ++i) mine[i] = tid + i * NT < n ? c.key[tid + i * NT] : 0;
  if (n <= P * kWave) {
    if (tid < kWave) {
      uint32_t v[P];
#pragma unroll
      for (int i = 0; i < P; ++i) v[i] = tid + i * kWave < n ? uint32_t(c.key[tid + i * kWave] >> 32) : 0;
      const uint32_t t = threshold(v, k);
      if (tid == 0) c.floor = t;
    }
    __syncthreads();
    least = uint64_t(c.floor) << 32;
    int kept = 0;
#pragma unroll
    for (int i = 0; i < PT; ++i) kept += mine[i] >= least && mine[i];
    if (hits<NT>(c, kept, turn) > most) least = 0;   // many equal logits
  }
  if (least == 0) {   // the k-th largest key itself, bit by bit
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t t = least | uint64_t(1) << bit;
      int above = 0;
#pragma unroll
      for (int i = 0; i < PT; ++i) above += mine[i] >= t;
      if (hits<NT>(c, above, turn) >= k) least = t;
    }
    if (tid == 0) c.floor = max(uint32_t(least >> 32), kLowestOrdered);
  }
  __syncthreads();
  if (tid == 0) c.n = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PT; ++i)
    if (mine[i] && mine[i] >= least) c.key[atomicAdd(&c.n, 1u)] = mine[i];
  __syncthreads();
}

// by the workgroup: the k first of the candidates, `put(rank, key)` for each; barriers in front
template <int NT, typename F>
__device__ __forceinline__ void rank_candidates(Candidates<NT> &c, int k, int &turn, F put) {
  if (int(c.n) > 2 * k + 64) thin_out<NT>(c, k, kRanked, turn);
  const int n = int(c.n), tid = threadIdx.x;
  for (int i = tid; i < n; i += NT) {
    const uint64_t mine = c.key[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += c.key[j] > mine;
    if (rank < k) put(rank, mine);
  }
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
__device__ __forceinline__ void put_row(const LogprobArgs &a, int row, const Sums &z, float target_logit, bool has_target) {
  const float log_sum = logf(z.S), ref = z.m == -INFINITY ? 0.f : z.m;
  if (a.logp) a.logp[row] = !has_target ? 0.f : z.S == 0.f ? -INFINITY : (target_logit - ref) * a.scale - log_sum;
  if (a.row_max) a.row_max[row] = z.m;
  if (a.log_sum) a.log_sum[row] = log_sum;
  if (a.entropy) a.entropy[row] = z.S == 0.f ? 0.f : log_sum - z.A * kLn2 / z.S;
}

// One workgroup per row, NT * NG groups of eight columns at a time, the next ones' loads on their way meanwhile.  One reading
// of the row: each thread keeps a running maximum and sums relative to it.  The list: the first columns give a floor that at
// least k of them reach (a bisection over the maxima of 256 groups of threads), from then on only what reaches the floor is
// looked at; the candidates are thinned out, and the floor raised, when there are many.
template <typename L, int NT, int NG, bool TOP>
__global__ __launch_bounds__(NT) void k_logprob(const L *logits, LogprobArgs a) {
  constexpr int kWaves = NT / kWave, kSegment = NT * NG;
  __shared__ Sums part[kWaves];
  __shared__ Candidates<TOP ? NT : 1> cand_;
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave), row = blockIdx.x;
  const float c = a.scale * kLog2e;
  const L *x = logits + int64_t(row) * a.ldl;
  const int groups = a.V / 8, segments = (groups + kSegment - 1) / kSegment;
  const int tgt = a.targets ? a.targets[row] : -1;
  const bool has_target = tgt >= 0 && tgt < a.V;
  const float target_logit = has_target ? to_f32(x[tgt]) : 0.f;
  Sums z = no_sums();
  int turn = 0;
  if constexpr (TOP) {
    if (tid == 0) {
      cand_.n = cand_.count[0] = cand_.count[1] = 0;
      cand_.floor = 0;
    }
    __syncthreads();
  }
  auto load = [&](Eight<L> (&v)[NG], int seg) {
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const int g = seg * kSegment + i * NT + tid;
      if (g < groups) load_whole(v[i], x + uint32_t(g) * 8);
      else v[i].all_no_weight();
    }
  };
  auto take = [&](Eight<L> (&v)[NG], int seg) {
    float top[NG], sm = z.m;
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      top[i] = v[i].at(0);
#pragma unroll
      for (int k = 1; k < 8; ++k) top[i] = fmaxf(top[i], v[i].at(k));
      sm = fmaxf(sm, top[i]);
      v[i].forget_floats();
    }
    if (sm > z.m) {
      const float d = fmaxf((z.m - sm) * c, kNoWeight), f = fast_exp2(d);
      z.A = f * fmaf(d, z.S, z.A);
      z.S *= f;
      z.m = sm;
    }
    const float ref = sm == -INFINITY ? 0.f : sm;
#pragma unroll
    for (int i = 0; i < NG; ++i) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float u = (v[i].at(k) - ref) * c, e = fast_exp2(u);
        z.S += e;
        z.A = fmaf(e, fmaxf(u, kNoWeight), z.A);
      }
      v[i].forget_floats();
    }
    if constexpr (TOP) {
      auto &cand = cand_;
      if (seg == 0) {
        float mine = top[0];
#pragma unroll
        for (int i = 1; i < NG; ++i) mine = fmaxf(mine, top[i]);
        cand.group[tid] = ordered(mine);
        __syncthreads();
        if (wave == 0) {
          uint32_t g[4] = {0, 0, 0, 0};
#pragma unroll
          for (int i = 0; i < NT / kWave; ++i) g[i % 4] = max(g[i % 4], cand.group[lane + i * kWave]);
          const uint32_t t = threshold(g, a.k);
          if (lane == 0) cand.floor = t;
        }
        __syncthreads();
      }
      const int before = int(cand.n);
      const float floor = unordered(__builtin_amdgcn_readfirstlane(cand.floor));
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NG; ++i)
        if (top[i] >= floor) {
          const int col = (seg * kSegment + i * NT + tid) * 8;
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (v[i].at(k) >= floor) {
              const uint32_t at = atomicAdd(&cand.n, 1u);
              if (at < kCandidates) cand.key[at] = rank_key(v[i].at(k), col + k);
            }
        }
      __syncthreads();
      const int n = int(cand.n);
      if (n > kCandidates) {
        // too many to keep (the largest logits are those of few threads, or very many are equal): the k-th largest of these
        // columns, bit by bit, and of those that equal it the lowest columns
        uint32_t t = 0;
        for (int bit = 31; bit >= 0; --bit) {
          const float f = unordered(t | 1u << bit);
          const bool can = (t | 1u << bit) >= kLowestOrdered;
          int above = 0;
#pragma unroll
          for (int i = 0; i < NG; ++i)
#pragma unroll
            for (int k = 0; k < 8; ++k) above += can ? v[i].at(k) >= f : v[i].at(k) > -INFINITY;
          if (hits<TOP ? NT : 1>(cand, above, turn) >= a.k) t |= 1u << bit;
        }
        t = max(t, kLowestOrdered);
        const float f = unordered(t);
        int above = 0;
#pragma unroll
        for (int i = 0; i < NG; ++i)
#pragma unroll
          for (int k = 0; k < 8; ++k) above += v[i].at(k) > f;
        const int want = a.k - hits<TOP ? NT : 1>(cand, above, turn);   // of those that equal f
        int last = 0;                                        // how many columns from this segment's first on
        for (int bit = 31 - __builtin_clz(kSegment * 8); bit >= 0; --bit) {
          const int to = last | 1 << bit;
          int equal = 0;
#pragma unroll
          for (int i = 0; i < NG; ++i)
#pragma unroll
            for (int k = 0; k < 8; ++k) equal += v[i].at(k) == f && (i * NT + tid) * 8 + k < to;
          if (hits<TOP ? NT : 1>(cand, equal, turn) <= want) last = to;
        }
        if (tid == 0) cand.n = before;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NG; ++i)
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const int off = (i * NT + tid) * 8 + k;
            if (v[i].at(k) > f || (v[i].at(k) == f && off < last))
              cand.key[atomicAdd(&cand.n, 1u)] = rank_key(v[i].at(k), seg * kSegment * 8 + off);
          }
        __syncthreads();
      }
      if (int(cand.n) > kCandidates / 4) thin_out<TOP ? NT : 1>(cand, a.k, kRanked, turn);
    }
  };
  Eight<L> v[NG], w[NG];
  if (segments > 0) load(v, 0);
  for (int seg = 0; seg < segments; seg += 2) {
    if (seg + 1 < segments) load(w, seg + 1);
    take(v, seg);
    if (seg + 1 < segments) {
      if (seg + 2 < segments) load(v, seg + 2);
      take(w, seg + 1);
    }
  }
  // the columns behind the groups
  const int behind = groups * 8 + tid;
  if (behind < a.V) {
    const float xb = to_f32(x[behind]);
    if (xb > z.m) {
      const float d = fmaxf((z.m - xb) * c, kNoWeight), f = fast_exp2(d);
      z.A = f * fmaf(d, z.S, z.A);
      z.S *= f;
      z.m = xb;
    }
    const float u = (xb - (z.m == -INFINITY ? 0.f : z.m)) * c, e = fast_exp2(u);
    z.S += e;
    z.A = fmaf(e, fmaxf(u, kNoWeight), z.A);
    if constexpr (TOP) {
      if (xb > -INFINITY) cand_.key[atomicAdd(&cand_.n, 1u)] = rank_key(xb, behind);   // at most seven more
    }
  }
  const Sums ws = wave_sums(z, a.scale);
  if (lane == 0) part[wave] = ws;
  __syncthreads();
  Sums all = lane < kWaves ? part[lane] : no_sums();
  all = wave_sums(all, a.scale);
  if (tid == 0) put_row(a, row, all, target_logit, has_target);
  if constexpr (TOP) {
    const float log_sum = logf(all.S);
    rank_candidates<TOP ? NT : 1>(cand_, a.k, turn, [&](int rank, uint64_t key) {
      a.top_ids[int64_t(row) * a.k + rank] = key ? key_column(key) : -1;
      a.top_logp[int64_t(row) * a.k + rank] = key ? (unordered(uint32_t(key >> 32)) - all.m) * a.scale - log_sum : -INFINITY;
    });
  }
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
// before its first store.  us (TB/s), rows x columns, U = 1 / 2 / 4: fp32 into bf16, 512 x 50257 31.2 / 30.7 (5.0) / 32.6; bf16,
// 1111 x 131071 134 / 112 (5.2) / 114, x 131072 119 / 105 (5.5) / 106: rows that start off any alignment cost 6 %.  A large copy
// runs at 5.06.
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

template <typename L, int NT, int NG>
void launch_rows(const L *x, LogprobArgs a, int rows, hipStream_t s) {
  for (; rows > 0; rows -= kMaxGrid) {   // a launch has a limited number of workgroups
    const dim3 grid(rows < kMaxGrid ? rows : kMaxGrid);
    if (a.k) hipLaunchKernelGGL((k_logprob<L, NT, NG, true>), grid, dim3(NT), 0, s, x, a);
    else hipLaunchKernelGGL((k_logprob<L, NT, NG, false>), grid, dim3(NT), 0, s, x, a);
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
template <typename L>
void launch_rows(const L *x, const LogprobArgs &a, int rows, hipStream_t s) {
  if (a.V <= 16384) launch_rows<L, 256, 2>(x, a, rows, s);
  else launch_rows<L, 1024, 2>(x, a, rows, s);
}

}  // namespace

int launch_logprob(const hmy_logprob_desc &g, stream_t st) {
  int rc = check_rows("logprob", g.logits_prec, g.logits, g.T, g.V, 0, g.ldl);
  if (rc) return rc;
  if (!positive(g.scale)) return fail(HMY_E_INVALID, "logprob: the scale must be positive and finite");
  if (g.k < 0 || g.k > HMY_MAX_TOP) return fail(HMY_E_INVALID, "logprob: k = %d is not in 0..%d", g.k, HMY_MAX_TOP);
  if (g.k > 0 && (!g.top_ids || !g.top_logp)) return fail(HMY_E_INVALID, "logprob: k > 0 needs top_ids and top_logp");
  if (!g.targets != !g.logp) return fail(HMY_E_INVALID, "logprob: targets and logp come together");
  if (!g.logp && !g.row_max && !g.log_sum && !g.entropy && !g.k) return fail(HMY_E_INVALID, "logprob: no output asked for");
  const void *words[] = {g.targets, g.logp, g.row_max, g.log_sum, g.entropy, g.top_ids, g.top_logp};
  for (const void *p : words)
    if (misaligned(p, 4)) return fail(HMY_E_INVALID, "logprob: misaligned array");
  const LogprobArgs a = {g.targets, g.logp, g.row_max, g.log_sum, g.entropy, g.top_ids, g.top_logp, g.V, g.k, g.ldl, g.scale};
  const hipStream_t s = (hipStream_t)st;
  if (g.logits_prec == HMY_PREC_BF16) launch_rows((const bf16_t *)g.logits, a, g.T, s);
  else launch_rows((const float *)g.logits, a, g.T, s);
  return check_launch("logprob");
}

int launch_logprob_bwd(const hmy_logprob_grad_desc &g, stream_t st) {
  int rc = check_rows("logprob_bwd", g.logits_prec, g.logits, g.T, g.V, 0, g.ldl);
  if (!rc) rc = check_rows("logprob_bwd", g.prec, g.dlogits, g.T, g.V, g.pad, g.ldd);
  if (rc) return rc;
  if (!positive(g.scale)) return fail(HMY_E_INVALID, "logprob_bwd: the scale must be positive and finite");
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
  // one group of eight columns per thread while the row gives a workgroup of 64, 128 or 256 threads no more, two beyond
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
