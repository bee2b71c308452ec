// The divergence of a student's rows of logits from a teacher's listed tokens, and its gradient.
//
// With u_j = s (x_j - m), S = sum exp u_j, l_j = u_j - log S, p_j = exp l_j, the teacher's q_k of listed tokens and, with a tail,
// q_r = 1 - sum q_k of all others together (the student's: p_r):
//   loss = sum q_k (log q_k - l_k) + q_r (log q_r - log p_r),  Q = sum q_k + q_r,
//   dloss/dz_j = Q p_j - q_j for listed tokens, p_j (Q - q_r / p_r) for the others (z = s x; without a tail q_r = 0, Q = 1).
// A divergence is small beside the logarithms that it is the difference of: the list's terms are held in 64 bits.  With a tail
// the row's sum is taken as that of the others (listed tokens are set to -inf where they are loaded) and that of the list, so
// that p_r of a student who is sure of listed tokens is no difference of two sums.  The others' sum and exponentials stay relative to
// their own largest logit: p_j / p_r is a quotient of numbers of ordinary size however little weight the class has.
#include <algorithm>

#include "logit_rows.h"

namespace hmy {

namespace {

struct DistillArgs {
  const int32_t *ids;
  const float *logp;
  float *row_loss;
  int T, V, K, pad;
  int64_t ldl, ldd;
  float scale, grad_scale;
  bool tail;
};

// A row's list, in LDS: written and read by one wave, entries lane and lane + 64 a lane's own.  An entry that names no token or
// has no weight is not there.
struct List {
  int id[HMY_MAX_TOP];      // -1: not there
  float t[HMY_MAX_TOP];     // the teacher's log probability
  float x[HMY_MAX_TOP];     // the student's logit
  double q[HMY_MAX_TOP];    // the teacher's probability, before it is divided by q_norm
  float gq[HMY_MAX_TOP];    // what the token's gradient is lowered by: grad_scale * scale * its q, all entries that name it together
};
// What the rest of the workgroup wants of it
struct ListSum {
  double q_sum, q_norm;   // sum of q_k, what they are divided by
  double sum;             // with a tail: sum over the tokens, each once, of exp(s (x - max))
  float t_max;            // q = exp(t - t_max) / q_norm
  float max;              // largest logit, -inf if there is none
  int any;
};

// exp in 64 bits on few registers: x = n ln 2 + r with |r| <= ln 2 / 2, Taylor's series up to r^11 (the next term is 6e-15, and with
// the terms behind it the whole error: 9e-15).  ln 2 is its nearest 64-bit number and what that leaves, 2.3e-17; a multiply-add
// rounds the exact product's difference once, so the first needs no zeros at its end.
__device__ __forceinline__ double exp64(double x) {
  x = x < -2000. ? -2000. : x;
  const double n = rint(x * 1.4426950408889634074), r = fma(n, -2.3190468138462996e-17, fma(n, -0.69314718055994530942, x));
  double p = 1. / 39916800.;
  p = fma(p, r, 1. / 3628800.);
  p = fma(p, r, 1. / 362880.);
  p = fma(p, r, 1. / 40320.);
  p = fma(p, r, 1. / 5040.);
  p = fma(p, r, 1. / 720.);
  p = fma(p, r, 1. / 120.);
  p = fma(p, r, 1. / 24.);
  p = fma(p, r, 1. / 6.);
  p = fma(p, r, 0.5);
  p = fma(p, r, 1.);
  p = fma(p, r, 1.);
  return ldexp(p, int(n));
}
// log of a positive number in 64 bits: y from the 32-bit logarithm, off by d < 1e-6, then d from x exp(-y) = exp d
__device__ __forceinline__ double log64(double x) {
  int e;
  const double f = frexp(x, &e), y = (double(__builtin_amdgcn_logf(float(f))) + double(e)) * 0.69314718055994530942;
  const double d = fma(x, exp64(-y), -1.);
  return y + fma(-0.5 * d, d, d);
}
__device__ __forceinline__ void lds_of_own_wave() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// this lane's two entries: the tokens, -1 where there is none, and the teacher's log probabilities
__device__ __forceinline__ void list_entries(const DistillArgs &a, int row, int lane, int (&id)[2], float (&tl)[2]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int k = lane + i * kWave;
    id[i] = -1;
    tl[i] = -INFINITY;
    if (k < a.K) {
      id[i] = a.ids[int64_t(row) * a.K + k];
      tl[i] = a.logp[int64_t(row) * a.K + k];
    }
    if (uint32_t(id[i]) >= uint32_t(a.V) || tl[i] == -INFINITY) id[i] = -1;
  }
}
// by one wave: the list and its sums
template <typename L>
__device__ __forceinline__ void read_list(const L *x, const DistillArgs &a, int lane, const int (&id)[2], const float (&tl)[2], List &l, ListSum &z) {
  float tm = -INFINITY, m = -INFINITY;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int k = lane + i * kWave;
    const float v = id[i] >= 0 ? to_f32(x[id[i]]) : -INFINITY;
    l.id[k] = id[i];
    l.t[k] = tl[i];
    l.x[k] = v;
    if (id[i] >= 0) tm = fmaxf(tm, tl[i]);
    m = fmaxf(m, v);
  }
  m = wave_top(m);
  tm = a.tail ? 0.f : wave_top(tm);
  if (tm == -INFINITY) tm = 0.f;
  lds_of_own_wave();
  const double ref = m == -INFINITY ? 0. : double(m), s = a.scale, w = s * double(a.grad_scale);
  double qs = 0., sum = 0.;
  bool any = false, again = false;
#pragma unroll 1
  for (int k = lane; k < a.K; k += kWave) {
    const int id = l.id[k];
    int same = 0;
#pragma unroll 2
    for (int o = 0; o < a.K; o += 4) {   // entries from K on are -1
      const int4 other = *reinterpret_cast<const int4 *>(l.id + o);
      same += (other.x == id) + (other.y == id) + (other.z == id) + (other.w == id);
    }
    bool first = id >= 0;
    if (first && same > 1) {
      again = true;
      for (int o = 0; o < k; ++o) first &= l.id[o] != id;
    }
    double q = 0.;
    if (id >= 0) {
      q = exp64(double(l.t[k]) - double(tm));
      if (first && a.tail) sum += exp64((double(l.x[k]) - ref) * s);
      any = true;
    }
    l.q[k] = q;
    qs += q;
  }
  qs = wave_total(qs);
  sum = wave_total(sum);
  const double inv = a.tail ? 1. : 1. / qs, lower = w * inv;
  lds_of_own_wave();
#pragma unroll 1
  for (int k = lane; k < a.K; k += kWave) {
    double q = l.q[k];
    if (__any(again)) {   // one token more than once: all of its q
      const int id = l.id[k];
      q = 0.;
      for (int o = 0; o < a.K; ++o)
        if (l.id[o] == id) q += l.q[o];
    }
    l.gq[k] = float(lower * q);
  }
  const bool any_there = __any(any);
  if (lane == 0) {
    z.q_sum = a.tail || qs != qs || !any_there ? qs : 1.;
    z.q_norm = a.tail ? 1. : qs;
    z.sum = sum;
    z.t_max = tm;
    z.max = m;
    z.any = any_there;
  }
}

// Whether the tokens that are not listed have any weight: exp(-745) is the least number of 64 bits.  One rule for loss and gradient.
// m_rest, rest: the sum of exp(s (x - m_rest)) over them (over all without a tail) and its reference, their largest logit, so that
// rest is at least 1 unless none of them has a logit above -inf; m: the row's largest logit
__device__ __forceinline__ bool others_weigh(float m_rest, float rest, float m, float scale) {
  return !(rest == 0.f) && !((double(m_rest) - double(m)) * double(scale) < -745.);
}
// What a row's gradient is made of once its sums are known
struct RowTerms {
  float m, c_list;        // the row's maximum, and what exp(s (x - m)) of a listed token is multiplied with
  float m_rest, c_rest;   // the others' maximum, and what exp(s (x - m_rest)) of any other is multiplied with
};                        // (maxima: 0 where nothing has any weight)
// The others' factor Q f / S - q_r / rest is a difference of nearly equal numbers where the student is near the teacher: it is formed
// in 64 bits, over a common denominator so that no division is (us with two of them / as it is, 8192 rows without a tail: 300 columns
// 14.3 / 13.9, 8000 columns 55.9 / 55.3).
__device__ __forceinline__ RowTerms row_terms(float m_rest, float rest, const ListSum &z, const DistillArgs &a) {
  const float m = a.tail ? fmaxf(m_rest, z.max) : m_rest, f = rebase(m_rest, m, a.scale);
  const double S = double(rest) * f + (a.tail ? z.sum * rebase(z.max, m, a.scale) : 0.);
  const double q_rest = a.tail && others_weigh(m_rest, rest, m, a.scale) ? fmax(1. - z.q_sum, 0.) : 0.;
  const float w = a.scale * a.grad_scale;
  const double Q = z.q_sum + q_rest;
  RowTerms r;
  r.m = m == -INFINITY ? 0.f : m;
  r.m_rest = m_rest == -INFINITY ? 0.f : m_rest;
  const float inv = S == 0. ? 0.f : 1.f / float(S);
  r.c_list = w * (float(Q) * inv);
  r.c_rest = q_rest > 0. ? w * (float(Q * (double(rest) * f) - q_rest * S) / float(double(rest) * S)) : r.c_list * f;
  return r;
}
// by one wave, the result in all lanes
__device__ __forceinline__ float row_loss(float m_rest, float rest, const List &l, const ListSum &z, const DistillArgs &a, int lane) {
  if (!z.any) return 0.f;
  const float m = a.tail ? fmaxf(m_rest, z.max) : m_rest;
  const double s = a.scale, mr = m == -INFINITY ? 0. : double(m);
  const double S_rest = m_rest == -INFINITY ? double(rest) : double(rest) * exp64((double(m_rest) - mr) * s);
  const double S = S_rest + (a.tail && z.max != -INFINITY ? z.sum * exp64((double(z.max) - mr) * s) : 0.);
  if (S == 0.) return z.q_sum > 0. ? INFINITY : 0.f;   // the student gives nothing any weight
  double loss = 0.;
#pragma unroll 1
  for (int k = lane; k < a.K; k += kWave) {
    const double q = l.q[k];
    if (!(q == 0.)) loss += q * ((double(l.t[k]) - double(z.t_max)) - (double(l.x[k]) - mr) * s);
  }
  loss = wave_total(loss);
  if (!a.tail) return float(loss / z.q_norm + log64(S / z.q_norm));
  loss += z.q_sum * log64(S);
  if (others_weigh(m_rest, rest, m, a.scale)) {
    const double q_rest = fmax(1. - z.q_sum, 0.);
    // p_r = exp(u) rest / S with u down to -745, where exp(u) keeps few bits: u is added outside of the logarithm
    if (q_rest > 0.) loss += q_rest * (log64(q_rest * (S / double(rest))) - (double(m_rest) - mr) * s);
  }
  return float(loss);
}

// Sets the listed tokens among a wave's own columns (groups g0 .. g1-1 of the row, dealt out over NT threads) to -inf: a wave looks
// for itself, with a bit in LDS for each of a thread's columns, and needs no barrier.  id: this lane's two entries.
template <int NT, int NG, typename L>
__device__ __forceinline__ void drop_listed(Eight<L> (&v)[NG], uint32_t *listed, const int (&id)[2], int g0, int g1, int wave) {
  constexpr int kWords = (NG + 3) / 4;
  const int tid = threadIdx.x;
#pragma unroll
  for (int w = 0; w < kWords; ++w) listed[w * NT + tid] = 0;
  lds_of_own_wave();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int off = id[i] / 8 - g0, owner = off % NT;
    if (id[i] >= 0 && off >= 0 && off < g1 - g0 && owner / kWave == wave) {
      const int slot = (off / NT) * 8 + id[i] % 8;
      atomicOr(&listed[(slot / 32) * NT + owner], 1u << (slot % 32));
    }
  }
  lds_of_own_wave();
#pragma unroll
  for (int w = 0; w < kWords; ++w) {
    const uint32_t bits = listed[w * NT + tid];
#pragma unroll
    for (int i = 4 * w; i < 4 * w + 4 && i < NG; ++i)
      if (bits >> (8 * (i % 4)) & 0xff) v[i].set_no_weight(bits >> (8 * (i % 4)));
  }
  lds_of_own_wave();   // the next columns' bits come behind the reads
}
// whether column `behind`, of the row's last V % 8, is listed: those are the first wave's
__device__ __forceinline__ bool is_listed_behind(const int (&id)[2], int V, int behind) {
  bool listed = false;
  for (int c = V / 8 * 8; c < V; ++c) {
    const bool any = __any(id[0] == c || id[1] == c);
    listed |= any && c == behind;
  }
  return listed;
}
// a thread's running maximum and sum of exp(s (x - m)) with more columns; HOLD: their exponentials stay in their place
template <bool HOLD, int NG, typename L>
__device__ __forceinline__ void add_columns(Eight<L> (&v)[NG], float xb, float &m, float &sum, float c) {
  float sm = fmaxf(m, xb);
#pragma unroll
  for (int i = 0; i < NG; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) sm = fmaxf(sm, v[i].at(k));
  const float ref = sm == -INFINITY ? 0.f : sm;
  sum *= fast_exp2((m - ref) * c);
  m = sm;
  sum += fast_exp2((xb - ref) * c);   // 0 for -inf
#pragma unroll
  for (int i = 0; i < NG; ++i) {
    v[i].forget_floats();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float e = fast_exp2((v[i].at(k) - ref) * c);
      sum += e;
      if constexpr (HOLD) v[i].w[k] = __float_as_uint(e);
    }
    v[i].forget_floats();
  }
}
// m and sum of a wave's lanes, the same for all of them
__device__ __forceinline__ void wave_sums(float &m, float &sum, float scale) {
  const float wm = wave_top(m);
  sum = wave_total(sum == 0.f ? 0.f : sum * rebase(m, wm, scale));
  m = wm;
}
// the same of a workgroup's first NT threads, for all of its threads
template <int NT>
__device__ __forceinline__ void block_sums(float &m, float &sum, float scale, float *scratch) {
  constexpr int kWaves = NT / kWave;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  wave_sums(m, sum, scale);
  if (lane == 0 && wave < kWaves) {
    scratch[wave] = m;
    scratch[kWaves + wave] = sum;
  }
  __syncthreads();
  m = lane < kWaves ? scratch[lane] : -INFINITY;
  sum = lane < kWaves ? scratch[kWaves + lane] : 0.f;
  wave_sums(m, sum, scale);
}
// gradient of one row's listed tokens, by one wave, behind the stores of the columns around them
template <typename E>
__device__ __forceinline__ void put_listed(E *d, const List &l, const RowTerms &r, const DistillArgs &a, int lane, int c0, int c1) {
#pragma unroll 1
  for (int k = lane; k < a.K; k += kWave)
    if (l.id[k] >= c0 && l.id[k] < c1) d[l.id[k]] = from_f32<E>(fmaf(rebase(l.x[k], r.m, a.scale), r.c_list, -l.gq[k]));
}

// One workgroup per row.  The row stays in registers between its sums and its gradient, as exponentials in fp32, as loaded in
// bf16; of a row beyond NT * NG groups of eight columns the last so many do, and those in front are read again.
// The list is the first wave's (short rows, of which many are at work at a time), or with LIST_WAVE one wave's more than the NT
// threads of the columns: the list is a chain of dependent loads and 64-bit arithmetic, and its wave's columns would wait for it.
// Bound by HBM, one reading and one writing, where there are rows for all compute units: 512 x 50257 fp32 into bf16 37 us (4.2
// TB/s: all of its rows are at work at once, two per compute unit, so that all read and then all write), 2048 x 50257 123 (5.0),
// 2048 x 131072 bf16 243 (4.4; one row per compute unit).  A few short rows: 6 us for 5003 columns, launch and one chain of
// latencies (ids, their logits, 64-bit sums, barrier, stores, barrier, the listed columns).  The loss alone takes the same way as far
// as the sums: 512 x 50257 fp32 21.3 us without a tail (4.8 TB/s), 22.7 with one; 2048 x 131072 bf16 116 (4.6) and 129.
template <typename L, typename E, int NT, int NG, bool TAIL, bool LIST_WAVE, int WPE>
__global__ __launch_bounds__(NT + (LIST_WAVE ? kWave : 0)) __attribute__((amdgpu_waves_per_eu(WPE))) void k_distill(const L *logits, E *dlogits, DistillArgs a) {
  constexpr int kSegment = NT * NG;
  constexpr bool kHold = sizeof(L) == 4;
  __shared__ uint32_t listed[TAIL ? NT * ((NG + 3) / 4) : 1];
  __shared__ float scratch[2 * NT / kWave];
  __shared__ ListSum z;
  __shared__ __attribute__((aligned(16))) List list;
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const bool lists = wave == (LIST_WAVE ? NT / kWave : 0), columns = !LIST_WAVE || !lists;
  const float c = a.scale * kLog2e;
  // segments of the row's groups: a short one first, if any, then whole ones, the last of which stays
  const int groups = a.V / 8, segments = max(1, (groups + kSegment - 1) / kSegment), lead = groups - (segments - 1) * kSegment;
  const int behind = groups * 8 + tid;   // this thread's column behind the groups, if it is less than V
  const int row = blockIdx.x;
  const L *x = logits + int64_t(row) * a.ldl;
  int id[2];
  float tl[2];
  if (TAIL || lists) list_entries(a, row, lane, id, tl);
  if (lists) read_list(x, a, lane, id, tl, list, z);
  Eight<L> v[NG];
  float xb = -INFINITY, m = -INFINITY, sum = 0.f;
  if (columns) {
    if (behind < a.V) xb = to_f32(x[behind]);
    if (TAIL && wave == 0 && is_listed_behind(id, a.V, behind)) xb = -INFINITY;
    for (int seg = 0; seg < segments; ++seg) {
      const int g0 = seg == 0 ? 0 : lead + (seg - 1) * kSegment, g1 = lead + seg * kSegment;
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        const int g = g0 + i * NT + tid;
        if (g < g1) load_whole(v[i], x + uint32_t(g) * 8);
        else v[i].all_no_weight();
      }
      if constexpr (TAIL) drop_listed<NT>(v, listed, id, g0, g1, wave);
      add_columns<kHold>(v, seg == 0 ? xb : -INFINITY, m, sum, c);
    }
  }
  float m_rest = m, rest = sum;
  block_sums<NT>(m_rest, rest, a.scale, scratch);
  if (dlogits) {
    E *d = dlogits + int64_t(row) * a.ldd;
    if (!z.any) {   // a row of padding: zeros whatever its logits are
      const float none[8] = {};
      if (columns) {
        for (int g = tid; g < groups; g += NT) store_whole(d + uint32_t(g) * 8, none);
        if (behind < a.V) d[behind] = from_f32<E>(0.f);
        zero_padding(d, a.V, a.pad, tid, NT);
      }
      if (tid == 0) a.row_loss[row] = 0.f;
      return;
    }
    const RowTerms r = row_terms(m_rest, rest, z, a);
    if (columns) {
      const float mine = r.c_rest * rebase(m, r.m_rest, a.scale);
      // (listed tokens may come out as anything: theirs is stored behind)
      auto grad = [&](float xj) { return fast_exp2((xj - r.m_rest) * c) * r.c_rest; };
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        const int g = (segments == 1 ? 0 : lead + (segments - 2) * kSegment) + i * NT + tid;
        if (g < groups) {
          float o[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) o[k] = kHold ? v[i].at(k) * mine : grad(v[i].at(k));
          store_whole(d + uint32_t(g) * 8, o);
        }
      }
      if (behind < a.V) d[behind] = from_f32<E>(grad(xb));
      for (int seg = segments - 2; seg >= 0; --seg) {
        const int g0 = seg == 0 ? 0 : lead + (seg - 1) * kSegment, g1 = lead + seg * kSegment;
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          const int g = g0 + i * NT + tid;
          if (g < g1) load_whole(v[i], x + uint32_t(g) * 8);
        }
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          const int g = g0 + i * NT + tid;
          if (g < g1) {
            float o[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] = grad(v[i].at(k));
            store_whole(d + uint32_t(g) * 8, o);
          }
        }
      }
      zero_padding(d, a.V, a.pad, tid, NT);
    }
    if (LIST_WAVE && lists) {   // while the others store
      const float loss = row_loss(m_rest, rest, list, z, a, lane);
      if (lane == 0) a.row_loss[row] = loss;
    }
    __syncthreads();   // behind the stores of the columns around
    if (lists) put_listed(d, list, r, a, lane, 0, a.V);
  }
  if (lists && !(LIST_WAVE && dlogits)) {
    const float loss = row_loss(m_rest, rest, list, z, a, lane);
    if (lane == 0) a.row_loss[row] = loss;
  }
}

// Few, long rows: workgroups each take `groups` of a row's groups of eight columns, once for the row's sums and once, in a second
// launch, for the gradient.  The list is the first part's.
struct RowParts {
  ListSum *z;        // [rows]
  List *list;        // [rows]
  float2 *sums;      // [rows * per_row]: maximum, sum relative to it
  int per_row, groups;
};
constexpr int kPartThreads = 512;

template <typename L, int NG, bool TAIL>
__global__ __launch_bounds__(kPartThreads) void k_distill_parts(const L *logits, DistillArgs a, RowParts p) {
  constexpr int NT = kPartThreads;
  __shared__ uint32_t listed[TAIL ? NT * ((NG + 3) / 4) : 1];
  __shared__ float scratch[2 * NT / kWave];
  __shared__ ListSum z;
  __shared__ __attribute__((aligned(16))) List list;
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int row = blockIdx.x / p.per_row, piece = blockIdx.x % p.per_row;
  const float c = a.scale * kLog2e;
  const L *x = logits + int64_t(row) * a.ldl;
  const int first = piece * p.groups, last = min(first + p.groups, a.V / 8), behind = a.V / 8 * 8 + tid;
  int id[2];
  float tl[2];
  list_entries(a, row, lane, id, tl);
  float xb = piece == p.per_row - 1 && behind < a.V ? to_f32(x[behind]) : -INFINITY, m = -INFINITY, sum = 0.f;
  if (TAIL && wave == 0 && is_listed_behind(id, a.V, behind)) xb = -INFINITY;
  Eight<L> v[NG];
  for (int g0 = first; g0 < last; g0 += NT * NG) {
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      if (g0 + i * NT + tid < last) load_whole(v[i], x + uint32_t(g0 + i * NT + tid) * 8);
      else v[i].all_no_weight();
    }
    if constexpr (TAIL) drop_listed<NT>(v, listed, id, g0, min(g0 + NT * NG, last), wave);
    add_columns<false>(v, -INFINITY, m, sum, c);
  }
  if (xb > -INFINITY || xb != xb) {
    const float sm = fmaxf(m, xb), ref = sm == -INFINITY ? 0.f : sm;
    sum = sum * fast_exp2((m - ref) * c) + fast_exp2((xb - ref) * c);
    m = sm;
  }
  block_sums<NT>(m, sum, a.scale, scratch);
  if (tid == 0) p.sums[blockIdx.x] = make_float2(m, sum);
  if (piece == 0 && wave == 0) {
    read_list(x, a, lane, id, tl, list, z);
    lds_of_own_wave();
    for (int i = lane; i < int(sizeof(List) / 4); i += kWave) reinterpret_cast<uint32_t *>(p.list + row)[i] = reinterpret_cast<const uint32_t *>(&list)[i];
    if (lane == 0) p.z[row] = z;
  }
}
template <typename L, typename E>
__global__ __launch_bounds__(kPartThreads) void k_distill_finish(const L *logits, E *dlogits, DistillArgs a, RowParts p) {
  constexpr int NT = kPartThreads, NG = 2;
  const int tid = threadIdx.x, lane = tid % kWave;
  const int row = blockIdx.x / p.per_row, piece = blockIdx.x % p.per_row;
  const float2 part = lane < p.per_row ? p.sums[row * p.per_row + lane] : make_float2(-INFINITY, 0.f);   // per_row <= 64
  float m_rest = part.x, rest = part.y;
  wave_sums(m_rest, rest, a.scale);
  const ListSum z = p.z[row];
  if (dlogits) {
    const RowTerms r = row_terms(m_rest, rest, z, a);
    const float c = a.scale * kLog2e;
    auto grad = [&](float xj) { return z.any ? fast_exp2((xj - r.m_rest) * c) * r.c_rest : 0.f; };
    const L *x = logits + int64_t(row) * a.ldl;
    E *d = dlogits + int64_t(row) * a.ldd;
    const int first = piece * p.groups, last = min(first + p.groups, a.V / 8);
    for (int g0 = first + tid; g0 < last; g0 += NT * NG) {
      Eight<L> v[NG];
#pragma unroll
      for (int i = 0; i < NG; ++i)
        if (g0 + i * NT < last) load_whole(v[i], x + uint32_t(g0 + i * NT) * 8);
#pragma unroll
      for (int i = 0; i < NG; ++i)
        if (g0 + i * NT < last) {
          float o[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) o[k] = grad(v[i].at(k));
          store_whole(d + uint32_t(g0 + i * NT) * 8, o);
        }
    }
    const bool ends = piece == p.per_row - 1;
    const int behind = a.V / 8 * 8 + tid;
    if (ends) {
      if (behind < a.V) d[behind] = from_f32<E>(grad(to_f32(x[behind])));
      zero_padding(d, a.V, a.pad, tid, NT);
    }
    __syncthreads();   // behind the stores of the columns around
    if (tid < kWave) put_listed(d, p.list[row], r, a, lane, first * 8, ends ? a.V : last * 8);
  }
  if (piece == 0 && tid < kWave) {
    const float loss = row_loss(m_rest, rest, p.list[row], z, a, lane);
    if (lane == 0) a.row_loss[row] = loss;
  }
}

// loss[0] += scale * the sum of the rows' losses, in one order whatever the launch; calls on other streams may add to it meanwhile
// One workgroup: 2.2 us of 24 rows, 2.4 of 2048, 4 of 8192, 270 of a million, whose other work takes 980 (with one load of each of 256
// threads at a time 3, 3.4, 9.4 and 1070).
constexpr int kSumThreads = 1024, kSumFlight = 8;   // loads on their way at a time, of a thread
__global__ __launch_bounds__(kSumThreads) void k_loss_sum(const float *row_loss, double *loss, int T, double scale) {
  __shared__ double scratch[kSumThreads / kWave];
  double v = 0.;
  for (int64_t first = threadIdx.x; first < T; first += kSumThreads * kSumFlight) {
    float x[kSumFlight];
#pragma unroll
    for (int o = 0; o < kSumFlight; ++o) x[o] = first + o * kSumThreads < T ? row_loss[first + o * kSumThreads] : 0.f;
#pragma unroll
    for (int o = 0; o < kSumFlight; ++o) v += double(x[o]);
  }
  v = wave_total(v);
  if (threadIdx.x % kWave == 0) scratch[threadIdx.x / kWave] = v;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kSumThreads / kWave; ++w) v += scratch[w];
    atomicAdd(loss, v * scale);
  }
}

template <typename L, typename E, int NT, int NG, bool LIST_WAVE, int WPE>
void launch_rows(const L *x, E *d, DistillArgs a, hipStream_t s) {
  for (int rows = a.T; rows > 0; rows -= kMaxGrid) {   // a launch has a limited number of workgroups
    const dim3 grid(rows < kMaxGrid ? rows : kMaxGrid), block(NT + (LIST_WAVE ? kWave : 0));
    if (a.tail) hipLaunchKernelGGL((k_distill<L, E, NT, NG, true, LIST_WAVE, WPE>), grid, block, 0, s, x, d, a);
    else hipLaunchKernelGGL((k_distill<L, E, NT, NG, false, LIST_WAVE, WPE>), grid, block, 0, s, x, d, a);
    x += int64_t(kMaxGrid) * a.ldl;
    if (d) d += int64_t(kMaxGrid) * a.ldd;
    a.ids += int64_t(kMaxGrid) * a.K;
    a.logp += int64_t(kMaxGrid) * a.K;
    a.row_loss += kMaxGrid;
  }
}

constexpr int kPartRows = 64, kPartLaunch = 512, kPartMinCols = 16384, kPartsMax = 64;
static_assert(kPartRows * (sizeof(List) + sizeof(ListSum)) + kPartLaunch * sizeof(float2) <= HMY_ROWS_WORKSPACE_BYTES, "the parts' sums and the lists fit the workspace");

template <typename L, typename E>
void launch_parts(const L *x, E *d, const DistillArgs &a, int parts, void *workspace, hipStream_t s) {
  RowParts p;
  p.groups = (a.V / 8 + parts - 1) / parts;
  p.per_row = (a.V / 8 + p.groups - 1) / p.groups;
  p.list = static_cast<List *>(workspace);
  p.z = reinterpret_cast<ListSum *>(p.list + a.T);
  p.sums = reinterpret_cast<float2 *>(p.z + a.T);
  const dim3 grid(a.T * p.per_row);
  constexpr int NG = sizeof(L) == 4 ? 2 : 4;
  if (a.tail) hipLaunchKernelGGL((k_distill_parts<L, NG, true>), grid, dim3(kPartThreads), 0, s, x, a, p);
  else hipLaunchKernelGGL((k_distill_parts<L, NG, false>), grid, dim3(kPartThreads), 0, s, x, a, p);
  hipLaunchKernelGGL((k_distill_finish<L, E>), grid, dim3(kPartThreads), 0, s, x, d, a, p);
}

}  // namespace

int launch_distill(const hmy_distill_desc &g, stream_t st) {
  int rc = check_rows("distill", g.logits_prec, g.logits, g.T, g.V, 0, g.ldl);
  if (!rc && g.dlogits) rc = check_rows("distill", g.prec, g.dlogits, g.T, g.V, g.pad, g.ldd);
  if (rc) return rc;
  if (!usable_scale(g.scale)) return fail(HMY_E_INVALID, "distill: the scale must be positive and finite");
  if (!std::isfinite(g.scale * g.grad_scale)) return fail(HMY_E_INVALID, "distill: the gradient's scale, and its product with the logits', must be finite");
  if (g.K < 1 || g.K > HMY_MAX_TOP) return fail(HMY_E_INVALID, "distill: K = %d is not in 1..%d", g.K, HMY_MAX_TOP);
  if (g.tail != 0 && g.tail != 1) return fail(HMY_E_INVALID, "distill: tail is 0 or 1");
  const void *words[] = {g.teacher_ids, g.teacher_logp, g.row_loss};
  for (const void *p : words)
    if (misaligned(p, 4)) return fail(HMY_E_INVALID, "distill: misaligned array");
  if (misaligned(g.loss_acc, 8)) return fail(HMY_E_INVALID, "distill: misaligned loss_acc");
  const int el = bytes_of(g.logits_prec), ee = bytes_of(g.prec);
  if (g.dlogits && rows_clash(g.logits, int64_t(g.V) * el, g.ldl * el, g.dlogits, (int64_t(g.V) + g.pad) * ee, g.ldd * ee, g.T, g.logits_prec == g.prec))
    return fail(HMY_E_INVALID, "distill: dlogits overlaps logits other than in place");
  const DistillArgs a = {g.teacher_ids, g.teacher_logp, g.row_loss, g.T, g.V, g.K, g.pad, g.ldl, g.ldd, g.scale, g.grad_scale, g.tail == 1};
  const hipStream_t s = (hipStream_t)st;
  void *ws = has_workspace(g.workspace, g.workspace_bytes) ? g.workspace : nullptr;
  if (misaligned(ws, 16)) return fail(HMY_E_INVALID, "distill: workspace not aligned to 16 bytes");
  const int parts = ws && g.T <= kPartRows ? std::min(std::min(kPartLaunch / g.T, kPartsMax), g.V / kPartMinCols) : 1;
  DISPATCH_ROWS(g.logits_prec, g.prec, {
    const L *x = (const L *)g.logits;
    E *d = (E *)g.dlogits;
    // As few waves as hold the row in up to four groups of eight columns a thread, while a workgroup has at most 256 threads: the
    // first wave's work on the list, which the others wait for, is then a smaller part (us, 8192 rows of 1000 columns in bf16 on
    // 64, 128, 256 threads: 19.5, 25, 36; the floor is 6.5).  Beyond, what a compute unit's registers hold of rows, two at a
    // time as far as they fit: 448 threads and a list wave (20000 columns 83, on 512 threads without one 90; the floor is 81), in
    // bf16 1024 threads of 64 registers although a part of the row is read twice then (80000 columns 102, on 110 registers
    // 110), and only beyond 110000 one row at a time (131072 columns 230 against 246).
    // fp32 rows of 25089 to 32768 columns stay there although their first columns, beyond 448 x 7 groups, are read twice; us so / on
    // 1024 threads without a list wave, a tail in fp32: 30522 columns, 6 rows 8.6 / 8.8, 256 15.7 / 15.9, 512 29.1 / 34.6, 3372 176 /
    // 183; 32768 columns, 512 rows 30.9 / 35.1, 3372 186 / 187 (into bf16 without a tail 133 / 129); 36000 columns, 3372 rows 211 / 206.
    // Few rows by parts, two launches, from four parts on, which read twice but on the whole device.  us by parts / by rows, fp32:
    // one row of 131072 columns 10.2 / 23.5, 64 rows of 80000 17.4 / 19.6, but 128 rows 25.6 / 21.6.
    constexpr bool wide = sizeof(L) == 4;
    if (parts >= 4) launch_parts(x, d, a, parts, ws, s);
    else if (g.V <= 512) launch_rows<L, E, 64, 1, false, 4>(x, d, a, s);
    else if (g.V <= 2048) launch_rows<L, E, 64, 4, false, 4>(x, d, a, s);
    else if (g.V <= 4096) launch_rows<L, E, 128, 4, false, 4>(x, d, a, s);
    else if (g.V <= 8192) launch_rows<L, E, 256, 4, false, 4>(x, d, a, s);
    else if (g.V <= 14336) launch_rows<L, E, 256, 7, false, 4>(x, d, a, s);
    else if (g.V <= (wide ? 32768 : 25088)) launch_rows<L, E, 448, 7, true, 4>(x, d, a, s);
    else if (wide) launch_rows<L, E, 1024, 7, false, 4>(x, d, a, s);
    else if (g.V <= 35840) launch_rows<L, E, 448, wide ? 7 : 10, true, 4>(x, d, a, s);
    else if (g.V <= 50176) launch_rows<L, E, 448, wide ? 7 : 14, true, 4>(x, d, a, s);
    else if (g.V <= 110000) launch_rows<L, E, 1024, 7, false, wide ? 4 : 8>(x, d, a, s);
    else launch_rows<L, E, 1024, wide ? 7 : 16, false, 4>(x, d, a, s);
  });
  if (g.loss_acc)
    hipLaunchKernelGGL(k_loss_sum, dim3(1), dim3(kSumThreads), 0, s, g.row_loss, g.loss_acc, g.T, double(g.grad_scale));
  return check_launch("distill");
}

}  // namespace hmy
