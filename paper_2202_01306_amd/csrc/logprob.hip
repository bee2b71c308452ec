// Operators on rows of logits x[T,V]: log probabilities of given tokens with entropy and the most likely tokens, their
// gradient, and the divergence from a teacher's listed tokens with its gradient.
//
// With the scale s, m = max x, u_j = s (x_j - m), S = sum exp u_j:  log p_j = u_j - log S,
//   H = log S - (sum u_j exp u_j) / S.
// u is taken from the difference to the maximum, so rows of the type's lowest value, or of very large values, lose nothing; a
// token at -inf has no weight (0 times its u counts as 0), a row of nothing else has m = -inf and S = 0.
#include <cmath>

#include "dev_common.h"
#include "hmy_internal.h"

namespace hmy {

namespace {

constexpr int kRowThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// below this (log2 units) an exponential is 0 and so is its product with its exponent, which may be -inf
constexpr float kNoWeight = -1e4f;

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

template <int NT>
__device__ __forceinline__ float block_sum(float v, float *scratch) {
  v = wave_sum(v);
  __syncthreads();
  if (threadIdx.x % kWave == 0) scratch[threadIdx.x / kWave] = v;
  __syncthreads();
  float r = 0.f;
#pragma unroll
  for (int w = 0; w < NT / kWave; ++w) r += scratch[w];
  return r;
}
template <int NT>
__device__ __forceinline__ float block_max(float v, float *scratch) {
  v = wave_max(v);
  __syncthreads();
  if (threadIdx.x % kWave == 0) scratch[threadIdx.x / kWave] = v;
  __syncthreads();
  float r = scratch[0];
#pragma unroll
  for (int w = 1; w < NT / kWave; ++w) r = fmaxf(r, scratch[w]);
  return r;
}
template <int NT>
__device__ __forceinline__ double block_sum(double v, double *scratch) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  __syncthreads();
  if (threadIdx.x % kWave == 0) scratch[threadIdx.x / kWave] = v;
  __syncthreads();
  double r = 0.;
#pragma unroll
  for (int w = 0; w < NT / kWave; ++w) r += scratch[w];
  return r;
}

// A token's rank as one number: the larger logit first, of equal ones the lower column.  +0 and -0 are equal.  A key is never
// 0, which stands for "none".
__device__ __forceinline__ uint64_t rank_key(float x, int col) {
  const uint32_t b = __float_as_uint(x + 0.f);
  const uint32_t o = b & 0x80000000u ? ~b : b | 0x80000000u;
  return (uint64_t(o) << 32) | uint32_t(~col);
}
__device__ __forceinline__ float key_logit(uint64_t key) {
  const uint32_t o = uint32_t(key >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ int key_column(uint64_t key) { return int(~uint32_t(key)); }

struct LogprobArgs {
  const int32_t *targets;
  float *logp, *row_max, *log_sum, *entropy;
  int32_t *top_ids;
  float *top_logp;
  int T, V, k;
  int64_t ldl;
  float scale;
};

// One workgroup per row: maximum, sums, then the list, one more reading of the row per entry.
template <typename L>
__global__ __launch_bounds__(kRowThreads) void k_logprob(const L *logits, LogprobArgs a) {
  __shared__ float scratch[kRowThreads / kWave];
  __shared__ uint64_t best[kRowThreads / kWave];
  const int tid = threadIdx.x;
  const float c = a.scale * kLog2e;
  for (int row = blockIdx.x; row < a.T; row += gridDim.x) {
    const L *x = logits + int64_t(row) * a.ldl;
    float m = -INFINITY;
    for (int j = tid; j < a.V; j += kRowThreads) m = fmaxf(m, to_f32(x[j]));
    m = block_max<kRowThreads>(m, scratch);
    const float ref = m == -INFINITY ? 0.f : m;
    float S = 0.f, A = 0.f;
    for (int j = tid; j < a.V; j += kRowThreads) {
      const float u = (to_f32(x[j]) - ref) * c, e = fast_exp2(u);
      S += e;
      A += e * fmaxf(u, kNoWeight);
    }
    S = block_sum<kRowThreads>(S, scratch);
    A = block_sum<kRowThreads>(A, scratch);
    const float log_sum = logf(S);
    auto log_p = [&](float v) { return S == 0.f ? -INFINITY : (v - ref) * a.scale - log_sum; };
    if (tid == 0) {
      const int tgt = a.targets ? a.targets[row] : -1;
      if (a.logp) a.logp[row] = tgt >= 0 && tgt < a.V ? log_p(to_f32(x[tgt])) : 0.f;
      if (a.row_max) a.row_max[row] = m;
      if (a.log_sum) a.log_sum[row] = log_sum;
      if (a.entropy) a.entropy[row] = S == 0.f ? 0.f : log_sum - A * kLn2 / S;
    }
    uint64_t last = ~uint64_t(0);
    for (int i = 0; i < a.k; ++i) {
      uint64_t b = 0;
      for (int j = tid; j < a.V; j += kRowThreads) {
        const float v = to_f32(x[j]);
        if (v > -INFINITY) {
          const uint64_t key = rank_key(v, j);
          if (key < last && key > b) b = key;
        }
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) b = max(b, uint64_t(__shfl_xor((unsigned long long)b, o, kWave)));
      __syncthreads();
      if (tid % kWave == 0) best[tid / kWave] = b;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kRowThreads / kWave; ++w) b = max(b, best[w]);
      last = b;
      if (tid == 0) {
        a.top_ids[int64_t(row) * a.k + i] = b ? key_column(b) : -1;
        a.top_logp[int64_t(row) * a.k + i] = b ? log_p(key_logit(b)) : -INFINITY;
      }
    }
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

// g_j = s (a (1[j = target] - p_j) - h p_j (log p_j + H)) with a = dL/dlogp, h = dL/dH
template <typename L, typename E>
__global__ __launch_bounds__(kRowThreads) void k_logprob_bwd(const L *logits, E *dlogits, LogprobGradArgs g) {
  for (int row = blockIdx.x; row < g.T; row += gridDim.x) {
    const L *x = logits + int64_t(row) * g.ldl;
    E *d = dlogits + int64_t(row) * g.ldd;
    const float m = g.row_max[row], z = g.log_sum[row];
    const int tgt = g.targets ? g.targets[row] : -1;
    const float a = g.d_logp && tgt >= 0 && tgt < g.V ? g.d_logp[row] : 0.f;
    const float h = g.d_entropy ? g.d_entropy[row] : 0.f, H = g.d_entropy ? g.entropy[row] : 0.f;
    for (int j = threadIdx.x; j < g.V + g.pad; j += kRowThreads) {
      float v = 0.f;
      if (j < g.V && z != -INFINITY) {
        const float l = (to_f32(x[j]) - m) * g.scale - z, p = fast_exp2(l * kLog2e);
        v = g.scale * ((j == tgt ? a : 0.f) - p * (a + h * (fmaxf(l, kNoWeight) + H)));
      } else if (j == tgt && j < g.V) {
        v = g.scale * a;
      }
      d[j] = from_f32<E>(v);
    }
  }
}

struct DistillArgs {
  const int32_t *ids;
  const float *logp;
  float *row_loss;
  int T, V, K, tail, pad;
  int64_t ldl, ldd;
  float scale, grad_scale;
};

// Loss and gradient of one row; the list's terms in 64 bits (a divergence is small beside the logarithms that it is the
// difference of), the row's exponentials in 32.  With a tail the row's sum is that of the listed tokens and that of the others.
template <typename L, typename E>
__global__ __launch_bounds__(kRowThreads) void k_distill(const L *logits, E *dlogits, DistillArgs a) {
  __shared__ float scratch[kRowThreads / kWave];
  __shared__ double dscratch[kRowThreads / kWave];
  __shared__ int ids[HMY_MAX_TOP];
  __shared__ double q_of[HMY_MAX_TOP];
  const int tid = threadIdx.x;
  const float c = a.scale * kLog2e;
  for (int row = blockIdx.x; row < a.T; row += gridDim.x) {
    const L *x = logits + int64_t(row) * a.ldl;
    E *d = dlogits ? dlogits + int64_t(row) * a.ldd : nullptr;
    // the list: thread k has entry k; an entry that names no token or has no weight is not there
    int id = -1;
    double t = -INFINITY;
    float xk = 0.f;
    if (tid < a.K) {
      id = a.ids[int64_t(row) * a.K + tid];
      t = a.logp[int64_t(row) * a.K + tid];
      if (id < 0 || id >= a.V || t == -INFINITY) id = -1;
      if (id >= 0) xk = to_f32(x[id]);
    }
    __syncthreads();
    if (tid < HMY_MAX_TOP) ids[tid] = id;
    const bool there = id >= 0, any = block_sum<kRowThreads>(there ? 1.f : 0.f, scratch) > 0.f;
    double q;
    if (a.tail) {
      q = there ? exp(t) : 0.;
    } else {
      const float tm = block_max<kRowThreads>(there ? float(t) : -INFINITY, scratch);
      const double e = there ? exp(t - double(tm)) : 0.;
      const double n = block_sum<kRowThreads>(e, dscratch);
      q = e / n;
      t = t - double(tm) - log(n);
    }
    const double q_sum = block_sum<kRowThreads>(there ? q : 0., dscratch);
    float m = -INFINITY;
    for (int j = tid; j < a.V; j += kRowThreads) m = fmaxf(m, to_f32(x[j]));
    m = block_max<kRowThreads>(m, scratch);
    const float ref = m == -INFINITY ? 0.f : m;
    float rest = 0.f, listed = 0.f;
    for (int j = tid; j < a.V; j += kRowThreads) {
      const float e = fast_exp2((to_f32(x[j]) - ref) * c);
      bool in = false;
      for (int k = 0; k < a.K; ++k) in |= ids[k] == j;
      if (in) listed += e;
      else rest += e;
    }
    const double S_rest = block_sum<kRowThreads>(rest, scratch), S = S_rest + block_sum<kRowThreads>(listed, scratch);
    const double u = (double(xk) - double(ref)) * a.scale;
    double loss = there && q > 0. ? q * (t - (u - log(S))) : (there ? q * 0. : 0.);
    loss = block_sum<kRowThreads>(loss, dscratch);
    double q_rest = a.tail && any && !(S_rest == 0.) ? fmax(1. - q_sum, 0.) : 0.;
    if (q_rest > 0.) loss += q_rest * (log(q_rest) - log(S_rest / S));
    if (tid == 0) a.row_loss[row] = any ? float(loss) : 0.f;
    if (!d) continue;
    const double w = double(a.scale) * double(a.grad_scale), inv = S == 0. || !any ? 0. : 1. / S;
    const float c_list = float(w * (q_sum + q_rest) * inv);
    const float c_rest = q_rest > 0. ? float(w * (q_sum + q_rest - q_rest * S / S_rest) * inv) : c_list;
    if (tid < HMY_MAX_TOP) q_of[tid] = q;
    __syncthreads();
    double same = 0.;
    if (there)
      for (int k = 0; k < a.K; ++k)
        if (ids[k] == id) same += q_of[k];
    for (int j = tid; j < a.V + a.pad; j += kRowThreads) {
      bool in = false;
      for (int k = 0; k < a.K; ++k) in |= ids[k] == j;
      if (!in) d[j] = from_f32<E>(j < a.V && any ? fast_exp2((to_f32(x[j]) - ref) * c) * c_rest : 0.f);
    }
    if (there) d[id] = from_f32<E>(float(double(fast_exp2((xk - ref) * c)) * double(c_list) - w * same));
    __syncthreads();
  }
}

// loss[0] += scale * the sum of the rows' losses, in one order whatever the launch
__global__ __launch_bounds__(kRowThreads) void k_loss_sum(const float *row_loss, double *loss, int T, double scale) {
  __shared__ double scratch[kRowThreads / kWave];
  double v = 0.;
  for (int i = threadIdx.x; i < T; i += kRowThreads) v += double(row_loss[i]);
  v = block_sum<kRowThreads>(v, scratch);
  if (threadIdx.x == 0) loss[0] += v * scale;
}

inline int check_launch(const char *what) {
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(HMY_E_HIP, "launch of %s failed: %s", what, hipGetErrorString(e));
  return HMY_OK;
}

constexpr int kMaxGrid = 1 << 20;   // workgroups; rows beyond are taken in further rounds
constexpr int kMaxColumns = 1 << 24;

inline bool misaligned(const void *p, int to) { return (reinterpret_cast<uintptr_t>(p) & uintptr_t(to - 1)) != 0; }
inline int bytes_of(int prec) { return prec == HMY_PREC_BF16 ? 2 : 4; }

int check_rows(const char *who, int prec, const void *p, int T, int V, int pad, int64_t ld) {
  if (prec != HMY_PREC_FP32 && prec != HMY_PREC_BF16) return fail(HMY_E_INVALID, "%s: unknown precision %d", who, prec);
  if (T < 1 || V < 1 || V > kMaxColumns) return fail(HMY_E_INVALID, "%s: T >= 1 and 1 <= V <= %d wanted, got T = %d, V = %d", who, kMaxColumns, T, V);
  if (pad < 0 || ld < int64_t(V) + pad) return fail(HMY_E_INVALID, "%s: a row stride of %lld does not hold %d columns and a padding of %d", who, (long long)ld, V, pad);
  if (ld > (int64_t(1) << 46) / T) return fail(HMY_E_INVALID, "%s: row stride out of range", who);
  if (misaligned(p, bytes_of(prec))) return fail(HMY_E_INVALID, "%s: rows not aligned to their elements", who);
  return HMY_OK;
}

// Whether rows of `a_cols` and `b_cols` bytes at pitches of `a_ld` and `b_ld` bytes share memory, other than as the same rows of
// the same type (in place).  Rows of one pitch may lie side by side in a wider array.
bool rows_clash(const void *a, int64_t a_cols, int64_t a_ld, const void *b, int64_t b_cols, int64_t b_ld, int T, bool same_type) {
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

bool positive(float s) { return s > 0.f && std::isfinite(s); }

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
  const LogprobArgs a = {g.targets, g.logp, g.row_max, g.log_sum, g.entropy, g.top_ids, g.top_logp, g.T, g.V, g.k, g.ldl, g.scale};
  const dim3 grid(g.T < kMaxGrid ? g.T : kMaxGrid);
  const hipStream_t s = (hipStream_t)st;
  if (g.logits_prec == HMY_PREC_BF16) hipLaunchKernelGGL(k_logprob<bf16_t>, grid, dim3(kRowThreads), 0, s, (const bf16_t *)g.logits, a);
  else hipLaunchKernelGGL(k_logprob<float>, grid, dim3(kRowThreads), 0, s, (const float *)g.logits, a);
  return check_launch("logprob");
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
  const dim3 grid(g.T < kMaxGrid ? g.T : kMaxGrid);
  DISPATCH_ROWS(g.logits_prec, g.prec, {
    hipLaunchKernelGGL((k_logprob_bwd<L, E>), grid, dim3(kRowThreads), 0, (hipStream_t)st, (const L *)g.logits, (E *)g.dlogits, a);
  });
  return check_launch("logprob_bwd");
}

int launch_distill(const hmy_distill_desc &g, stream_t st) {
  int rc = check_rows("distill", g.logits_prec, g.logits, g.T, g.V, 0, g.ldl);
  if (!rc && g.dlogits) rc = check_rows("distill", g.prec, g.dlogits, g.T, g.V, g.pad, g.ldd);
  if (rc) return rc;
  if (!positive(g.scale)) return fail(HMY_E_INVALID, "distill: the scale must be positive and finite");
  if (!std::isfinite(g.grad_scale)) return fail(HMY_E_INVALID, "distill: the gradient's scale must be finite");
  if (g.K < 1 || g.K > HMY_MAX_TOP) return fail(HMY_E_INVALID, "distill: K = %d is not in 1..%d", g.K, HMY_MAX_TOP);
  if (g.tail != 0 && g.tail != 1) return fail(HMY_E_INVALID, "distill: tail is 0 or 1");
  const void *words[] = {g.teacher_ids, g.teacher_logp, g.row_loss};
  for (const void *p : words)
    if (misaligned(p, 4)) return fail(HMY_E_INVALID, "distill: misaligned array");
  if (misaligned(g.loss_acc, 8)) return fail(HMY_E_INVALID, "distill: misaligned loss_acc");
  const int el = bytes_of(g.logits_prec), ee = bytes_of(g.prec);
  if (g.dlogits && rows_clash(g.logits, int64_t(g.V) * el, g.ldl * el, g.dlogits, (int64_t(g.V) + g.pad) * ee, g.ldd * ee, g.T, g.logits_prec == g.prec))
    return fail(HMY_E_INVALID, "distill: dlogits overlaps logits other than in place");
  const DistillArgs a = {g.teacher_ids, g.teacher_logp, g.row_loss, g.T, g.V, g.K, g.tail, g.pad, g.ldl, g.ldd, g.scale, g.grad_scale};
  const dim3 grid(g.T < kMaxGrid ? g.T : kMaxGrid);
  DISPATCH_ROWS(g.logits_prec, g.prec, {
    hipLaunchKernelGGL((k_distill<L, E>), grid, dim3(kRowThreads), 0, (hipStream_t)st, (const L *)g.logits, (E *)g.dlogits, a);
  });
  if (g.loss_acc)
    hipLaunchKernelGGL(k_loss_sum, dim3(1), dim3(kRowThreads), 0, (hipStream_t)st, g.row_loss, g.loss_acc, g.T, double(g.grad_scale));
  return check_launch("distill");
}

}  // namespace hmy
