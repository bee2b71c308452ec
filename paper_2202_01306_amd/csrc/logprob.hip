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

constexpr int kRowThreads = 256;

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
