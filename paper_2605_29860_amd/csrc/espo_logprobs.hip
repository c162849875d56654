// espo_logprobs, espo_logprobs_backward, espo_policy_loss: log-probabilities of given tokens, the entropy of their
// distributions, the gradient of both on the logits, and the clipped objective of PPO (Section 3, Eq. ppo) on top of them.
//
// With t_v = (x_v - m) / T, S = sum_v e^t_v and pi_v = e^t_v / S:
//   ln pi_a = t_a - ln S,   H = ln S - sum_v pi_v t_v,
//   dx_v = (g ([v = a] - pi_v) - h pi_v (ln pi_v + H)) / T   for dL/d(ln pi_a) = g, dL/dH = h.
// Exponents are to base 2, so that dx_v = 2^t (p0 + p1 t) with two numbers per row, plus g / T at the token.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/espo.h"
#include "espo_device.h"
#include "espo_host.h"
#include "espo_rows.h"

namespace espo {
namespace {

constexpr int kRowWaves = 8, kRowThreads = kRowWaves * kWave;
constexpr int kGradThreads = 256, kGradLoads = 4;
constexpr int kGradSpan = kGradThreads * kGradLoads;  // vectors of a workgroup
constexpr int kSumThreads = 1024, kSumWaves = kSumThreads / kWave;

struct RowArgs {
  const char* logits;
  int64_t row_bytes, N;
  uint32_t V;
  float temperature, k2;
  const int32_t* tokens;
};

struct RowOutputs {  // of a forward pass; what is not wanted is null
  float *logprob, *entropy;
  float2* stats;     // row maximum and sum of e^t
};

__device__ __forceinline__ bool used_row(int32_t token, uint32_t V) { return (uint32_t)token < V; }  // a negative token is beyond any V

// What a row's sums come to.  A row without any logit has the statistics of an empty sum, and its token is masked.
__device__ __forceinline__ void row_results(const RowArgs& a, float x_token, const SoftmaxSums& p, float& logprob, float& entropy, float2& stats) {
  const bool any = p.m > kMaskedRow;
  const float ln_s = any ? logf(p.s) : 0.0f;
  logprob = x_token > kMaskedRow ? -(p.m - x_token) / a.temperature - ln_s : kNegInf;
  entropy = any ? ln_s - p.a / p.s * kLn2 : 0.0f;
  stats = any ? float2{p.m, p.s} : float2{0.0f, 1.0f};
}

__device__ __forceinline__ void store_row(const RowOutputs& o, int64_t row, float logprob, float entropy, float2 stats) {
  if (o.logprob) o.logprob[row] = logprob;
  if (o.entropy) o.entropy[row] = entropy;
  if (o.stats) o.stats[row] = stats;
}

// One workgroup per row, which is read once.
template <int DT, bool kEntropy>
__global__ __launch_bounds__(kRowThreads) void espo_logprobs_kernel(RowArgs a, RowOutputs o) {
  __shared__ SoftmaxSums lds[kRowWaves];
  constexpr int E = vec_elems<DT>();
  const int64_t row = blockIdx.x;
  const int32_t token = a.tokens[row];
  if (!used_row(token, a.V)) {
    if (threadIdx.x == 0) store_row(o, row, 0.0f, 0.0f, float2{0.0f, 1.0f});
    return;
  }
  const char* x = a.logits + row * a.row_bytes;
  const RowView r = row_view<DT>(x, a.V);
  SoftmaxSums p{kMaskedRow, 0.0f, 0.0f};
  stream_tiles(r, threadIdx.x >> 6, r.ntiles, kRowWaves, [&](uint32_t t, const u32x4* raw) {
    float y[kAhead][E], m = p.m;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (t + j * kRowWaves >= r.ntiles) {
#pragma unroll
        for (int i = 0; i < E; ++i) y[j][i] = kNegInf;
        continue;
      }
      tile_logits<DT>(r, t + j * kRowWaves, raw[j], y[j]);
#pragma unroll
      for (int i = 0; i < E; ++i) m = fmaxf(m, y[j][i]);
    }
    rescale<kEntropy>(p, m, a.k2);
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (t + j * kRowWaves < r.ntiles) {
#pragma unroll
        for (int i = 0; i < E; ++i) add_logit<kEntropy>(p, y[j][i], a.k2);
      }
  });
  p = block_merge<kRowWaves, kEntropy>(p, a.k2, lds);
  if (threadIdx.x == 0) {
    float logprob, entropy;
    float2 stats;
    row_results(a, logit_at<DT>(x, (uint32_t)token), p, logprob, entropy, stats);
    store_row(o, row, logprob, entropy, stats);
  }
}

// The objective at one token: L = s w (-min(r A, clip(r) A) - c H) with r = exp(ln pi - ln pi_old).
struct PolicyArgs {
  const float *old_logprob, *adv, *weights;
  float clip_low, clip_high, entropy_coef, scale;
};

struct Surrogate {
  float ratio, diff, weight;
  bool cut;  // the clipped branch is the smaller one, and no gradient passes
};

// The ratio is held below e^88, the largest power of e that fp32 holds: a product with an advantage of 0 stays 0.
__device__ __forceinline__ Surrogate surrogate(const PolicyArgs& q, int64_t row, float logprob, float adv) {
  Surrogate c;
  c.diff = logprob - q.old_logprob[row];
  c.ratio = expf(fminf(c.diff, 88.0f));
  c.weight = q.scale * (q.weights ? q.weights[row] : 1.0f);
  c.cut = adv >= 0.0f ? c.ratio > 1.0f + q.clip_high : c.ratio < 1.0f - q.clip_low;
  return c;
}

// A row's gradient: dx_v = 2^t (p0 + p1 t) with t = (x_v - m) k2, and `at` more at the token.
struct RowGrad {
  float m, p0, p1, at;
};

// m, s: the row's largest logit and sum; `entropy` only counts where h is not 0.
__device__ __forceinline__ RowGrad row_grad(const RowArgs& a, float m, float s, float entropy, float g, float h) {
  const float per = 1.0f / (a.temperature * s);
  return RowGrad{m, -(h != 0.0f ? g + h * (entropy - logf(s)) : g) * per, -h * kLn2 * per, g / a.temperature};
}

template <int DT, bool kSlope>
__device__ __forceinline__ u32x4 grad_vec(const RowArgs& a, const RowGrad& c, u32x4 raw, uint32_t i, int32_t token) {
  constexpr int E = vec_elems<DT>();
  float y[E];
  vec_unpack<DT>(raw, y);
  const bool here = i == (uint32_t)token / E;
#pragma unroll
  for (int k = 0; k < E; ++k) {
    const float x = y[k];
    float t = (x - c.m) * a.k2;
    if constexpr (kSlope) t = fmaxf(t, kLeastExponent);
    const float e = __builtin_amdgcn_exp2f(t);
    y[k] = e * (kSlope ? __builtin_fmaf(c.p1, t, c.p0) : c.p0);
    if (here && (uint32_t)token % E == (uint32_t)k && x > kMaskedRow) y[k] += c.at;
  }
  return vec_pack<DT>(y);
}

struct GradArgs {
  char* dlogits;
  int64_t grad_bytes;
  uint32_t spans;
  const float2* stats;
  const float *entropy, *dlogprob, *dentropy;  // the caller's loss
  const float* logprob;                        // the policy loss
};

// A workgroup writes kGradSpan vectors of one row's gradient.
template <int DT, bool kPolicy>
__global__ __launch_bounds__(kGradThreads) void espo_logits_grad_kernel(RowArgs a, GradArgs d, PolicyArgs q) {
  constexpr int E = vec_elems<DT>();
  const int64_t row = blockIdx.x / d.spans;
  const uint32_t base = (uint32_t)(blockIdx.x - row * d.spans) * kGradSpan, nvec = (a.V + E - 1) / E;
  const int32_t token = a.tokens[row];
  char* out = d.dlogits + row * d.grad_bytes;
  if (!used_row(token, a.V)) {
#pragma unroll
    for (int j = 0; j < kGradLoads; ++j) {
      const uint32_t i = base + j * kGradThreads + threadIdx.x;
      if (i < nvec) vec_store<DT>(out, i, a.V, u32x4{0, 0, 0, 0});
    }
    return;
  }
  const char* x = a.logits + row * a.row_bytes;
  u32x4 r[kGradLoads];
#pragma unroll
  for (int j = 0; j < kGradLoads; ++j) r[j] = vec_load<DT>(x, base + j * kGradThreads + threadIdx.x, a.V);
  float g, h = 0.0f;
  if constexpr (kPolicy) {
    const float adv = q.adv[row];
    const Surrogate c = surrogate(q, row, d.logprob[row], adv);
    g = c.cut ? 0.0f : -c.weight * c.ratio * adv;
    h = -c.weight * q.entropy_coef;
  } else {
    g = d.dlogprob[row];
    if (d.dentropy) h = d.dentropy[row];
  }
  const float2 st = d.stats[row];
  const RowGrad c = row_grad(a, st.x, st.y, h != 0.0f ? d.entropy[row] : 0.0f, g, h);
#pragma unroll
  for (int j = 0; j < kGradLoads; ++j) {
    const uint32_t i = base + j * kGradThreads + threadIdx.x;
    if (i >= nvec) break;
    vec_store<DT>(out, i, a.V, c.p1 != 0.0f ? grad_vec<DT, true>(a, c, r[j], i, token) : grad_vec<DT, false>(a, c, r[j], i, token));
  }
}

// The sums of the objective over all rows, in double and in a fixed order: one workgroup, thread i takes rows i, i + 1024, ...
__global__ __launch_bounds__(kSumThreads) void espo_policy_sums_kernel(const int32_t* tokens, const float* logprob, const float* entropy,
                                                                       int64_t N, uint32_t V, PolicyArgs q, espo_policy_result* out) {
  constexpr int kSums = 5;
  __shared__ double lds[kSums + 1][kSumWaves];
  double v[kSums + 1] = {};
  for (int64_t row = threadIdx.x; row < N; row += kSumThreads) {
    if (!used_row(tokens[row], V)) continue;
    const float adv = q.adv[row];
    const Surrogate c = surrogate(q, row, logprob[row], adv);
    const double w = c.weight, H = entropy[row], bound = c.cut ? (adv >= 0.0f ? 1.0 + q.clip_high : 1.0 - q.clip_low) : (double)c.ratio;
    v[0] += w * (-bound * adv - q.entropy_coef * H);
    v[1] += w * (-bound * adv);
    v[2] += w * H;
    v[3] += w * (exp((double)fminf(c.diff, 88.0f)) - 1.0 - c.diff);
    v[4] += c.cut ? w : 0.0;
    v[5] += 1.0;
  }
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i <= kSums; ++i) {
    v[i] = wave_sum_f64(v[i]);
    if (lane == 0) lds[i][wave] = v[i];
  }
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int i = 0; i <= kSums; ++i) v[i] = wave_sum_f64(lane < kSumWaves ? lds[i][lane] : 0.0);
  if (lane == 0)
    *out = espo_policy_result{(float)v[0], (float)v[1], (float)v[2], (float)v[3], (float)v[4], 0, (int64_t)v[5]};
}

RowArgs row_args(const void* logits, int dt, int64_t N, int64_t V, int64_t row_stride, float temperature, const int32_t* tokens) {
  const int es = dt == ESPO_BF16 ? 2 : 4;
  return RowArgs{(const char*)logits, row_stride * es, N, (uint32_t)V, temperature, (float)(1.4426950408889634 / (double)temperature), tokens};
}

template <int DT>
void forward(const RowArgs& a, const RowOutputs& o, hipStream_t stream) {
  if (o.entropy)
    hipLaunchKernelGGL((espo_logprobs_kernel<DT, true>), dim3((unsigned)a.N), dim3(kRowThreads), 0, stream, a, o);
  else
    hipLaunchKernelGGL((espo_logprobs_kernel<DT, false>), dim3((unsigned)a.N), dim3(kRowThreads), 0, stream, a, o);
}

template <int DT, bool kPolicy>
void backward(const RowArgs& a, const GradArgs& d, const PolicyArgs& q, hipStream_t stream) {
  hipLaunchKernelGGL((espo_logits_grad_kernel<DT, kPolicy>), dim3((unsigned)(a.N * d.spans)), dim3(kGradThreads), 0, stream, a, d, q);
}

uint32_t grad_spans(int dt, int64_t V) {
  const int64_t span = (int64_t)kGradSpan * (dt == ESPO_BF16 ? 8 : 4);
  return (uint32_t)((V + span - 1) / span);
}

int launched() { return hipGetLastError() == hipSuccess ? ESPO_OK : ESPO_EHIP; }

}  // namespace

bool grad_indexable(int dt, int64_t N, int64_t V) { return N * (int64_t)grad_spans(dt, V) <= 0x7fffffff; }

int launch_logprobs(const void* logits, int dt, int64_t N, int64_t V, int64_t row_stride, float temperature, const int32_t* tokens,
                    float* logprob, float* entropy, float* stats, hipStream_t stream) {
  const RowArgs a = row_args(logits, dt, N, V, row_stride, temperature, tokens);
  const RowOutputs o{logprob, entropy, (float2*)stats};
  if (dt == ESPO_BF16) forward<ESPO_BF16>(a, o, stream);
  else forward<ESPO_F32>(a, o, stream);
  return launched();
}

int launch_logprobs_backward(const void* logits, int dt, int64_t N, int64_t V, int64_t row_stride, float temperature, const int32_t* tokens,
                             const float* stats, const float* entropy, const float* dlogprob, const float* dentropy, void* dlogits,
                             int64_t grad_stride, hipStream_t stream) {
  const RowArgs a = row_args(logits, dt, N, V, row_stride, temperature, tokens);
  const GradArgs d{(char*)dlogits, grad_stride * (dt == ESPO_BF16 ? 2 : 4), grad_spans(dt, V), (const float2*)stats, entropy, dlogprob, dentropy, nullptr};
  if (dt == ESPO_BF16) backward<ESPO_BF16, false>(a, d, PolicyArgs{}, stream);
  else backward<ESPO_F32, false>(a, d, PolicyArgs{}, stream);
  return launched();
}

// Per row: maximum and sum, log-probability, entropy.
size_t policy_workspace(int64_t N) { return (size_t)N * 16; }

int launch_policy_loss(const void* logits, int dt, int64_t N, int64_t V, int64_t row_stride, float temperature, const int32_t* tokens,
                       const float* old_logprob, const float* adv, const float* weights, const espo_policy_ctrl& c, void* dlogits,
                       int64_t grad_stride, float* logprob, float* entropy, espo_policy_result* out, void* workspace, hipStream_t stream) {
  const RowArgs a = row_args(logits, dt, N, V, row_stride, temperature, tokens);
  const PolicyArgs q{old_logprob, adv, weights, c.clip_low, c.clip_high, c.entropy_coef, c.scale};
  float2* stats = (float2*)workspace;
  if (!logprob) logprob = (float*)(stats + N);
  if (!entropy) entropy = (float*)(stats + N) + N;
  const RowOutputs o{logprob, entropy, stats};
  const GradArgs d{(char*)dlogits, grad_stride * (dt == ESPO_BF16 ? 2 : 4), grad_spans(dt, V), stats, entropy, nullptr, nullptr, logprob};
  if (N > 0) {
    if (dt == ESPO_BF16) forward<ESPO_BF16>(a, o, stream);
    else forward<ESPO_F32>(a, o, stream);
    if (launched() != ESPO_OK) return ESPO_EHIP;
    if (dlogits) {
      if (dt == ESPO_BF16) backward<ESPO_BF16, true>(a, d, q, stream);
      else backward<ESPO_F32, true>(a, d, q, stream);
      if (launched() != ESPO_OK) return ESPO_EHIP;
    }
  }
  hipLaunchKernelGGL(espo_policy_sums_kernel, dim3(1), dim3(kSumThreads), 0, stream, tokens, logprob, entropy, N, (uint32_t)V, q, out);
  return launched();
}

}  // namespace espo
