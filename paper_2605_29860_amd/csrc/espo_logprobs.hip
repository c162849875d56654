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
constexpr int kComputeUnits = 256, kMostParts = 16;
// Rows are held by a workgroup each from this many waves on (the chip has 4096 at a time); fewer leave compute units idle, and two passes of
// smaller workgroups are faster.  us, held / two passes, by how full the registers of the row's workgroup are:
//   V = 152064 bf16  16 waves, 98 %  N = 64 31.6 / 18.4   128 32.2 / 30.2   160 32.6 / 33.4   256 40.1 / 43.6   1000 114 / 146
//   V = 70000 bf16    8 waves, 90 %  N = 200 22.5 / 21.1  256 23.7 / 24.5
//   V = 32000 bf16    4 waves, 82 %  N = 400 21.5 / 19.0  512 22.4 / 23.0
//   V = 80000 bf16   16 waves, 51 %  N = 128 23.6 / 17.4  256 26.7 / 26.8   1000 75 / 82
//   V = 40000 bf16    8 waves, 51 %  N = 256 18.8 / 15.4  512 25.6 / 27.4   4096 140 / 159
//   V = 20000 bf16    4 waves, 51 %  N = 512 19.1 / 16.2  1024 28.3 / 29.3  4096 85 / 90
//   V = 8000 bf16     4 waves, 21 %  N = 512 14.7 / 12.0  1024 20.7 / 16.1  4096 58 / 52
// So the line is near the crossing for full registers (2 us late at 16 waves), for half full ones the crossing is at twice as many rows, and rows
// of a fifth, whose other loads fetch their last vector again, would always be faster in two passes.  All rows count, used or not: of N = 128
// with half of them unused, 32.7 / 28.0.
constexpr int64_t kHeldWaves = 2048;
constexpr int kSumThreads = 1024, kSumWaves = kSumThreads / kWave;

struct RowArgs {
  const char* logits;
  int64_t row_bytes, N;
  uint32_t V;
  float temperature, inv_t, k2;
  const int32_t* tokens;
};

struct RowOutputs {  // of a forward pass; what is not wanted is null
  float *logprob, *entropy;
  float2* stats;     // row maximum and sum of e^t
};

__device__ __forceinline__ bool used_row(int32_t token, uint32_t V) { return (uint32_t)token < V; }  // a negative token is beyond any V

// What a row's sums (of row_sums) come to.  A row without any logit has the statistics of an empty sum, and its token is masked.
__device__ __forceinline__ void row_results(const RowArgs& a, float x_token, const SoftmaxSums& q, float& logprob, float& entropy, float2& stats) {
  const bool any = q.m > kMaskedRow;
  const float ln_s = any ? logf(q.s) : 0.0f;
  logprob = x_token > kMaskedRow ? -(q.m - x_token) * a.inv_t - ln_s : kNegInf;
  entropy = any ? ln_s - q.a * __builtin_amdgcn_rcpf(q.s) * kLn2 : 0.0f;
  stats = any ? float2{q.m, q.s} : float2{0.0f, 1.0f};
}

__device__ __forceinline__ void store_row(const RowOutputs& o, int64_t row, float logprob, float entropy, float2 stats) {
  if (o.logprob) o.logprob[row] = logprob;
  if (o.entropy) o.entropy[row] = entropy;
  if (o.stats) o.stats[row] = stats;
}

// The sums of tiles t0 .. t1 - 1 of a row, the same in every thread.
template <int DT, bool kEntropy>
__device__ __forceinline__ SoftmaxSums sum_tiles(const RowArgs& a, const RowView& r, uint32_t t0, uint32_t t1, SoftmaxSums* lds) {
  constexpr int E = vec_elems<DT>();
  SoftmaxSums p = kNoSums;
  stream_tiles(r, t0 + (threadIdx.x >> 6), t1, kRowWaves, [&](uint32_t t, const u32x4* raw) {
    float y[kAhead][E], m = p.m;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (t + j * kRowWaves >= t1) {
#pragma unroll
        for (int i = 0; i < E; ++i) y[j][i] = kNegInf;
        continue;
      }
      tile_logits<DT>(r, t + j * kRowWaves, raw[j], y[j]);
#pragma unroll
      for (int i = 0; i < E; ++i) m = fmaxf(m, y[j][i]);
    }
    follow<kEntropy>(p, m, a.k2);
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (t + j * kRowWaves < t1) {
#pragma unroll
        for (int i = 0; i < E; ++i) add_logit<kEntropy>(p, y[j][i], a.k2);
      }
  });
  return block_merge<kRowWaves, kEntropy>(p, a.k2, lds);
}

// Bound by memory and, nearly as much, by the vector units: with the entropy 9.3 operations per logit, one of them an exponential at a quarter of the others'
// rate, take 44 us of the launch's 47 (V = 152064 bf16, 922 rows of N = 1024: 280 MB, 5.9 TB/s; a bare read of as much takes 39).
// One workgroup per row, which is read once; or, where there are few rows, `parts` workgroups that leave their sums for
// espo_logprobs_join_kernel.
template <int DT, bool kEntropy, bool kSplit>
__global__ __launch_bounds__(kRowThreads) void espo_logprobs_kernel(RowArgs a, RowOutputs o, SoftmaxSums* split, uint32_t parts) {
  __shared__ SoftmaxSums lds[kRowWaves];
  const int64_t row = kSplit ? blockIdx.x / parts : blockIdx.x;
  const int32_t token = a.tokens[row];
  if (!used_row(token, a.V)) {
    if (!kSplit && threadIdx.x == 0) store_row(o, row, 0.0f, 0.0f, float2{0.0f, 1.0f});
    return;
  }
  const char* x = a.logits + row * a.row_bytes;
  const RowView r = row_view<DT>(x, a.V);
  if constexpr (kSplit) {
    const uint32_t part = blockIdx.x % parts, each = (r.ntiles + parts - 1) / parts, t0 = part * each;
    const SoftmaxSums p = sum_tiles<DT, kEntropy>(a, r, t0, min(t0 + each, r.ntiles), lds);
    if (threadIdx.x == 0) split[blockIdx.x] = p;
  } else {
    const SoftmaxSums p = row_sums<DT, kRowWaves>(r, sum_tiles<DT, kEntropy>(a, r, 0, r.ntiles, lds), a.k2, lds);
    if (threadIdx.x == 0) {
      float logprob, entropy;
      float2 stats;
      row_results(a, logit_at<DT>(x, (uint32_t)token), p, logprob, entropy, stats);
      store_row(o, row, logprob, entropy, stats);
    }
  }
}

// The parts' sums of a row put together, by a wave.
template <int DT, bool kEntropy>
__global__ __launch_bounds__(kWave) void espo_logprobs_join_kernel(RowArgs a, RowOutputs o, const SoftmaxSums* split, uint32_t parts) {
  const int64_t row = blockIdx.x;
  const int32_t token = a.tokens[row];
  float logprob = 0.0f, entropy = 0.0f;
  float2 stats{0.0f, 1.0f};
  if (used_row(token, a.V)) {
    const char* x = a.logits + row * a.row_bytes;
    const SoftmaxSums p = wave_merge<kEntropy>(threadIdx.x < parts ? split[row * parts + threadIdx.x] : kNoSums, a.k2);
    row_results(a, logit_at<DT>(x, (uint32_t)token), row_sums<DT, 1>(row_view<DT>(x, a.V), p, a.k2, nullptr), logprob, entropy, stats);
  }
  if (threadIdx.x == 0) store_row(o, row, logprob, entropy, stats);
}

// The objective at one token: L = s w (-min(r A, clip(r) A) - c H) with r = exp(ln pi - ln pi_old).
struct PolicyArgs {
  const float *old_logprob, *adv, *weights;
  float clip_low, clip_high, entropy_coef, scale;
};

struct Surrogate {
  float ratio, diff;
  bool cut;  // the clipped branch is the smaller one, and no gradient passes
};

struct TokenInputs {
  float old_logprob, adv, weight;
};
__device__ __forceinline__ TokenInputs token_inputs(const PolicyArgs& q, int64_t row) {
  return TokenInputs{q.old_logprob[row], q.adv[row], q.scale * (q.weights ? q.weights[row] : 1.0f)};
}

// The ratio is held below e^88, the largest power of e that fp32 holds: a product with an advantage of 0 stays 0.
__device__ __forceinline__ Surrogate surrogate(const PolicyArgs& q, const TokenInputs& in, float logprob) {
  Surrogate c;
  c.diff = logprob - in.old_logprob;
  c.ratio = expf(fminf(c.diff, 88.0f));
  c.cut = in.adv >= 0.0f ? c.ratio > 1.0f + q.clip_high : c.ratio < 1.0f - q.clip_low;
  return c;
}

// A row's gradient: dx_v = 2^t (p0 + p1 t) with t = x_v k2 + nb, and `at` more at the token.
struct RowGrad {
  float k2, nb, p0, p1, at;
};

// k2 for a row's gradient.  From kFarLane on nb's rounding alone would be no number as a power of 2, and nothing but the largest logit has a
// weight: then any factor does that keeps logits which differ apart, and m times a power of 2 is exact.
__device__ __forceinline__ float grad_slope(float m, float k2) {
  if (fabsf(m * k2) < kFarLane) return k2;
  return __builtin_bit_cast(float, (286u << 23) - (__builtin_bit_cast(uint32_t, m) & 0x7f800000u));  // |m| times this is 2^32 to 2^33, neighbours differ by 2^9
}

// m, s: the row's largest logit and sum; `entropy` only counts where h is not 0.
__device__ __forceinline__ RowGrad row_grad(const RowArgs& a, float m, float s, float entropy, float g, float h) {
#pragma clang fp contract(off)  // nb is a rounded product
  const float k2 = uniform_f32(grad_slope(m, a.k2), 0), nb = -m * k2, d = exponent_short(m, nb, k2);  // t is short by the rounding of nb, and 2^t by a factor
  const float per = a.inv_t * __builtin_amdgcn_rcpf(s) * __builtin_amdgcn_exp2f(d), p1 = -h * kLn2 * per;
  return RowGrad{k2, nb, p1 * d - (h != 0.0f ? g + h * (entropy - logf(s)) : g) * per, p1, g * a.inv_t};
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
    float t = __builtin_fmaf(x, c.k2, c.nb);
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

// The sums of the objective over all rows, in double and in a fixed order: one workgroup of W threads, thread i takes rows i, i + W, ...,
// `kRows` of them on their way at once.
struct PolicySums {
  const float *logprob, *entropy;
  espo_policy_result* out;
};
template <int W, int kRows>
__device__ __forceinline__ void policy_sums(const RowArgs& a, const PolicySums& p, const PolicyArgs& q) {
  constexpr int kSums = 5, kWaves = W / kWave;
  __shared__ double lds[kSums + 1][kWaves];
  double v[kSums + 1] = {};
#pragma unroll 1
  for (int64_t first = threadIdx.x; first < a.N; first += kRows * W) {
    TokenInputs in[kRows];
    float logprob[kRows], entropy[kRows];
    int32_t token[kRows];
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      const int64_t row = first + j * W < a.N ? first + j * W : first;
      token[j] = first + j * W < a.N ? a.tokens[row] : -1;
      in[j] = token_inputs(q, row);
      logprob[j] = p.logprob[row], entropy[j] = p.entropy[row];
    }
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      if (!used_row(token[j], a.V)) continue;
      const Surrogate c = surrogate(q, in[j], logprob[j]);
      const double w = in[j].weight, adv = in[j].adv, H = entropy[j], bound = c.cut ? (adv >= 0.0 ? 1.0 + q.clip_high : 1.0 - q.clip_low) : (double)c.ratio;
      v[0] += w * (-bound * adv - q.entropy_coef * H);
      v[1] += w * (-bound * adv);
      v[2] += w * H;
      v[3] += w != 0.0 ? w * (exp((double)fminf(c.diff, 88.0f)) - 1.0 - c.diff) : 0.0;  // ln r is -inf for a token that is masked
      v[4] += c.cut ? w : 0.0;
      v[5] += 1.0;
    }
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
  for (int i = 0; i <= kSums; ++i) v[i] = wave_sum_f64(lane < kWaves ? lds[i][lane] : 0.0);
  if (lane == 0)
    *p.out = espo_policy_result{(float)v[0], (float)v[1], (float)v[2], (float)v[3], (float)v[4], 0, (int64_t)v[5]};
}

// A workgroup writes kGradSpan vectors of one row's gradient: four loads per thread on their way before anything else, no loop, so that
// loads and stores of many small workgroups mix.  Bound by memory (V = 152064 bf16, 1638 of 2048 rows used: 498 MB in, 623 MB out in 187 us, 6.0 TB/s; a
// copy reaches 6.1).  kPolicy: the launch's first workgroup has the objective's sums instead, which a launch
// of their own would add 3 us for.
template <int DT, bool kPolicy>
__global__ __launch_bounds__(kGradThreads) void espo_logits_grad_kernel(RowArgs a, GradArgs d, PolicyArgs q, PolicySums p) {
  constexpr int E = vec_elems<DT>();
  if constexpr (kPolicy) {
    if (blockIdx.x == 0) {
      policy_sums<kGradThreads, 1>(a, p, q);
      return;
    }
  }
  const uint32_t group = blockIdx.x - (kPolicy ? 1 : 0);
  const int64_t row = group / d.spans;
  const uint32_t base = (uint32_t)(group - row * d.spans) * kGradSpan, nvec = (a.V + E - 1) / E;
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
    const TokenInputs in = token_inputs(q, row);
    const Surrogate c = surrogate(q, in, d.logprob[row]);
    g = c.cut ? 0.0f : -in.weight * c.ratio * in.adv;
    h = -in.weight * q.entropy_coef;
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

// Forward, objective and gradient of a row by one workgroup that holds the row in registers, so that the logits come in once and the gradient
// goes out once.  While a row's sums are formed, the first vectors of the workgroup's next row travel to LDS; as a vector's gradient is
// stored, its registers take that vector of the next row, from LDS or from memory.  So there is always something under way, also
// where all compute units are at the same point, which they are more often than not.  Bound by memory: V = 152064 bf16, 3686 of 4096 rows used:
// 1.12 GB in, 1.25 GB out in 480 us, 4.9 TB/s (without any exponential 2 % less; 6.1 TB/s for a copy, whose loads and stores do not come in turns of a row).
// The workgroups share the used rows
// evenly, by rank among the used rows, and then the zeros of the unused ones, from the other end.
constexpr int kHeld = 19;                        // vectors of a thread: 76 of the 128 registers that 16 waves per compute unit leave
constexpr int kStaged = 8;                       // of them through LDS: 128 KB of the compute unit's 160
constexpr int kDealt = 256;                      // rows of a workgroup
constexpr int64_t kDealtEach = kDealt - 2;       // of both kinds together, rounded up each

// 16 bytes per lane straight into LDS, the wave's 1024 bytes from `to` on (the same in all its lanes).  The compiler knows nothing of the load: who
// reads what it brings waits for vmcnt(0) first, and the compiler's own waits for other loads come out as too long, never as too short.  (Of the
// builtin for it it does know, and lets every load wait for all that are on their way.)
__device__ __forceinline__ void load_to_lds(const char* from, const u32x4* to) {
  const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)to);
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(at) : "memory", "m0");
}

// A workgroup's rows, and what belongs to the used ones: a load of these in the row loop would wait for all the logits on their way.
struct DealtRows {
  int32_t row[kDealt], token[kDealt];
  TokenInputs in[kDealt];
};

// Keeps what was formed from a vector before from being kept in registers of its own (its logits as floats take twice the room).
__device__ __forceinline__ void hold(u32x4& v) { asm volatile("" : "+v"(v)); }

// The workgroup's share of the rows: the used ones from the front of `rows`, the others from its end, and how many of each.
template <int W>
__device__ __forceinline__ void deal_rows(const RowArgs& a, const PolicyArgs& q, DealtRows& rows, uint32_t (*counts)[W], int& nused, int& nother) {
  const uint32_t lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6, groups = gridDim.x, g = blockIdx.x, N = (uint32_t)a.N;
  uint32_t base = 0;                             // used rows so far
#pragma unroll 1
  for (uint32_t row = 0; row < N; row += W * kWave) {
    const bool mine = row + threadIdx.x < N;
    const int32_t token = mine ? a.tokens[row + threadIdx.x] : -1;
    const bool used = used_row(token, a.V);
    const uint64_t mask = __builtin_amdgcn_ballot_w64(used);
    uint32_t* count = counts[(row / (W * kWave)) & 1];
    if (lane == 0) count[wave] = (uint32_t)__builtin_popcountll(mask);
    __syncthreads();
    uint32_t rank = base + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
#pragma unroll
    for (uint32_t w = 0; w < W; ++w) {
      rank += w < wave ? count[w] : 0;
      base += count[w];
    }
    const uint32_t other = row + threadIdx.x - rank;
    if (used) {
      if (rank % groups == g) {
        const uint32_t at = rank / groups;
        rows.row[at] = (int32_t)(row + threadIdx.x);
        rows.token[at] = token;
        rows.in[at] = token_inputs(q, row + threadIdx.x);
      }
    } else if (mine) {
      if (other % groups == groups - 1 - g) rows.row[kDealt - 1 - other / groups] = (int32_t)(row + threadIdx.x);
    }
  }
  __syncthreads();
  const uint32_t others = N - base, h = groups - 1 - g;
  nused = (int)(base > g ? (base - g + groups - 1) / groups : 0);
  nother = (int)(others > h ? (others - h + groups - 1) / groups : 0);
}

template <int DT, int W, bool kSlope>
__global__ __launch_bounds__(W* kWave) __attribute__((amdgpu_waves_per_eu(4, 4))) void espo_policy_kernel(RowArgs a, RowOutputs o, GradArgs d, PolicyArgs q) {
  constexpr uint32_t E = vec_elems<DT>(), kThreads = W * kWave;
  extern __shared__ __align__(16) u32x4 staged[];  // [kStaged][kThreads]
  __shared__ SoftmaxSums lds[2][W];
  __shared__ uint32_t counts[2][W];
  __shared__ DealtRows rows;
  __shared__ float token_logit[2];
  const uint32_t nvec = (a.V + E - 1) / E;
  const int last = (int)((nvec - 1) / kThreads);  // of the vectors raw[0 .. last] of a thread, all but the last lie within the row
  // The thread's index, not to be seen through: its vectors' offsets would be kept in registers from row to row.
  const auto own_index = [] {
    uint32_t t = threadIdx.x;
    asm volatile("" : "+v"(t));
    return t;
  };
  // Where vector r of a row is, or where there is no row to come the same one again and again: no register waits for a branch.  (Those behind
  // the row's last vector are that one.)
  const auto place = [&](const char* x, bool any, int r) { return x + (size_t)min((any ? r * kThreads : 0) + own_index(), nvec - 1) * 16; };
  int nused, nother;
  deal_rows<W>(a, q, rows, counts, nused, nother);
  const auto row_at = [&](int i) { return (int64_t)__builtin_amdgcn_readfirstlane(rows.row[i]); };
  u32x4 raw[kHeld];
  {
    const char* x = a.logits + (nused > 0 ? row_at(0) : 0) * a.row_bytes;
#pragma unroll
    for (int r = 0; r < kHeld; ++r) raw[r] = __builtin_nontemporal_load((const u32x4*)place(x, nused > 0, r));
    __builtin_amdgcn_s_waitcnt(0x0F70);          // vmcnt(0), so that the loop's first vectors are waited for as LDS reads only
  }
#pragma unroll 1
  for (int i = 0; i < nused; ++i) {
    const int64_t row = row_at(i);
    const bool more = i + 1 < nused;
    const char* next_x = a.logits + row_at(more ? i + 1 : i) * a.row_bytes;
    char* out = d.dlogits + row * d.grad_bytes;
    const int32_t token = __builtin_amdgcn_readfirstlane(rows.token[i]);
    const int token_round = (int)((uint32_t)token / E / kThreads);
    const bool holds_token = threadIdx.x == (uint32_t)token / E % kThreads;
    SoftmaxSums p = kNoSums;
    u32x4 tail = vec_masked<DT>();
#pragma unroll
    for (int r = 0; r < kHeld; ++r) {
      if (r == token_round && holds_token) token_logit[i & 1] = logit_in<DT>(raw[r], (uint32_t)token % E);
      if (r < last) {
        float y[E], m = p.m;
        hold(raw[r]);
        vec_unpack<DT>(raw[r], y);
#pragma unroll
        for (uint32_t k = 0; k < E; ++k) m = fmaxf(m, y[k]);
        follow<true>(p, m, a.k2);
#pragma unroll
        for (uint32_t k = 0; k < E; ++k) add_logit<true>(p, y[k], a.k2);
      } else if (r == last) {
        tail = raw[r];
      }
      // The first vectors have come from LDS and have been waited for, so their place there is free; and a load behind which these are issued
      // would be waited for as if it were they.
      if (r >= kStaged && r < 2 * kStaged)
        load_to_lds(place(next_x, more, r - kStaged), staged + (r - kStaged) * kThreads + (threadIdx.x & ~(kWave - 1)));
    }
    const uint32_t last_vec = last * kThreads + own_index();
    {
      float y[E], m = p.m;
      vec_unpack<DT>(tail, y);
#pragma unroll
      for (uint32_t k = 0; k < E; ++k) {
        if (last_vec * E + k >= a.V) y[k] = kNegInf;
        m = fmaxf(m, y[k]);
      }
      follow<true>(p, m, a.k2);
#pragma unroll
      for (uint32_t k = 0; k < E; ++k) add_logit<true>(p, y[k], a.k2);
    }
    p = row_sums<DT, W>(row_view<DT>(a.logits + row * a.row_bytes, a.V), block_merge<W, true>(p, a.k2, lds[i & 1]), a.k2, lds[i & 1]);
    float logprob, entropy;
    float2 stats;
    row_results(a, token_logit[i & 1], p, logprob, entropy, stats);
    if (threadIdx.x == 0) store_row(o, row, logprob, entropy, stats);
    const TokenInputs in = rows.in[i];
    const Surrogate c = surrogate(q, in, logprob);
    const RowGrad g = row_grad(a, stats.x, stats.y, entropy, c.cut ? 0.0f : -in.weight * c.ratio * in.adv, kSlope ? -in.weight * q.entropy_coef : 0.0f);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the wave's part of `staged` is there
#pragma unroll
    for (int r = 0; r < kHeld; ++r) {
      hold(raw[r]);
      if (r < last) {
        const uint32_t at = r * kThreads + own_index();
        __builtin_nontemporal_store(grad_vec<DT, kSlope>(a, g, raw[r], at, token), (u32x4*)(out + (size_t)at * 16));
      }
      if (r < kStaged)
        raw[r] = staged[r * kThreads + own_index()];
      else
        raw[r] = __builtin_nontemporal_load((const u32x4*)place(next_x, more, r));
    }
    if (last_vec < nvec) vec_store<DT>(out, last_vec, a.V, grad_vec<DT, kSlope>(a, g, tail, last_vec, token));
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // the last loads, of no row
#pragma unroll 1
  for (int i = 0; i < nother; ++i) {
    const int64_t row = row_at(kDealt - 1 - i);
    char* out = d.dlogits + row * d.grad_bytes;
    if (threadIdx.x == 0) store_row(o, row, 0.0f, 0.0f, float2{0.0f, 1.0f});
#pragma unroll 1
    for (uint32_t j = threadIdx.x; j < nvec; j += kThreads) vec_store<DT>(out, j, a.V, u32x4{0, 0, 0, 0});
  }
}

__global__ __launch_bounds__(kSumThreads) void espo_policy_sums_kernel(RowArgs a, PolicySums p, PolicyArgs q) {
  policy_sums<kSumThreads, 4>(a, p, q);
}

RowArgs row_args(const void* logits, int dt, int64_t N, int64_t V, int64_t row_stride, float temperature, const int32_t* tokens) {
  const int es = dt == ESPO_BF16 ? 2 : 4;
  return RowArgs{(const char*)logits, row_stride * es, N, (uint32_t)V, temperature, 1.0f / temperature,
                 (float)(1.4426950408889634 / (double)temperature), tokens};
}

// Workgroups that a row of few is split over: what two per compute unit allow, of at least 32 tiles each (four per wave), and at least 8,
// because the second launch costs 2 to 3 us.  (With the entropy, us, whole and split: bf16 V = 152064 N = 1 12.6 and 5.3, N = 64 13.3 and 9.0,
// N = 100, over 5, 13.6 and 10.2, all without the host's time; fp32 V = 65536 N = 32 8.2 and 5.6; bf16 V = 65536, over 4, 7.2 and 6.0.)
uint32_t forward_parts(int dt, int64_t N, int64_t V) {
  const int64_t tiles = V / (kWave * (dt == ESPO_BF16 ? 8 : 4));
  int64_t n = 2 * kComputeUnits / N;
  if (n > tiles / 32) n = tiles / 32;
  if (n > kMostParts) n = kMostParts;
  return n < 8 ? 1u : (uint32_t)n;
}

template <int DT, bool kEntropy>
void forward(const RowArgs& a, const RowOutputs& o, SoftmaxSums* split, hipStream_t stream) {
  const uint32_t parts = split ? forward_parts(DT, a.N, a.V) : 1;
  if (parts > 1) {
    hipLaunchKernelGGL((espo_logprobs_kernel<DT, kEntropy, true>), dim3((unsigned)(a.N * parts)), dim3(kRowThreads), 0, stream, a, o, split, parts);
    hipLaunchKernelGGL((espo_logprobs_join_kernel<DT, kEntropy>), dim3((unsigned)a.N), dim3(kWave), 0, stream, a, o, split, parts);
  } else {
    hipLaunchKernelGGL((espo_logprobs_kernel<DT, kEntropy, false>), dim3((unsigned)a.N), dim3(kRowThreads), 0, stream, a, o, nullptr, 1u);
  }
}
template <int DT>
void forward(const RowArgs& a, const RowOutputs& o, SoftmaxSums* split, hipStream_t stream) {
  if (o.entropy)
    forward<DT, true>(a, o, split, stream);
  else
    forward<DT, false>(a, o, split, stream);
}

template <int DT, bool kPolicy>
void backward(const RowArgs& a, const GradArgs& d, const PolicyArgs& q, const PolicySums& p, hipStream_t stream) {
  hipLaunchKernelGGL((espo_logits_grad_kernel<DT, kPolicy>), dim3((unsigned)(a.N * d.spans) + (kPolicy ? 1 : 0)), dim3(kGradThreads), 0, stream, a, d, q, p);
}

// Waves of the workgroup that holds a row of V logits, 0 if none does.
template <int DT>
int held_waves(int64_t V) {
  const int64_t nvec = (V + vec_elems<DT>() - 1) / vec_elems<DT>();
  for (int w = 4; w <= 16; w *= 2)
    if (nvec <= (int64_t)w * kWave * kHeld) return w;
  return 0;
}

// The same arguments from row `from` on, for n rows.
RowArgs rows_from(RowArgs a, int64_t from, int64_t n) {
  a.logits += from * a.row_bytes;
  a.tokens += from;
  a.N = n;
  return a;
}

template <int DT, int W>
void policy_held(const RowArgs& a, const RowOutputs& o, const GradArgs& d, const PolicyArgs& q, hipStream_t stream) {
  const int64_t groups = a.N < kComputeUnits * (16 / W) ? a.N : kComputeUnits * (16 / W);
  for (int64_t from = 0; from < a.N; from += groups * kDealtEach) {  // one launch up to 65024 rows
    const int64_t n = a.N - from < groups * kDealtEach ? a.N - from : groups * kDealtEach;
    const RowArgs ra = rows_from(a, from, n);
    const RowOutputs ro{o.logprob + from, o.entropy + from, o.stats + from};
    GradArgs rd = d;
    rd.dlogits += from * d.grad_bytes;
    PolicyArgs rq = q;
    rq.old_logprob += from, rq.adv += from, rq.weights += q.weights ? from : 0;
    const dim3 grid((unsigned)(n < groups ? n : groups)), block(W * kWave);
    const size_t lds = (size_t)kStaged * W * kWave * 16;
    if (q.entropy_coef != 0.0f)
      hipLaunchKernelGGL((espo_policy_kernel<DT, W, true>), grid, block, lds, stream, ra, ro, rd, rq);
    else
      hipLaunchKernelGGL((espo_policy_kernel<DT, W, false>), grid, block, lds, stream, ra, ro, rd, rq);
  }
}

// Log-probabilities, entropy, the objective and, if it is wanted, its gradient.
template <int DT>
void policy(const RowArgs& a, const RowOutputs& o, const GradArgs& d, const PolicyArgs& q, const PolicySums& p, SoftmaxSums* split, hipStream_t stream) {
  const int waves = d.dlogits ? held_waves<DT>(a.V) : 0;
  switch (a.N * waves >= kHeldWaves ? waves : 0) {
    case 4: policy_held<DT, 4>(a, o, d, q, stream); break;
    case 8: policy_held<DT, 8>(a, o, d, q, stream); break;
    case 16: policy_held<DT, 16>(a, o, d, q, stream); break;
    default:
      if (a.N > 0) forward<DT>(a, o, split, stream);
      if (a.N > 0 && d.dlogits) return backward<DT, true>(a, d, q, p, stream);
  }
  hipLaunchKernelGGL(espo_policy_sums_kernel, dim3(1), dim3(kSumThreads), 0, stream, a, p, q);
}

uint32_t grad_spans(int dt, int64_t V) {
  const int64_t span = (int64_t)kGradSpan * (dt == ESPO_BF16 ? 8 : 4);
  return (uint32_t)((V + span - 1) / span);
}

int launched() { return hipGetLastError() == hipSuccess ? ESPO_OK : ESPO_EHIP; }

}  // namespace

// (A launch has fewer than 2^32 threads; one workgroup more than the gradient needs is the policy loss's.)
bool grad_indexable(int dt, int64_t N, int64_t V) { return N * (int64_t)grad_spans(dt, V) + 1 < ((int64_t)1 << 32) / kGradThreads; }

int launch_logprobs(const void* logits, int dt, int64_t N, int64_t V, int64_t row_stride, float temperature, const int32_t* tokens,
                    float* logprob, float* entropy, float* stats, void* workspace, hipStream_t stream) {
  const RowArgs a = row_args(logits, dt, N, V, row_stride, temperature, tokens);
  const RowOutputs o{logprob, entropy, (float2*)stats};
  if (dt == ESPO_BF16) forward<ESPO_BF16>(a, o, (SoftmaxSums*)workspace, stream);
  else forward<ESPO_F32>(a, o, (SoftmaxSums*)workspace, stream);
  return launched();
}

size_t logprobs_workspace(int dt, int64_t N, int64_t V) {
  const uint32_t parts = forward_parts(dt, N, V);
  return parts > 1 ? (size_t)N * parts * sizeof(SoftmaxSums) : 0;
}

int launch_logprobs_backward(const void* logits, int dt, int64_t N, int64_t V, int64_t row_stride, float temperature, const int32_t* tokens,
                             const float* stats, const float* entropy, const float* dlogprob, const float* dentropy, void* dlogits,
                             int64_t grad_stride, hipStream_t stream) {
  const RowArgs a = row_args(logits, dt, N, V, row_stride, temperature, tokens);
  const GradArgs d{(char*)dlogits, grad_stride * (dt == ESPO_BF16 ? 2 : 4), grad_spans(dt, V), (const float2*)stats, entropy, dlogprob, dentropy, nullptr};
  if (dt == ESPO_BF16) backward<ESPO_BF16, false>(a, d, PolicyArgs{}, PolicySums{}, stream);
  else backward<ESPO_F32, false>(a, d, PolicyArgs{}, PolicySums{}, stream);
  return launched();
}

// Per row: maximum and sum, log-probability, entropy; behind them what the forward pass needs.
size_t policy_workspace(int dt, int64_t N, int64_t V) { return (size_t)N * 16 + logprobs_workspace(dt, N, V); }

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
  const PolicySums p{logprob, entropy, out};
  SoftmaxSums* split = (SoftmaxSums*)(stats + 2 * N);
  if (dt == ESPO_BF16) policy<ESPO_BF16>(a, o, d, q, p, split, stream);
  else policy<ESPO_F32>(a, o, d, q, p, split, stream);
  return launched();
}

}  // namespace espo
