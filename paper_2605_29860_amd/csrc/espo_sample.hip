// espo_sample: a token per row from given random numbers, every row with its own temperature, top-k, top-p and min-p.
//
// With t_v = (x_v - m) / T and w_v = e^t_v, the kept tokens are those whose logit reaches a cut, the largest of what the three
// filters ask for; the token is the first, in the order of the vocabulary, at which the running sum of the kept weights exceeds
// u times their total.  Which token that is turns on sums of up to V weights: with V of 10^5 and a flat distribution two
// neighbouring sums differ by 10^-5 of the total, and the rounding errors of fp32 sums (10^-7) would move one draw in a hundred.  So
// weights and sums are doubles, and sums that are formed by atomics are integers (the order of additions then changes nothing).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/espo.h"
#include "espo_device.h"
#include "espo_host.h"
#include "espo_rows.h"

namespace espo {
namespace {

constexpr int kWaves = 16, kThreads = kWaves * kWave;
constexpr int kBins = 2048;                 // of a level of the search for a cut: 11, 11 and 10 bits of the key
constexpr double kFixed = 8796093022208.0;  // 2^43: a weight of 1 as an integer; 2^20 of them stay below 2^63

typedef unsigned long long u64;

struct SampleArgs {
  const char* logits;
  int64_t row_bytes;
  uint32_t V;
  const float* temperature;
  const int32_t* top_k;
  const float *top_p, *min_p, *u;
  const uint8_t* alive;
  int32_t* tokens;
  float* logprob;
};

// Order of the logits as unsigned integers; both zeros are one value.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}

struct SampleShared {
  u64 mass[kBins];
  uint32_t count[kBins];
  double part[256];  // sums of a row's sixteenths, then of the tiles of one of them
  float m[kWaves];
  uint32_t at[kWaves];
  u64 found_mass, above_mass;
  uint32_t found_bin, above_count;
  int32_t token;
  double sum;
};

// The inclusive sums over the lanes before and at this one.
template <typename T>
__device__ __forceinline__ T wave_scan(T v) {
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const T o = __shfl_up(v, d);
    if ((int)(threadIdx.x & (kWave - 1)) >= d) v += o;
  }
  return v;
}

struct Row {
  const char* x;
  uint32_t V, nvec;
  double inv_t, m;  // 1 / temperature, largest logit
  __device__ __forceinline__ double weight(float v) const { return exp(((double)v - m) * inv_t); }
};

// What decides a cut: the k-th largest logit, or the logit at which the mass from the top reaches `target`.
struct Goal {
  bool by_count;
  u64 k;
  double target;
  __device__ __forceinline__ bool reached(u64 count, u64 mass) const { return by_count ? count >= k : (double)mass >= target; }
};

// The key of the logit at which the goal is reached from the top among keys of at least `floor`, and the mass of all keys down to it.
template <int DT>
__device__ uint32_t find_cut(const Row& r, uint32_t floor, const Goal& goal, SampleShared& s, u64& mass_to_cut) {
  constexpr int E = vec_elems<DT>();
  uint32_t prefix = 0;
  u64 above_count = 0, above_mass = 0;
#pragma unroll 1
  for (int level = 0; level < 3; ++level) {
    const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11;
    for (int i = threadIdx.x; i < kBins; i += kThreads) s.count[i] = 0, s.mass[i] = 0;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < r.nvec; i += kThreads) {
      float y[E];
      vec_unpack<DT>(vec_load<DT>(r.x, i, r.V), y);
      for (int j = 0; j < E; ++j) {
        const uint32_t key = key_of(y[j]);
        if (!(y[j] > kMaskedRow) || key < floor || (level > 0 && (key >> (shift + bits)) != prefix)) continue;
        const uint32_t bin = (key >> shift) & ((1u << bits) - 1);
        atomicAdd(&s.count[bin], 1u);
        atomicAdd(&s.mass[bin], (u64)(r.weight(y[j]) * kFixed + 0.5));
      }
    }
    __syncthreads();
    if (threadIdx.x < kWave) {  // lane l has the bins from kBins - 32 (l + 1) on, so that lower lanes come first from the top
      constexpr int kEach = kBins / kWave;
      const int first = kBins - kEach * ((int)threadIdx.x + 1);
      u64 c = 0, w = 0;
      for (int i = 0; i < kEach; ++i) c += s.count[first + i], w += s.mass[first + i];
      const u64 cs = above_count + wave_scan(c), ws = above_mass + wave_scan(w);
      const uint64_t hit = __builtin_amdgcn_ballot_w64(c > 0 && goal.reached(cs, ws)), some = __builtin_amdgcn_ballot_w64(c > 0);
      // rounding may leave a target just above the mass of everything: the last bin that holds a logit is then the one
      const int lane = hit ? (int)__builtin_ctzll(hit) : 63 - (int)__builtin_clzll(some);
      if ((int)threadIdx.x == lane) {
        u64 ca = cs - c, wa = ws - w;
        int bin = -1;
        u64 cb = 0, wb = 0;
        for (int i = kEach - 1; i >= 0; --i) {
          const u64 ci = s.count[first + i], wi = s.mass[first + i];
          if (ci == 0) continue;
          if (bin >= 0) ca += cb, wa += wb;
          bin = first + i, cb = ci, wb = wi;
          if (goal.reached(ca + cb, wa + wb)) break;
        }
        s.found_bin = (uint32_t)bin;
        s.above_count = (uint32_t)ca;
        s.above_mass = wa;
        s.found_mass = wa + wb;
      }
    }
    __syncthreads();
    prefix = (prefix << bits) | s.found_bin;
    above_count = s.above_count;
    above_mass = s.above_mass;
  }
  mass_to_cut = s.found_mass;
  return prefix;
}

// The lane at which the running sum of v exceeds `rest`, or the last one with v > 0; `rest` becomes what is left before it.
__device__ __forceinline__ int pick_lane(double v, double& rest) {
  const double upto = wave_scan(v);
  const uint64_t hit = __builtin_amdgcn_ballot_w64(v > 0.0 && upto > rest), some = __builtin_amdgcn_ballot_w64(v > 0.0);
  const int lane = hit ? (int)__builtin_ctzll(hit) : 63 - (int)__builtin_clzll(some | 1);
  rest -= __shfl(upto - v, lane);
  return lane;
}

template <int DT>
__global__ __launch_bounds__(kThreads) void espo_sample_kernel(SampleArgs a) {
  __shared__ SampleShared s;
  constexpr uint32_t E = vec_elems<DT>();
  const int64_t b = blockIdx.x;
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  const auto result = [&](int32_t token, float logprob) {
    a.tokens[b] = token;
    if (a.logprob) a.logprob[b] = logprob;
  };
  if (a.alive && !a.alive[b]) {
    if (threadIdx.x == 0) result(-1, 0.0f);
    return;
  }
  const float T = a.temperature ? a.temperature[b] : 1.0f;
  Row r{a.logits + b * a.row_bytes, a.V, (a.V + E - 1) / E, 1.0 / (double)T, 0.0};
  // the largest logit, and the first index that has it
  float m = kMaskedRow;
  uint32_t at = 0xffffffffu;
  for (uint32_t i = threadIdx.x; i < r.nvec; i += kThreads) {
    float y[E];
    vec_unpack<DT>(vec_load<DT>(r.x, i, r.V), y);
    for (uint32_t j = 0; j < E; ++j)
      if (y[j] > m) m = y[j], at = i * E + j;
  }
  const float mw = wave_max(m);
  const uint32_t aw = wave_min_u32(m == mw ? at : 0xffffffffu);
  if (lane == 0) s.m[wave] = mw, s.at[wave] = aw;
  __syncthreads();
  m = s.m[0];
  for (int i = 1; i < kWaves; ++i) m = fmaxf(m, s.m[i]);
  at = 0xffffffffu;
  for (int i = 0; i < kWaves; ++i)
    if (s.m[i] == m) at = min(at, s.at[i]);
  if (!(m > kMaskedRow) || !(T > 0.0f)) {  // nothing to draw from, or greedy
    if (threadIdx.x == 0) result(m > kMaskedRow ? (int32_t)at : -1, 0.0f);
    return;
  }
  r.m = (double)m;
  // the cut
  const int32_t k = a.top_k ? a.top_k[b] : 0;
  const float p = a.top_p ? a.top_p[b] : 1.0f, min_p = a.min_p ? fminf(a.min_p[b], 1.0f) : 0.0f;
  uint32_t floor = 0;
  u64 mass = 0;
  if (k > 0 && (uint32_t)k < a.V) floor = find_cut<DT>(r, 0, Goal{true, (u64)k, 0.0}, s, mass);
  if (p > 0.0f && p < 1.0f) {
    if (mass == 0) find_cut<DT>(r, 0, Goal{true, (u64)a.V + 1, 0.0}, s, mass);  // the mass of the whole row
    floor = find_cut<DT>(r, floor, Goal{false, 0, (double)p * (double)mass}, s, mass);
  }
  const auto kept = [&](float x) {
    if (!(x > kMaskedRow) || key_of(x) < floor) return 0.0;
    const double w = r.weight(x);
    return w >= (double)min_p ? w : 0.0;
  };
  // the draw: sums of the row's sixteenths, of the tiles (64 vectors) of one of them, of the vectors of one tile
  const uint32_t ntiles = (r.nvec + kWave - 1) / kWave, per = (ntiles + kWaves - 1) / kWaves;
  const auto vector_sum = [&](uint32_t i) {
    double w = 0.0;
    float y[E];
    vec_unpack<DT>(vec_load<DT>(r.x, i, r.V), y);
    for (uint32_t j = 0; j < E; ++j) w += kept(y[j]);
    return w;
  };
  double sum = 0.0;
  for (uint32_t t = wave * per; t < min((wave + 1) * per, ntiles); ++t) sum += vector_sum(t * kWave + lane);
  sum = wave_sum_f64(sum);
  if (lane == 0) s.part[wave] = sum;
  __syncthreads();
  const double each = lane < kWaves ? s.part[lane] : 0.0, total = wave_sum_f64(each);
  double rest = (double)a.u[b] * total;
  const uint32_t seg = (uint32_t)pick_lane(each, rest);
  __syncthreads();
  const uint32_t t0 = seg * per, t1 = min(t0 + per, ntiles);
  for (uint32_t t = t0 + wave; t < t1; t += kWaves) {
    const double w = wave_sum_f64(vector_sum(t * kWave + lane));
    if (lane == 0) s.part[t - t0] = w;
  }
  __syncthreads();
  if (wave != 0) return;
  uint32_t tile = t0;
  double left = rest;
  for (uint32_t t = t0; t < t1; t += kWave) {
    const double w = t + lane < t1 ? s.part[t + lane - t0] : 0.0, all = wave_sum_f64(w);
    if (all <= 0.0) continue;
    double here = rest;
    tile = t + (uint32_t)pick_lane(w, here);
    left = here;
    if (all > rest) break;
    rest -= all;
  }
  const uint32_t i = tile * kWave + lane;
  const double w = vector_sum(i);
  const int who = pick_lane(w, left);
  if (lane != who) return;
  float y[E];
  vec_unpack<DT>(vec_load<DT>(r.x, i, r.V), y);
  int32_t token = -1;
  float x = m;
  double upto = 0.0;
  for (uint32_t j = 0; j < E; ++j) {
    const double wj = kept(y[j]);
    if (wj <= 0.0) continue;
    token = (int32_t)(i * E + j), x = y[j];
    upto += wj;
    if (upto > left) break;
  }
  result(token, (float)(((double)x - r.m) * r.inv_t - log(total)));
}

}  // namespace

int launch_sample(const void* logits, int dt, int64_t B, int64_t V, int64_t row_stride, const float* temperature, const int32_t* top_k,
                  const float* top_p, const float* min_p, const float* u, const uint8_t* alive, int32_t* tokens, float* logprob,
                  hipStream_t stream) {
  const SampleArgs a{(const char*)logits, row_stride * (dt == ESPO_BF16 ? 2 : 4), (uint32_t)V, temperature, top_k, top_p, min_p, u, alive, tokens, logprob};
  if (dt == ESPO_BF16)
    hipLaunchKernelGGL(espo_sample_kernel<ESPO_BF16>, dim3((unsigned)B), dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(espo_sample_kernel<ESPO_F32>, dim3((unsigned)B), dim3(kThreads), 0, stream, a);
  return hipGetLastError() == hipSuccess ? ESPO_OK : ESPO_EHIP;
}

}  // namespace espo
