// espo_sample: a token per row from given random numbers, every row with its own temperature, top-k, top-p and min-p.
//
// With t_v = (x_v - m) / T and w_v = e^t_v, the kept tokens are those whose logit reaches a cut, the largest of what the three
// filters ask for; the token is the first, in the order of the vocabulary, at which the running sum of the kept weights exceeds
// u times their total.  Which token that is turns on sums of up to V weights: with V of 10^5 and a flat distribution two
// neighbouring sums differ by 10^-5 of the total, and the rounding errors of fp32 sums (10^-7) would move one draw in a hundred.  So
// weights and sums are doubles (a v_fma_f64 takes no longer than a v_fma_f32 here), and sums that are formed by atomics are integers
// (the order of additions then changes nothing).
//
// One workgroup per row, which is streamed once.  A row without filters leaves the sum of each wave's part; the part, the tile and
// the vector that the draw falls into are read again.  A filtered row leaves how many logits (and, of fp32 logits under top-p, how
// much mass) fall into each of 4355 bins, which are the bf16 numbers from 2^-10 to 128 of either sign, and the largest logit of
// every block of 16 vectors.  The bins say where the cut is: exactly so for bf16 logits, whose bins hold one value each, and up to one
// bin's members for fp32 logits, which are then collected and ranked.  Only blocks that reach the cut are read again.
// Rows that the bins do not describe (logits of 128 and more, a cut among the numbers next to 0, a nucleus that -128 still has a
// share in, a bin with thousands of members) find their cut by three levels of 2048 bins over the whole key, one pass over the row each.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/espo.h"
#include "espo_device.h"
#include "espo_host.h"
#include "espo_rows.h"

namespace espo {
namespace {

typedef unsigned long long u64;

constexpr int kAhead = 4;                   // vectors of a lane in flight
constexpr int kBlockVecs = 16;              // vectors of a block: one row of 16 lanes, whose maximum takes four DPP steps
constexpr double kFixed = 8796093022208.0;  // 2^43: a weight of 1 as an integer; 2^20 of them stay below 2^63
constexpr double kNoWeight = 1e-250;        // weights below this count as none

// ---------------------------------------------------------------- bins of bf16 numbers
constexpr int kMagBelow = ((127 - 10) << 7) - 1;  // the bf16 number before 2^-10
constexpr int kMagSpan = 17 << 7;                 // numbers from 2^-10 to 128
constexpr int kBinZero = kMagSpan + 2;            // bin of everything next to 0
constexpr int kBins = 2 * kBinZero + 1;           // the first and the last usable one, 1 and kBins - 2, stand for all beyond 128
constexpr float kBinsBelow = 128.0f;
constexpr double kBinMass = 1099511627776.0;      // 2^40: the mass of a bin is in units of 2^-40 of its own number's weight

__device__ __forceinline__ int bin_of(uint32_t bits) {
  const int j = min(max((int)((bits >> 16) & 0x7fffu) - kMagBelow, 0), kMagSpan + 1), s = (int32_t)bits >> 31;
  return kBinZero + ((j ^ s) - s);
}
// The same for the two bf16 numbers in a word, as byte offsets of entries of `kEntry` bytes.
template <int kEntry>
__device__ __forceinline__ uint32_t bins_of_pair(uint32_t w) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  typedef short i16x2 __attribute__((ext_vector_type(2)));
  u16x2 j = __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, w & 0x7fff7fffu), (u16x2)(unsigned short)kMagBelow);
  j = __builtin_elementwise_min(j, (u16x2)(unsigned short)(kMagSpan + 1));
  const i16x2 s = __builtin_bit_cast(i16x2, w) >> 15;
  const i16x2 b = (__builtin_bit_cast(i16x2, j) ^ s) - s;
  return __builtin_bit_cast(uint32_t, __builtin_bit_cast(u16x2, b) * (unsigned short)kEntry + (u16x2)(unsigned short)(kBinZero * kEntry));
}
// The number of a bin: the one nearest to 0 that falls into it.
__device__ __forceinline__ float bin_number(int bin) {
  const int j = bin - kBinZero;
  if (j == 0) return 0.0f;
  return __builtin_bit_cast(float, (uint32_t)((abs(j) + kMagBelow) << 16) | (j < 0 ? 0x80000000u : 0u));
}
// No logit of the bin or of a higher one is below this.
__device__ __forceinline__ float bin_floor(int bin) {
  const int j = bin - kBinZero;
  if (j > 0) return bin_number(bin);
  return -__builtin_bit_cast(float, (uint32_t)((1 - j + kMagBelow) << 16));
}

// ---------------------------------------------------------------- 2^t in double
// 2^t for t up to 1000, 2^-1021 below that: t = n + f with |f| <= 1/2, a polynomial for 2^f that is exact at 0 (Chebyshev fit of (2^f - 1) / f,
// relative error 4e-14), n added to the exponent.
__device__ __forceinline__ double exp2_f64(double t) {
  constexpr double kRound = 6755399441055744.0;  // 1.5 * 2^52: the sum's low word is the nearest integer
  t = fmax(t, -1021.0);
  const double z = t + kRound, f = t - (z - kRound);
  double q = 0x1.b63880a30e9ffp-24;
  q = fma(q, f, 0x1.63d136366db24p-20);
  q = fma(q, f, 0x1.ffcb9515a8016p-17);
  q = fma(q, f, 0x1.4308ac85aa947p-13);
  q = fma(q, f, 0x1.5d87fe86fe88ep-10);
  q = fma(q, f, 0x1.3b2ab7181b755p-7);
  q = fma(q, f, 0x1.c6b08d7047e52p-5);
  q = fma(q, f, 0x1.ebfbdff823cedp-3);
  q = fma(q, f, 0x1.62e42fefa39efp-1);
  q = fma(q, f, 1.0);
  return __hiloint2double(__double2hiint(q) + (int)((uint32_t)__double2loint(z) << 20), __double2loint(q));
}

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
  uint32_t lds_blocks, lds_members;  // where the blocks' maxima and a bin's members start in dynamic LDS
};

struct Row {
  const char* x;
  uint32_t V, nvec, ntiles;
  double c, inv_t, m;  // log2(e) / T, 1 / T, largest logit
  __device__ __forceinline__ double weight(float v) const { return exp2_f64(((double)v - m) * c); }
};

// Order of the logits as unsigned integers; both zeros are one value.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}

constexpr int kLevelBins = 2048;            // of a level of the search over whole keys: 11, 11 and 10 bits
constexpr int kMostMembers = 512;           // of a bin that are ranked, each against all others

template <int W>
struct SampleShared {
  double part[4096 / W + 1];  // sums of the tiles of a wave's part
  double wave_f64[W];
  u64 found_mass, above_mass, kept_mass;
  float m[W];
  uint32_t at[W], wave_u32[W];
  uint32_t found_bin, above_count, first, last, nmembers, cut_key;
  double rest;
};

// The inclusive sums over the lanes before and at this one.
__device__ __forceinline__ double wave_scan(double v) {
  v += dpp_f64<kDppRowShr1, 0xf>(v);
  v += dpp_f64<kDppRowShr2, 0xf>(v);
  v += dpp_f64<kDppRowShr4, 0xf>(v);
  v += dpp_f64<kDppRowShr8, 0xf>(v);
  v += dpp_f64<kDppBcast15, 0xa>(v);
  v += dpp_f64<kDppBcast31, 0xc>(v);
  return v;
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
  v += dpp_u32<kDppRowShr1, 0xf>(0u, v);
  v += dpp_u32<kDppRowShr2, 0xf>(0u, v);
  v += dpp_u32<kDppRowShr4, 0xf>(0u, v);
  v += dpp_u32<kDppRowShr8, 0xf>(0u, v);
  v += dpp_u32<kDppBcast15, 0xa>(0u, v);
  v += dpp_u32<kDppBcast31, 0xc>(0u, v);
  return v;
}
__device__ __forceinline__ u64 wave_scan(u64 v) {
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const u64 o = __shfl_up(v, d);
    if ((int)(threadIdx.x & (kWave - 1)) >= d) v += o;
  }
  return v;
}

// The sum over the threads before this one, and over all of them; lds: W entries that a barrier has freed.
template <int W, typename T>
__device__ __forceinline__ T block_before(T v, T* lds, T& total) {
  const int wave = threadIdx.x >> 6;
  const T upto = wave_scan(v);
  if ((threadIdx.x & (kWave - 1)) == kWave - 1) lds[wave] = upto;
  __syncthreads();
  T before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < W; ++i) {
    const T each = lds[i];
    if (i < wave) before += each;
    all += each;
  }
  total = all;
  return before + upto - v;
}

// The thread whose part [before, before + v) of a running sum holds `target`: the first with before + v beyond it (or, where `reach`,
// at it); the last with any part if rounding leaves none.  The same in all threads; s.first and s.last have been reset before a barrier.
template <int W>
__device__ __forceinline__ uint32_t block_pick(double before, double v, double least, double target, bool reach, SampleShared<W>& s) {
  if (v > least) {
    const double upto = before + v;
    if (upto > target || (reach && upto == target)) atomicMin(&s.first, threadIdx.x);
    atomicMax(&s.last, threadIdx.x);
  }
  __syncthreads();
  return s.first != 0xffffffffu ? s.first : s.last;
}

// Calls use(tile, vector) for tiles first, first + step, ... below end, kAhead of them in flight while the kAhead before are used.
// A vector's index is clamped to the row's last one; `use` looks at what lies beyond V.
template <typename Use>
__device__ __forceinline__ void stream(const Row& r, uint32_t first, uint32_t end, uint32_t step, Use&& use) {
  const uint32_t lane = threadIdx.x & (kWave - 1);
  const auto load = [&](uint32_t t) {
    return __builtin_nontemporal_load((const u32x4*)(r.x + (size_t)min(t * kWave + lane, r.nvec - 1) * 16));
  };
  if (first >= end) return;
  u32x4 cur[kAhead], nxt[kAhead];
#pragma unroll
  for (int j = 0; j < kAhead; ++j) cur[j] = load(first + j * step);
  for (uint32_t t = first; t < end; t += kAhead * step) {
    const bool more = t + kAhead * step < end;
    if (more) {
#pragma unroll
      for (int j = 0; j < kAhead; ++j) nxt[j] = load(t + (kAhead + j) * step);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (t + j * step < end) use(t + j * step, cur[j]);
    if (more) {
#pragma unroll
      for (int j = 0; j < kAhead; ++j) cur[j] = nxt[j];
    }
  }
}

// A vector's logits; those at or beyond V are masked.
template <int DT>
__device__ __forceinline__ void logits_of(const Row& r, uint32_t i, u32x4 raw, float y[vec_elems<DT>()]) {
  constexpr uint32_t E = vec_elems<DT>();
  vec_unpack<DT>(raw, y);
  if (i * E + E > r.V) {
#pragma unroll
    for (uint32_t j = 0; j < E; ++j)
      if (i * E + j >= r.V) y[j] = kNegInf;
  }
}

template <int E>
__device__ __forceinline__ float max_of(const float y[E]) {
  float m = y[0];
#pragma unroll
  for (int j = 1; j < E; ++j) m = fmaxf(m, y[j]);
  return m;
}

// The largest logit of the row from each thread's largest.
template <int W>
__device__ __forceinline__ float block_max(float m, SampleShared<W>& s) {
  m = wave_max(m);
  const int lane = threadIdx.x & (kWave - 1);
  if (lane == 0) s.m[threadIdx.x >> 6] = m;
  __syncthreads();
  return wave_max(lane < W ? s.m[lane] : kMaskedRow);
}

// ---------------------------------------------------------------- the cut by whole keys, a pass per level
// What decides a cut: the k-th largest logit, or the logit at which the mass from the top reaches `target`.
struct Goal {
  bool by_count;
  u64 k;
  double target;
  __device__ __forceinline__ bool reached(u64 count, u64 mass) const { return by_count ? count >= k : (double)mass >= target; }
};

// The key of the logit at which the goal is reached from the top among keys of at least `floor`, and the mass of all keys down to it.
template <int DT, int W>
__device__ __forceinline__ uint32_t find_cut(const Row& r, uint32_t floor, const Goal& goal, unsigned char* lds, SampleShared<W>& s, u64& mass_to_cut) {
  constexpr uint32_t E = vec_elems<DT>();
  u64* mass = (u64*)lds;
  uint32_t* count = (uint32_t*)(mass + kLevelBins);
  uint32_t prefix = 0;
  u64 above_count = 0, above_mass = 0;
#pragma unroll 1
  for (int level = 0; level < 3; ++level) {
    const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11;
    __syncthreads();
    for (int i = threadIdx.x; i < kLevelBins; i += W * kWave) count[i] = 0, mass[i] = 0;
    __syncthreads();
#pragma unroll 1
    for (uint32_t i = threadIdx.x; i < r.nvec; i += W * kWave) {
      float y[E];
      vec_unpack<DT>(vec_load<DT>(r.x, i, r.V), y);
#pragma unroll 1
      for (uint32_t j = 0; j < E; ++j) {
        float x = y[0];
#pragma unroll
        for (uint32_t k = 1; k < E; ++k) x = j == k ? y[k] : x;
        const uint32_t key = key_of(x);
        if (!(x > kMaskedRow) || key < floor || (level > 0 && (key >> (shift + bits)) != prefix)) continue;
        const uint32_t bin = (key >> shift) & ((1u << bits) - 1);
        atomicAdd(&count[bin], 1u);
        atomicAdd(&mass[bin], (u64)(r.weight(x) * kFixed + 0.5));
      }
    }
    __syncthreads();
    if (threadIdx.x < kWave) {  // lane l has the bins from kLevelBins - 32 (l + 1) on, so that lower lanes come first from the top
      constexpr int kEach = kLevelBins / kWave;
      const int first = kLevelBins - kEach * ((int)threadIdx.x + 1);
      u64 c = 0, w = 0;
#pragma unroll 1
      for (int i = 0; i < kEach; ++i) c += count[first + i], w += mass[first + i];
      const u64 cs = above_count + wave_scan(c), ws = above_mass + wave_scan(w);
      const uint64_t hit = __builtin_amdgcn_ballot_w64(c > 0 && goal.reached(cs, ws)), some = __builtin_amdgcn_ballot_w64(c > 0);
      // rounding may leave a target just above the mass of everything: the last bin that holds a logit is then the one
      const int lane = hit ? (int)__builtin_ctzll(hit) : 63 - (int)__builtin_clzll(some | 1);
      if ((int)threadIdx.x == lane) {
        u64 ca = cs - c, wa = ws - w, cb = 0, wb = 0;
        int bin = 0;
#pragma unroll 1
        for (int i = kEach - 1; i >= 0; --i) {
          const u64 ci = count[first + i], wi = mass[first + i];
          if (ci == 0) continue;
          ca += cb, wa += wb;
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

// ---------------------------------------------------------------- the draw
// The lane at which the running sum of v exceeds `rest`, or the last one with any weight; `rest` becomes what is left before it.
__device__ __forceinline__ int pick_lane(double v, double& rest) {
  const double upto = wave_scan(v);
  const uint64_t hit = __builtin_amdgcn_ballot_w64(v > kNoWeight && upto > rest), some = __builtin_amdgcn_ballot_w64(v > kNoWeight);
  const int lane = hit ? (int)__builtin_ctzll(hit) : 63 - (int)__builtin_clzll(some | 1);
  rest -= __shfl(upto - v, lane);
  return lane;
}

__device__ __forceinline__ void store_result(const SampleArgs& a, int64_t b, int32_t token, float logprob) {
  a.tokens[b] = token;
  if (a.logprob) a.logprob[b] = logprob;
}

// The draw among one vector per lane of a wave, starting at vector i0: `rest` of the running sum is left before it.
template <int DT, typename Kept>
__device__ __forceinline__ void draw_in_vectors(const SampleArgs& a, int64_t b, const Row& r, uint32_t i, bool mine, double rest, double total,
                                                Kept&& kept) {
  constexpr uint32_t E = vec_elems<DT>();
  const u32x4 raw = mine ? vec_load<DT>(r.x, i, r.V) : vec_masked<DT>();
  const double ln_total = log(total);       // while the load is on its way
  float y[E];
  vec_unpack<DT>(raw, y);
  double w[E], sum = 0.0;
#pragma unroll
  for (uint32_t j = 0; j < E; ++j) sum += w[j] = kept(y[j]);
  const int who = pick_lane(sum, rest);
  if ((int)(threadIdx.x & (kWave - 1)) != who) return;
  int32_t token = -1;
  float x = 0.0f;
  double upto = 0.0;
  bool found = false;
#pragma unroll
  for (uint32_t j = 0; j < E; ++j) {
    if (found || !(w[j] > 0.0)) continue;
    token = (int32_t)(i * E + j), x = y[j];
    upto += w[j];
    found = upto > rest;
  }
  store_result(a, b, token, (float)(((double)x - r.m) * r.inv_t - ln_total));
}

// The draw within tiles t0 .. t1 - 1, where the running sum falls: the tiles' sums, the tile, its vectors.
template <int DT, int W, typename Kept>
__device__ __forceinline__ void draw_in_tiles(const SampleArgs& a, int64_t b, const Row& r, uint32_t t0, uint32_t t1, double rest, double total,
                                              SampleShared<W>& s, Kept&& kept) {
  constexpr uint32_t E = vec_elems<DT>();
  const uint32_t lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  stream(r, t0 + wave, t1, W, [&](uint32_t t, u32x4 raw) {
    const uint32_t i = t * kWave + lane;
    float y[E];
    logits_of<DT>(r, i, raw, y);
    double w = 0.0;
#pragma unroll
    for (uint32_t j = 0; j < E; ++j) w += kept(y[j]);
    w = wave_sum_f64(w);
    if (lane == 0) s.part[t - t0] = w;
  });
  __syncthreads();
  if (wave != 0) return;
  uint32_t tile = t0;
  double left = rest;
#pragma unroll 1
  for (uint32_t t = t0; t < t1; t += kWave) {
    const double w = t + lane < t1 ? s.part[t + lane - t0] : 0.0, all = wave_sum_f64(w);
    if (!(all > kNoWeight)) continue;
    left = rest;
    tile = t + (uint32_t)pick_lane(w, left);
    if (all > rest) break;
    rest -= all;
  }
  draw_in_vectors<DT>(a, b, r, tile * kWave + lane, true, left, total, kept);
}

// Greedy: the first index of the largest logit.
template <int DT, int W>
__device__ __forceinline__ void greedy(const SampleArgs& a, int64_t b, const Row& r, SampleShared<W>& s) {
  constexpr uint32_t E = vec_elems<DT>();
  const uint32_t lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  float m = kMaskedRow;
  uint32_t at = 0xffffffffu;
  stream(r, wave, r.ntiles, W, [&](uint32_t t, u32x4 raw) {
    const uint32_t i = t * kWave + lane;
    float y[E];
    logits_of<DT>(r, i, raw, y);
    const float top = max_of<E>(y);
    if (top > m) {
      m = top;
#pragma unroll
      for (int j = E - 1; j >= 0; --j)
        if (y[j] == top && i * E + j < r.V) at = i * E + j;
    }
  });
  const float top = wave_max(m);
  const uint32_t first = wave_min_u32(m == top ? at : 0xffffffffu);
  if (lane == 0) s.m[wave] = top, s.at[wave] = first;
  __syncthreads();
  if (wave != 0) return;
  m = lane < W ? s.m[lane] : kMaskedRow;
  const float all = wave_max(m);
  at = wave_min_u32(lane < W && m == all ? s.at[lane] : 0xffffffffu);
  if (lane == 0) store_result(a, b, all > kMaskedRow ? (int32_t)at : -1, 0.0f);
}

// No filter: each wave sums its part of the row, relative to a reference of its own that follows the largest logit only when that
// runs 2^500 ahead.
template <int DT, int W>
__device__ __forceinline__ void draw_plain(const SampleArgs& a, int64_t b, Row& r, SampleShared<W>& s) {
  constexpr uint32_t E = vec_elems<DT>();
  const uint32_t lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6, per = (r.ntiles + W - 1) / W;
  float m = kMaskedRow, limit = kMaskedRow;
  double sum = 0.0, ref = 0.0;
  const float lead = (float)(500.0 / r.c);
  stream(r, wave * per, min((wave + 1) * per, r.ntiles), 1, [&](uint32_t t, u32x4 raw) {
    const uint32_t i = t * kWave + lane;
    float y[E];
    logits_of<DT>(r, i, raw, y);
    const float top = max_of<E>(y);
    m = fmaxf(m, top);
    if (__builtin_amdgcn_ballot_w64(top > limit) != 0) {
      const float to = wave_max(m);
      sum = limit > kMaskedRow ? sum * exp2_f64((ref - (double)to) * r.c) : 0.0;
      ref = (double)to;
      limit = to + lead;
    }
#pragma unroll
    for (uint32_t j = 0; j < E; ++j) sum += exp2_f64(((double)y[j] - ref) * r.c);
  });
  const float top = block_max<W>(m, s);
  if (!(top > kMaskedRow)) {
    if (threadIdx.x == 0) store_result(a, b, -1, 0.0f);
    return;
  }
  r.m = (double)top;
  sum = limit > kMaskedRow ? wave_sum_f64(sum) * exp2_f64((ref - r.m) * r.c) : 0.0;
  if (lane == 0) s.wave_f64[wave] = sum;
  __syncthreads();
  const double each = lane < W ? s.wave_f64[lane] : 0.0, total = wave_sum_f64(each);
  double rest = (double)a.u[b] * total;
  const uint32_t seg = (uint32_t)pick_lane(each, rest);
  draw_in_tiles<DT, W>(a, b, r, seg * per, min((seg + 1) * per, r.ntiles), rest, total, s,
                       [&](float x) { return x > kMaskedRow ? r.weight(x) : 0.0; });
}

// A filtered row whose cut the bins do not give: the cut by whole keys, then the sum of each wave's part.
template <int DT, int W>
__device__ __forceinline__ void draw_by_keys(const SampleArgs& a, int64_t b, const Row& r, int32_t k, float p, double min_p, unsigned char* lds,
                                             SampleShared<W>& s) {
  constexpr uint32_t E = vec_elems<DT>();
  const uint32_t lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6, per = (r.ntiles + W - 1) / W;
  uint32_t floor = 0;
  u64 mass = 0;
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {  // the k largest (or the mass of the whole row), then the nucleus
    if (pass == 0 && k == 0 && p == 0.0f) continue;
    if (pass == 1 && p == 0.0f) continue;
    const Goal goal = pass == 1 ? Goal{false, 0, (double)p * (double)mass} : Goal{true, k > 0 ? (u64)k : (u64)r.V + 1, 0.0};
    const uint32_t cut = find_cut<DT, W>(r, floor, goal, lds, s, mass);
    if (pass == 1 || k > 0) floor = cut;
  }
  const auto kept = [&](float x) {
    if (!(x > kMaskedRow) || key_of(x) < floor) return 0.0;
    const double w = r.weight(x);
    return w >= min_p ? w : 0.0;
  };
  double sum = 0.0;
  stream(r, wave * per, min((wave + 1) * per, r.ntiles), 1, [&](uint32_t t, u32x4 raw) {
    float y[E];
    logits_of<DT>(r, t * kWave + lane, raw, y);
#pragma unroll
    for (uint32_t j = 0; j < E; ++j) sum += kept(y[j]);
  });
  sum = wave_sum_f64(sum);
  if (lane == 0) s.wave_f64[wave] = sum;
  __syncthreads();
  const double each = lane < W ? s.wave_f64[lane] : 0.0, total = wave_sum_f64(each);
  double rest = (double)a.u[b] * total;
  const uint32_t seg = (uint32_t)pick_lane(each, rest);
  draw_in_tiles<DT, W>(a, b, r, seg * per, min((seg + 1) * per, r.ntiles), rest, total, s, kept);
}

// Collects the logits of one bin; false if there are more than are ranked.
template <int DT, int W>
__device__ __forceinline__ bool collect_members(const Row& r, int bin, const float* blocks, uint32_t nblocks, float* members, SampleShared<W>& s) {
  constexpr uint32_t E = vec_elems<DT>();
  __syncthreads();
  if (threadIdx.x == 0) s.nmembers = 0;
  __syncthreads();
  const float floor = bin_floor(bin);
#pragma unroll 1
  for (uint32_t j = threadIdx.x / kBlockVecs; j < nblocks; j += W * kWave / kBlockVecs) {
    if (!(blocks[j] >= floor)) continue;
    const uint32_t i = j * kBlockVecs + threadIdx.x % kBlockVecs;
    float y[E];
    vec_unpack<DT>(vec_load<DT>(r.x, i, r.V), y);
#pragma unroll
    for (uint32_t e = 0; e < E; ++e) {
      if (!(y[e] > -kBinsBelow) || bin_of(__builtin_bit_cast(uint32_t, y[e])) != bin) continue;
      const uint32_t at = atomicAdd(&s.nmembers, 1u);
      if (at < kMostMembers) members[at] = y[e];
    }
  }
  __syncthreads();
  return s.nmembers <= kMostMembers;
}

template <int DT, int W>
__device__ __forceinline__ void draw_filtered(const SampleArgs& a, int64_t b, Row& r, int32_t k, float p, double min_p, unsigned char* lds,
                                              SampleShared<W>& s) {
  constexpr uint32_t E = vec_elems<DT>();
  constexpr int kThreads = W * kWave;
  constexpr bool kOne = DT == ESPO_BF16;    // one value per bin: its mass follows from its count
  const uint32_t lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  const uint32_t nblocks = r.ntiles * (kWave / kBlockVecs);
  uint32_t* count = (uint32_t*)lds;
  u64* mass = (u64*)(lds + (kBins + 3) / 4 * 16);
  float* blocks = (float*)(lds + a.lds_blocks);
  float* members = (float*)(lds + a.lds_members);
  const bool counts = k > 0 || (kOne && p > 0.0f), masses = !kOne && p > 0.0f;

  for (int i = threadIdx.x; i < kBins; i += kThreads) {
    count[i] = 0;
    if (masses) mass[i] = 0;
  }
  if (threadIdx.x == 0) s.first = 0xffffffffu, s.last = 0, s.found_bin = 0;
  __syncthreads();
  float m = kMaskedRow;
  double next_to_0 = 0.0;                   // mass of bf16 logits next to 0, relative to e^0
  stream(r, wave, r.ntiles, W, [&](uint32_t t, u32x4 raw) {
    float y[E];
    logits_of<DT>(r, t * kWave + lane, raw, y);
    float top = max_of<E>(y);
    m = fmaxf(m, top);
    ESPO_DPP_STEP("v_max_f32", top, "row_shr:1 row_mask:0xf bank_mask:0xf");
    ESPO_DPP_STEP("v_max_f32", top, "row_shr:2 row_mask:0xf bank_mask:0xf");
    ESPO_DPP_STEP("v_max_f32", top, "row_shr:4 row_mask:0xf bank_mask:0xf");
    ESPO_DPP_STEP("v_max_f32", top, "row_shr:8 row_mask:0xf bank_mask:0xf");
    if (lane % kBlockVecs == kBlockVecs - 1) blocks[t * (kWave / kBlockVecs) + lane / kBlockVecs] = top;
    if (counts) {
      if constexpr (kOne) {
        float low = y[0], least = fabsf(y[0]);
#pragma unroll
        for (uint32_t j = 1; j < E; ++j) low = fminf(low, y[j]), least = fminf(least, fabsf(y[j]));
        const bool all = __builtin_amdgcn_ballot_w64(!(low > -kBinsBelow)) == 0;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
          const uint32_t at = bins_of_pair<4>(raw[j]);
          if (all) {
            atomicAdd((uint32_t*)(lds + (at & 0xffffu)), 1u);
            atomicAdd((uint32_t*)(lds + (at >> 16)), 1u);
          } else {                          // masked logits would all wait for one counter
            if (y[2 * j] > -kBinsBelow) atomicAdd((uint32_t*)(lds + (at & 0xffffu)), 1u);
            if (y[2 * j + 1] > -kBinsBelow) atomicAdd((uint32_t*)(lds + (at >> 16)), 1u);
          }
        }
        if (p > 0.0f && __builtin_amdgcn_ballot_w64(least < 0x1p-10f) != 0) {
#pragma unroll 1
          for (uint32_t j = 0; j < E; ++j) {
            const float v = logit_in<DT>(raw, j);
            if (fabsf(v) < 0x1p-10f) next_to_0 += exp2_f64((double)v * r.c);
          }
        }
      } else {
#pragma unroll
        for (uint32_t j = 0; j < E; ++j)
          if (y[j] > -kBinsBelow) atomicAdd(&count[bin_of(__builtin_bit_cast(uint32_t, y[j]))], 1u);
      }
    }
    if (masses) {
#pragma unroll
      for (uint32_t j = 0; j < E; ++j) {
        if (!(y[j] > -kBinsBelow)) continue;
        const int bin = bin_of(__builtin_bit_cast(uint32_t, y[j]));
        const double rel = exp2_f64((double)(y[j] - bin_number(bin)) * r.c);
        atomicAdd(&mass[bin], (u64)(rel * kBinMass + 0.5));
      }
    }
  });
  const float top = block_max<W>(m, s);
  if (!(top > kMaskedRow)) {
    if (threadIdx.x == 0) store_result(a, b, -1, 0.0f);
    return;
  }
  r.m = (double)top;

  // the cut: logits of at least this are kept, as far as top-k and top-p go
  float cut = -3.402823466e38f;
  // The bins must hold all logits that have a say, a bin's mass must fit (numbers of a bin differ by 2^-7 relative), and e^(x / T) of the
  // logits next to 0 must be a number.
  bool known = (k == 0 && p == 0.0f) ||
               (top < kBinsBelow && (!masses || (double)top * r.inv_t < 300.0) && (p == 0.0f || r.inv_t < 300000.0) &&
                (p == 0.0f || k > 0 || ((double)top + kBinsBelow) * r.inv_t > 50.0));
  constexpr int kEach = (kBins - 2 + kThreads - 1) / kThreads;  // bins of a thread, from the top
  const int highest = kBins - 2 - (int)threadIdx.x * kEach;
  int kbin = 0;                             // bins below it are out by top-k
  if (known && k > 0) {
    uint32_t mine = 0, all;
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (highest - i > 0) mine += count[highest - i];
    uint32_t before = block_before<W>(mine, s.wave_u32, all);
    known = (uint32_t)k <= all;
    if (known) {
      if (before < (uint32_t)k && (uint32_t)k <= before + mine) {
#pragma unroll 1
        for (int i = 0; i < kEach; ++i) {
          const uint32_t c = highest - i > 0 ? count[highest - i] : 0;
          if (before + c >= (uint32_t)k) {
            s.found_bin = (uint32_t)(highest - i);
            s.above_count = before;
            break;
          }
          before += c;
        }
      }
      __syncthreads();
      kbin = (int)s.found_bin;
      if (kOne && kbin != kBinZero) {
        cut = bin_number(kbin);
      } else {
        const uint32_t rank = (uint32_t)k - s.above_count;  // within the bin, from 1
        known = collect_members<DT, W>(r, kbin, blocks, nblocks, members, s);
        if (known) {
          const uint32_t n = s.nmembers;
          for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
            uint32_t above = 0, level = 0;
            for (uint32_t j = 0; j < n; ++j) above += members[j] > members[i], level += members[j] == members[i];
            if (above < rank && rank <= above + level) s.cut_key = __builtin_bit_cast(uint32_t, members[i]);
          }
          if (threadIdx.x == 0) s.kept_mass = 0;
          __syncthreads();
          cut = __builtin_bit_cast(float, s.cut_key);
          if (p > 0.0f)
            for (uint32_t i = threadIdx.x; i < n; i += kThreads)
              if (members[i] >= cut) atomicAdd(&s.kept_mass, (u64)(r.weight(members[i]) * kFixed + 0.5));
          __syncthreads();
        }
      }
    }
  }
  if (known && p > 0.0f) {
    double zero = 0.0;
    if constexpr (kOne) {
      block_before<W>(next_to_0, s.wave_f64, zero);
      zero *= exp2_f64(-r.m * r.c);
      __syncthreads();
    }
    const bool ranked = k > 0 && !(kOne && kbin != kBinZero);  // bin kbin has been ranked for top-k
    double w[kEach], mine = 0.0, all;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int bin = highest - i;
      double n = 0.0;
      if (bin > 0) n = kOne ? (double)count[bin] : (double)mass[bin] * (1.0 / kBinMass);
      w[i] = n * r.weight(bin_number(bin));
      if (kOne && bin == kBinZero) w[i] = zero;
      if (bin < kbin) w[i] = 0.0;
      if (ranked && bin == kbin) w[i] = (double)s.kept_mass * (1.0 / kFixed);
      mine += w[i];
    }
    double before = block_before<W>(mine, s.wave_f64, all);
    const double target = (double)p * all;
    const uint32_t who = block_pick<W>(before, mine, kNoWeight, target, true, s);
    if (threadIdx.x == who) {
      bool done = false;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        if (done || !(w[i] > kNoWeight)) continue;
        s.found_bin = (uint32_t)(highest - i);
        s.rest = before;
        before += w[i];
        done = before >= target;
      }
    }
    __syncthreads();
    const int bin = (int)s.found_bin;
    const double above = s.rest;
    if (kOne && bin != kBinZero) {
      cut = bin_number(bin);
    } else {
      if (bin != kbin || k == 0) known = collect_members<DT, W>(r, bin, blocks, nblocks, members, s);
      if (known) {
        const uint32_t n = s.nmembers;
        u64* weights = (u64*)lds;           // over the bins
        if (threadIdx.x == 0) s.cut_key = 0xffffffffu;
        for (uint32_t i = threadIdx.x; i < n; i += kThreads) weights[i] = (u64)(r.weight(members[i]) * kFixed + 0.5);
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
          if (members[i] < cut) continue;   // out by top-k
          u64 higher = 0;
          for (uint32_t j = 0; j < n; ++j)
            if (members[j] > members[i]) higher += weights[j];
          if (higher == 0 || above + (double)higher * (1.0 / kFixed) < target) atomicMin(&s.cut_key, key_of(members[i]));
        }
        __syncthreads();
        const uint32_t key = s.cut_key;
        cut = __builtin_bit_cast(float, key >> 31 ? key & 0x7fffffffu : ~key);
      }
    }
  }
  if (!known) {
    draw_by_keys<DT, W>(a, b, r, k, p, min_p, lds, s);
    return;
  }

  // the blocks that reach the cut, in the order of the vocabulary, and their kept sums
  float least = cut;
  if (min_p > 0.0) {
    const float down = (float)(log2(min_p) / r.c);
    least = fmaxf(least, top + down - 1e-5f * (fabsf(top) + fabsf(down)) - 1e-30f);
  }
  uint32_t* visit = (uint32_t*)lds;
  double* sums = (double*)(lds + (nblocks + 3) / 4 * 16);
  const uint32_t range = (nblocks + kThreads - 1) / kThreads, from = threadIdx.x * range;
  uint32_t n = 0, nvisit;
  for (uint32_t j = from; j < min(from + range, nblocks); ++j) n += blocks[j] >= least && blocks[j] > kMaskedRow;
  __syncthreads();
  if (threadIdx.x == 0) s.first = 0xffffffffu, s.last = 0;
  uint32_t at = block_before<W>(n, s.wave_u32, nvisit);
  for (uint32_t j = from; j < min(from + range, nblocks); ++j)
    if (blocks[j] >= least && blocks[j] > kMaskedRow) visit[at++] = j;
  __syncthreads();
  const auto kept = [&](float x) {
    if (!(x >= cut) || !(x > kMaskedRow)) return 0.0;
    const double w = r.weight(x);
    return w >= min_p ? w : 0.0;
  };
  {
    constexpr uint32_t kStep = kThreads / kBlockVecs;
    const uint32_t sub = threadIdx.x % kBlockVecs;
    const auto load = [&](uint32_t j) {
      return j < nvisit ? __builtin_nontemporal_load((const u32x4*)(r.x + (size_t)min(visit[j] * kBlockVecs + sub, r.nvec - 1) * 16)) : vec_masked<DT>();
    };
    u32x4 cur[kAhead];
#pragma unroll
    for (int h = 0; h < kAhead; ++h) cur[h] = load(threadIdx.x / kBlockVecs + h * kStep);
#pragma unroll 1
    for (uint32_t j = threadIdx.x / kBlockVecs; j < nvisit; j += kAhead * kStep) {
      u32x4 nxt[kAhead];
#pragma unroll
      for (int h = 0; h < kAhead; ++h) nxt[h] = load(j + (kAhead + h) * kStep);
#pragma unroll
      for (int h = 0; h < kAhead; ++h) {
        const uint32_t q = j + h * kStep;
        if (q >= nvisit) break;
        float y[E];
        logits_of<DT>(r, visit[q] * kBlockVecs + sub, cur[h], y);
        uint32_t in = 0;                    // most vectors hold one kept logit or none
#pragma unroll
        for (uint32_t e = 0; e < E; ++e) in |= y[e] >= cut && y[e] > kMaskedRow ? 1u << e : 0u;
        double w = 0.0;
        for (; in != 0; in &= in - 1) w += kept(logit_in<DT>(cur[h], (uint32_t)__builtin_ctz(in)));
        w += dpp_f64<kDppRowShr1, 0xf>(w);
        w += dpp_f64<kDppRowShr2, 0xf>(w);
        w += dpp_f64<kDppRowShr4, 0xf>(w);
        w += dpp_f64<kDppRowShr8, 0xf>(w);
        if (sub == kBlockVecs - 1) sums[q] = w;
      }
#pragma unroll
      for (int h = 0; h < kAhead; ++h) cur[h] = nxt[h];
    }
  }
  __syncthreads();
  // the block that the draw falls into
  const uint32_t each = (nvisit + kThreads - 1) / kThreads, q0 = threadIdx.x * each;
  double mine = 0.0, total;
  for (uint32_t q = q0; q < min(q0 + each, nvisit); ++q) mine += sums[q];
  const double before = block_before<W>(mine, s.wave_f64, total);
  const double target = (double)a.u[b] * total;
  const uint32_t who = block_pick<W>(before, mine, kNoWeight, target, false, s);
  if (threadIdx.x == who) {
    double rest = target - before, left = rest;
    uint32_t q = q0;
    for (uint32_t i = q0; i < min(q0 + each, nvisit); ++i) {
      if (!(sums[i] > kNoWeight)) continue;
      q = i, left = rest;
      if (sums[i] > rest) break;
      rest -= sums[i];
    }
    s.found_bin = visit[q];
    s.rest = left;
  }
  __syncthreads();
  if (wave != 0) return;
  draw_in_vectors<DT>(a, b, r, s.found_bin * kBlockVecs + lane, lane < kBlockVecs, s.rest, total, kept);
}

template <int DT, int W, bool kFilters>
__global__ __launch_bounds__(W* kWave) void espo_sample_kernel(SampleArgs a) {
  __shared__ SampleShared<W> s;
  extern __shared__ __align__(16) unsigned char lds[];
  constexpr uint32_t E = vec_elems<DT>();
  const int64_t b = blockIdx.x;
  if (a.alive && !a.alive[b]) {
    if (threadIdx.x == 0) store_result(a, b, -1, 0.0f);
    return;
  }
  // beyond 1e25 the distribution is flat, and masked logits still are 10^5 times T below any other
  const float T = a.temperature ? fminf(a.temperature[b], 1e25f) : 1.0f;
  const uint32_t nvec = (a.V + E - 1) / E;
  Row r{a.logits + b * a.row_bytes, a.V, nvec, (nvec + kWave - 1) / kWave, 1.4426950408889634 / (double)T, 1.0 / (double)T, 0.0};
  if (!(T > 0.0f)) {
    greedy<DT, W>(a, b, r, s);
    return;
  }
  if constexpr (kFilters) {
    int32_t k = a.top_k ? a.top_k[b] : 0;
    float p = a.top_p ? a.top_p[b] : 0.0f;
    const float min_p = a.min_p ? fminf(a.min_p[b], 1.0f) : 0.0f;
    if (!(k > 0 && (uint32_t)k < a.V)) k = 0;
    if (!(p > 0.0f && p < 1.0f)) p = 0.0f;
    if (k > 0 || p > 0.0f || min_p > 0.0f) {
      draw_filtered<DT, W>(a, b, r, k, p, (double)min_p, lds, s);
      return;
    }
  }
  draw_plain<DT, W>(a, b, r, s);
}

// Dynamic LDS of a filtered draw: bins, then (over them) the blocks that are visited and their sums; the blocks' maxima; members.
template <int DT>
size_t filter_lds(int64_t V, uint32_t& blocks, uint32_t& members) {
  const size_t E = DT == ESPO_BF16 ? 8 : 4, ntiles = (V + kWave * E - 1) / (kWave * E), nblocks = ntiles * (kWave / kBlockVecs);
  size_t bins = (size_t)(kBins + 3) / 4 * 16 + (DT == ESPO_BF16 ? 0 : (size_t)kBins * 8), visited = (nblocks + 3) / 4 * 16 + nblocks * 8;
  size_t first = bins > visited ? bins : visited;
  if (first < (size_t)kLevelBins * 12) first = (size_t)kLevelBins * 12;
  first = (first + 15) / 16 * 16;
  blocks = (uint32_t)first;
  members = (uint32_t)(first + (nblocks + 3) / 4 * 16);
  return members + (size_t)kMostMembers * 4;
}

template <int DT, int W>
void launch(SampleArgs& a, int64_t B, hipStream_t stream) {
  if (a.top_k || a.top_p || a.min_p) {
    const size_t lds = filter_lds<DT>(a.V, a.lds_blocks, a.lds_members);
    hipLaunchKernelGGL((espo_sample_kernel<DT, W, true>), dim3((unsigned)B), dim3(W * kWave), lds, stream, a);
  } else {
    hipLaunchKernelGGL((espo_sample_kernel<DT, W, false>), dim3((unsigned)B), dim3(W * kWave), 0, stream, a);
  }
}

}  // namespace

int launch_sample(const void* logits, int dt, int64_t B, int64_t V, int64_t row_stride, const float* temperature, const int32_t* top_k,
                  const float* top_p, const float* min_p, const float* u, const uint8_t* alive, int32_t* tokens, float* logprob,
                  hipStream_t stream) {
  SampleArgs a{(const char*)logits, row_stride * (dt == ESPO_BF16 ? 2 : 4), (uint32_t)V, temperature, top_k, top_p, min_p, u, alive, tokens, logprob, 0, 0};
  const bool many = B > 256;
  if (dt == ESPO_BF16)
    many ? launch<ESPO_BF16, 8>(a, B, stream) : launch<ESPO_BF16, 16>(a, B, stream);
  else
    many ? launch<ESPO_F32, 8>(a, B, stream) : launch<ESPO_F32, 16>(a, B, stream);
  return hipGetLastError() == hipSuccess ? ESPO_OK : ESPO_EHIP;
}

}  // namespace espo
