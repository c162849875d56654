// espo_sample: a token per row from given random numbers, every row with its own temperature, top-k, top-p and min-p.
//
// With t_v = (x_v - m) / T and w_v = e^t_v, the kept tokens are those whose logit reaches a cut, the largest of what the three
// filters ask for; the token is the first, in the order of the vocabulary, at which the running sum of the kept weights exceeds
// u times their total.  Which token that is turns on sums of up to V weights: with V of 10^5 and a flat distribution two
// neighbouring sums differ by 10^-5 of the total, and the rounding errors of fp32 sums (10^-7) would move one draw in a hundred.  So
// weights and sums are doubles (a v_fma_f64 takes no longer than a v_fma_f32 here), and sums that are formed by atomics are integers
// (the order of additions then changes nothing).
//
// One workgroup per row, which is streamed once.  A row without filters leaves the sum of every chunk of four tiles; the chunk that the
// draw falls into is read again.  A filtered row leaves how many logits (and, of fp32 logits under top-p, how much mass) fall into
// each of 4355 bins, which are the bf16 numbers from 2^-10 to 128 of either sign with two for all beyond, and the largest logit of every block of 16
// vectors.  The bins say where the cut is: exactly so for bf16 logits, whose bins hold one value each, and up to one bin's
// members for fp32 logits, which are then collected and ranked.  Only blocks that reach the cut are read again, or, where those
// are many, the row.  Rows that the bins do not describe (a largest logit of 128 and more, a cut among logits of -128 and less or a nucleus
// that they have a share in, a bin with thousands of members, an fp32 nucleus whose largest logit is beyond 300 T, or 900 T below 0, or whose T is below
// 4e-4) find their cut by three levels of 2048 bins over the whole key, one pass over the row each.
//
// What follows the stream is a chain of short steps that run once per row, and what they cost is the fetching of their instructions: a first
// version that unrolled them took 7 us for each of cut, second reading and draw, at any batch size.  So they are loops, of one
// instance of each thing.
//
// What bounds it, and us a call on an MI355X at T = 1 where no other is named: large batches, LDS and double arithmetic per logit, not memory.
// V = 152064 bf16, B = 512: plain, T = 0.6, 445 rows alive, 36 (135 MB at 3.7 TB/s; a look-up of 8 bytes per logit, 36 % of LDS's cycles conflicts),
// nucleus of 0.7 60 (a count per logit besides, cut, second reading and draw).  Small ones, the chain of phases of one row: B = 64, settings of
// all kinds, 36 (11 the parts' pass, 26 joining, cut and draw); B = 100, V = 50003 f32, the same, 55 to 59 (a mass takes a power of 2 in double and an addition of
// 8 bytes in LDS, for each logit); B = 4, V = 32768 f32, plain 10.
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

constexpr int kChunk = 4;                   // tiles of a chunk, the unit of a pass that sums weights
constexpr int kBlockVecs = 16;              // vectors of a block: one row of 16 lanes, whose maximum takes four DPP steps
constexpr double kFixed = 8796093022208.0;  // 2^43: a weight of 1 as an integer; 2^20 of them stay below 2^63
constexpr double kNoWeight = 1e-250;        // weights below this count as none

// ---------------------------------------------------------------- bins of bf16 numbers
constexpr int kMagBelow = ((127 - 10) << 7) - 1;  // the bf16 number before 2^-10
constexpr int kMagSpan = 17 << 7;                 // numbers from 2^-10 to 128
constexpr int kBinZero = kMagSpan + 2;            // bin of everything next to 0
constexpr int kBins = 2 * kBinZero + 1;
constexpr int kBinLow = 1, kBinHigh = kBins - 2;  // of -128 and less (not masked), of 128 and more
constexpr float kBinsBelow = 128.0f;
constexpr size_t kCountBytes = (size_t)(kBins + 3) / 4 * 16;
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
// The smaller one of two numbers of 16 bits, in both halves.
__device__ __forceinline__ uint32_t min_of_pairs(uint32_t a, uint32_t b) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
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

// The integer nearest to w * scale, which is below 2^51: the low bits of the sum with 2^52.
__device__ __forceinline__ unsigned long long fixed_point(double w, double scale) {
  return __builtin_bit_cast(unsigned long long, fma(w, scale, 4503599627370496.0)) - 0x4330000000000000ull;
}

// What the workgroups of a split row leave for its draw: its blocks' maxima (or, without a filter, its chunks' sums and references), and
// of each workgroup its largest logit, its mass next to 0 and its bins.
struct PartRecord {
  double next_to_0;
  float m, pad;
};
constexpr uint32_t kMostParts = 8;
struct SplitLayout {
  char* base;
  size_t row, bins;  // bytes of a row, of a workgroup's bins
  uint32_t parts, front;
  __device__ __forceinline__ char* of(int64_t b) const { return base + (size_t)b * row; }
  __device__ __forceinline__ PartRecord* records(int64_t b) const { return (PartRecord*)(of(b) + front); }
  __device__ __forceinline__ char* part_bins(int64_t b, uint32_t part) const { return of(b) + front + parts * sizeof(PartRecord) + part * bins; }
};

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
  SplitLayout split;
};

struct Row : RowView {
  double c, inv_t, m;  // log2(e) / T, 1 / T, largest logit
  __device__ __forceinline__ double weight(float v) const { return exp2_f64(((double)v - m) * c); }
};

// Order of the logits as unsigned integers; both zeros are one value.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t key) { return __builtin_bit_cast(float, key >> 31 ? key & 0x7fffffffu : ~key); }

constexpr int kLevelBins = 2048;            // of a level of the search over whole keys: 11, 11 and 10 bits
// Logits of a bin that are ranked, each against all others.  (V = 152064 f32, B = 128, settings of all kinds: 518 us with 512 of them, because a few rows
// went to whole keys, 159 with these.)
constexpr int kMostMembers = 2048;
constexpr int kMostFew = 400;               // top-k up to this ranks the k largest of fp32 logits, with their bin's others
constexpr uint32_t kMostRounds = 8;         // of the workgroup over the blocks that are visited; beyond that the row is streamed again

template <int W>
struct SampleShared {
  double wave_f64[3][W];
  u64 found_mass, above_mass, kept_mass;
  double rest;
  float m[W];
  int2 picks[3][W];
  uint32_t at[W], wave_u32[W];
  uint32_t found_bin, above_count, nmembers, cut_key;
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
#pragma unroll 1
  for (int d = 1; d < kWave; d *= 2) {
    const u64 o = __shfl_up(v, d);
    if ((int)(threadIdx.x & (kWave - 1)) >= d) v += o;
  }
  return v;
}
__device__ __forceinline__ double lane_f64(double v, int lane) {  // the same lane in the whole wave
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane), __builtin_amdgcn_readlane(__double2loint(v), lane));
}

// The sum over the threads before this one, and over all of them; lds: W entries that a barrier has freed.
template <int W>
__device__ __forceinline__ uint32_t block_before(uint32_t v, uint32_t* lds, uint32_t& total) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  const uint32_t upto = wave_scan(v);
  if (lane == kWave - 1) lds[wave] = upto;
  __syncthreads();
  const uint32_t all = wave_scan(lane < W ? lds[lane] : 0u);
  total = (uint32_t)__builtin_amdgcn_readlane((int)all, kWave - 1);
  return upto - v + (wave > 0 ? (uint32_t)__builtin_amdgcn_readlane((int)all, wave - 1) : 0u);
}
template <int W>
__device__ __forceinline__ double block_before(double v, double* lds, double& total) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  const double upto = wave_scan(v);
  if (lane == kWave - 1) lds[wave] = upto;
  __syncthreads();
  const double all = wave_scan(lane < W ? lds[lane] : 0.0);
  total = lane_f64(all, kWave - 1);
  return upto - v + (wave > 0 ? lane_f64(all, wave - 1) : 0.0);
}

// The thread whose part [before, before + v) of a running sum holds `target`: the first with before + v beyond it (or, where `reach`,
// at it); the last with any part if rounding leaves none; kNone if there is no part at all (rows with NaN only).  The same in all
// threads.  (By ballots: LDS atomics on one word are turned into a loop over the lanes, 4 us here.)
constexpr uint32_t kNone = 0xffffffffu;
template <int W>
__device__ __forceinline__ uint32_t block_pick(double before, double v, double target, bool reach, int2* lds) {
  const double upto = before + v;
  const int lane = threadIdx.x & (kWave - 1);
  const bool any = v > kNoWeight;
  const uint64_t hit = __builtin_amdgcn_ballot_w64(any && (upto > target || (reach && upto == target))), some = __builtin_amdgcn_ballot_w64(any);
  const int base = (int)(threadIdx.x - lane);
  if (lane == 0) lds[threadIdx.x >> 6] = int2{hit ? base + (int)__builtin_ctzll(hit) : -1, some ? base + 63 - (int)__builtin_clzll(some) : -1};
  __syncthreads();
  const int2 w = lane < W ? lds[lane] : int2{-1, -1};
  const uint64_t hits = __builtin_amdgcn_ballot_w64(w.x >= 0), somes = __builtin_amdgcn_ballot_w64(w.y >= 0);
  if (hits) return (uint32_t)__builtin_amdgcn_readlane(w.x, (int)__builtin_ctzll(hits));
  return somes ? (uint32_t)__builtin_amdgcn_readlane(w.y, 63 - (int)__builtin_clzll(somes)) : kNone;
}

// Calls use(t, raw) for tiles first, first + step, ... below end, one after the other, with the next three on their way: a loop of little
// code.  Every load is in bounds (see stream_tiles); tile_logits masks what lies beyond V.
template <typename Use>
__device__ __forceinline__ void stream_ring(const RowView& r, uint32_t first, uint32_t end, uint32_t step, Use&& use) {
  const uint32_t lane = threadIdx.x & (kWave - 1);
  const auto load = [&](uint32_t t) {
    return __builtin_nontemporal_load((const u32x4*)(r.x + (size_t)min(min(t, end - 1) * kWave + lane, r.nvec - 1) * 16));
  };
  if (first >= end) return;
  u32x4 a = load(first), b = load(first + step), c = load(first + 2 * step), d = load(first + 3 * step);
#pragma unroll 1
  for (uint32_t t = first; t < end; t += step) {
    const u32x4 raw = a;
    a = b, b = c, c = d, d = load(t + 4 * step);
    use(t, raw);
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
      const u32x4 raw = vec_load<DT>(r.x, i, r.V);
#pragma unroll 1
      for (uint32_t j = 0; j < E; ++j) {
        const float x = logit_in<DT>(raw, j);
        const uint32_t key = key_of(x);
        if (!(x > kMaskedRow) || key < floor || (level > 0 && (key >> (shift + bits)) != prefix)) continue;
        const uint32_t bin = (key >> shift) & ((1u << bits) - 1);
        atomicAdd(&count[bin], 1u);
        atomicAdd(&mass[bin], fixed_point(r.weight(x), kFixed));
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
__device__ __forceinline__ void store_result(const SampleArgs& a, int64_t b, int32_t token, float logprob) {
  a.tokens[b] = token;
  if (a.logprob) a.logprob[b] = logprob;
}

// ln v for a normal number: the hardware's logarithm of the mantissa, and one step of Newton's method.
__device__ __forceinline__ double log_f64(double v) {
  const int e = ((__double2hiint(v) >> 20) & 0x7ff) - 1023;
  const double f = __hiloint2double(__double2hiint(v) - (int)((uint32_t)e << 20), __double2loint(v));  // in [1, 2)
  const double y = (double)__builtin_amdgcn_logf((float)f);
  return (y + (double)e) * 0.693147180559945309 + (f * exp2_f64(-y) - 1.0);
}

// What is kept of a row, as far as it is known.
struct Kept {
  float cut;    // logits of at least this
  double min_p; // weights of at least this
  __device__ __forceinline__ double weight(const Row& r, float x) const {
    if (!(x >= cut) || !(x > kMaskedRow)) return 0.0;
    const double w = r.weight(x);
    return w >= min_p ? w : 0.0;
  }
};

// The draw from n sums over `span` consecutive vectors each, the q-th of them starting at start(q): the one that the draw falls
// into, its vector, its logit.  A barrier has passed since the sums were stored.
template <int DT, int W, typename Start>
__device__ __forceinline__ void draw(const SampleArgs& a, int64_t b, const Row& r, const Kept& keep, const double* sums, uint32_t n, uint32_t span,
                                     SampleShared<W>& s, Start&& start) {
  constexpr uint32_t E = vec_elems<DT>(), kThreads = W * kWave;
  const uint32_t each = (n + kThreads - 1) / kThreads, q0 = threadIdx.x * each, q1 = min(q0 + each, n);
  double mine = 0.0, total;
#pragma unroll 1
  for (uint32_t q = q0; q < q1; ++q) mine += sums[q];
  double before = block_before<W>(mine, s.wave_f64[1], total);
  const double target = (double)a.u[b] * total;
  uint32_t who = block_pick<W>(before, mine, target, false, s.picks[1]);
  if (who == kNone) {
    if (threadIdx.x == 0) store_result(a, b, -1, 0.0f);
    return;
  }
  if (threadIdx.x == who) {
    double rest = target - before;
    uint32_t at = q0;
#pragma unroll 1
    for (uint32_t q = q0; q < q1; ++q) {
      const double w = sums[q];
      if (!(w > kNoWeight)) continue;
      at = q;
      s.rest = rest;
      if (w > rest) break;
      rest -= w;
    }
    s.found_bin = start(at);
  }
  __syncthreads();
  const uint32_t i = s.found_bin + threadIdx.x;
  const u32x4 raw = threadIdx.x < span ? vec_load<DT>(r.x, i, r.V) : vec_masked<DT>();
  const double ln_total = log_f64(total);   // while the load is on its way
  mine = 0.0;
  if (threadIdx.x < span) {
#pragma unroll 1
    for (uint32_t j = 0; j < E; ++j) mine += keep.weight(r, logit_in<DT>(raw, j));
  }
  double all;
  before = block_before<W>(mine, s.wave_f64[2], all);
  who = block_pick<W>(before, mine, s.rest, false, s.picks[2]);
  if (threadIdx.x != (who == kNone ? 0 : who)) return;
  int32_t token = -1;
  float x = 0.0f;
#pragma unroll 1
  for (uint32_t j = 0; j < E; ++j) {
    const float xj = logit_in<DT>(raw, j);
    const double w = keep.weight(r, xj);
    if (!(w > 0.0)) continue;
    token = (int32_t)(i * E + j), x = xj;
    before += w;
    if (before > s.rest) break;
  }
  store_result(a, b, token, (float)(((double)x - r.m) * r.inv_t - ln_total));
}

// Greedy: the first index of the largest logit.
template <int DT, int W>
__device__ __forceinline__ void greedy(const SampleArgs& a, int64_t b, const Row& r, SampleShared<W>& s) {
  constexpr uint32_t E = vec_elems<DT>();
  const uint32_t lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  float m = kMaskedRow;
  uint32_t at = 0xffffffffu;
  stream_ring(r, wave, r.ntiles, W, [&](uint32_t t, u32x4 raw) {
    float y[E];
    tile_logits<DT>(r, t, raw, y);
    const float top = max_of<E>(y);
    if (top > m) {
      m = top;
      const uint32_t i = t * kWave + lane;
#pragma unroll
      for (int j = E - 1; j >= 0; --j)
        if (y[j] == top) at = i * E + j;
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

// Chunks c0 .. c1 - 1 of a row: kChunk tiles each, a wave takes every W-th.  Calls use(t, raw) for a chunk's tiles and done(chunk) after them, and
// first, for the wave's first tile (the last chunk's where a wave has none), ready(t, raw); false of it ends the pass.
template <int W, typename Ready, typename Use, typename Done>
__device__ __forceinline__ void stream_chunks(const RowView& r, uint32_t c0, uint32_t c1, Ready&& ready, Use&& use, Done&& done) {
  const uint32_t lane = threadIdx.x & (kWave - 1);
  const auto load = [&](uint32_t c, uint32_t j) {
    return __builtin_nontemporal_load((const u32x4*)(r.x + (size_t)min((min(c, c1 - 1) * kChunk + j) * kWave + lane, r.nvec - 1) * 16));
  };
  uint32_t c = c0 + (threadIdx.x >> 6);
  u32x4 cur[kChunk], nxt[kChunk];
#pragma unroll
  for (uint32_t j = 0; j < kChunk; ++j) cur[j] = load(c, j);
  if (!ready(min(c, c1 - 1) * kChunk, cur[0])) return;
#pragma unroll 1
  for (; c < c1; c += W) {
#pragma unroll
    for (uint32_t j = 0; j < kChunk; ++j) nxt[j] = load(c + W, j);
#pragma unroll
    for (uint32_t j = 0; j < kChunk; ++j)
      if (c * kChunk + j < r.ntiles) use(c * kChunk + j, cur[j]);
    done(c);
#pragma unroll
    for (uint32_t j = 0; j < kChunk; ++j) cur[j] = nxt[j];
  }
}

// The kept sum of every chunk of bf16 logits, with weights from a table of all bins: 2^((x - base) c), 0 of what is not kept.  A look-up takes
// less than half the time of a power of 2 in double (B = 512, V = 152064, plain: 62 -> 41 us).  Logits next to 0, of which one bin
// holds many, are weighed one by one; those of -128 and less count as nothing, and the caller sees to it that they may.  Weights are relative to
// r.m, the row's largest logit, or if that is not known (`find`) to the largest one of the waves' first tiles, which r.m then becomes: any
// logit near the top does.  Returns the largest of what the thread's sums are: 0 nothing, 1 numbers, 2 no use (a logit of 128 or
// more, a low temperature, or first tiles that are masked throughout).
template <int W>
__device__ __forceinline__ float sum_by_table(Row& r, uint32_t c0, uint32_t c1, const Kept& keep, bool find, unsigned char* lds, double* sums, SampleShared<W>& s) {
  constexpr uint32_t E = vec_elems<ESPO_BF16>();
  double* table = (double*)lds;
  const auto weight = [&](float x) {
    const double w = exp2_f64(fmin(((double)x - r.m) * r.c, 1000.0));  // the table has entries above the largest logit too
    return x >= keep.cut && w >= keep.min_p ? w : 0.0;
  };
  float is = 0.0f;
  double sum = 0.0;
  stream_chunks<W>(
      r, c0, c1,
      [&](uint32_t t, u32x4 raw) {
        if (find) {
          float y[E];
          tile_logits<ESPO_BF16>(r, t, raw, y);
          const float top = block_max<W>(max_of<E>(y), s);
          r.m = (double)top;
          // Weights would not be numbers; or all is masked, and nothing is known of the largest logit that those of -128 and less have to be far below.
          if (!(((double)kBinsBelow - r.m) * r.c < 1000.0) || !(top > kMaskedRow)) {
            __syncthreads();                // the caller's block_max writes what this one has left
            is = 2.0f;
            return false;
          }
        }
#pragma unroll 1
        for (int i = threadIdx.x; i < kBins; i += W * kWave)
          table[i] = i > kBinLow && i < kBinHigh && i != kBinZero ? weight(bin_number(i)) : i == kBinHigh ? __builtin_huge_val() : 0.0;
        __syncthreads();
        return true;
      },
      [&](uint32_t t, u32x4 raw) {
        if (t + 1 >= r.ntiles) {
          float y[E];
          tile_logits<ESPO_BF16>(r, t, raw, y);
          raw = vec_pack<ESPO_BF16>(y);
        }
        uint32_t least = 0x7fff7fffu;       // of both halves, without the sign
        double w[E];
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
          const uint32_t at = bins_of_pair<8>(raw[j]);
          least = min_of_pairs(least, raw[j] & 0x7fff7fffu);
          w[2 * j] = *(const double*)(lds + (at & 0xffffu));
          w[2 * j + 1] = *(const double*)(lds + (at >> 16));
        }
        sum += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
        if (__builtin_amdgcn_ballot_w64((least & 0xffffu) <= kMagBelow || (least >> 16) <= kMagBelow) != 0) {
#pragma unroll 1
          for (uint32_t j = 0; j < E; ++j) {
            const float x = logit_in<ESPO_BF16>(raw, j);
            if (fabsf(x) < 0x1p-10f) sum += weight(x);
          }
        }
      },
      [&](uint32_t c) {
        sum = wave_sum_f64(sum);
        if (threadIdx.x % kWave == 0) sums[c] = sum;
        is = fmaxf(is, sum > 1e300 ? 2.0f : sum > kNoWeight ? 1.0f : 0.0f);
        sum = 0.0;
      });
  return is;
}

// The same with a power of 2 for every logit.  Without a filter the largest logit is not known before: the sums are then
// relative to a reference that follows the wave's largest logit only when that runs 2^500 ahead, and `refs` takes what each is relative to.
template <int DT, int W, bool kFiltered>
__device__ __forceinline__ float sum_by_powers(const Row& r, uint32_t c0, uint32_t c1, const Kept& keep, double* sums, float* refs) {
  constexpr uint32_t E = vec_elems<DT>();
  float m = kMaskedRow, ref = kFiltered ? (float)r.m : kMaskedRow, limit = kMaskedRow;
  double sum = 0.0;
  const float lead = (float)(500.0 / r.c);
  stream_chunks<W>(
      r, c0, c1, [](uint32_t, u32x4) { return true; },
      [&](uint32_t t, u32x4 raw) {
        float y[E];
        tile_logits<DT>(r, t, raw, y);
        if constexpr (!kFiltered) {
          const float top = max_of<E>(y);
          m = fmaxf(m, top);
          if (__builtin_amdgcn_ballot_w64(top > limit) != 0) {
            const float to = wave_max(m);
            sum = limit > kMaskedRow ? sum * exp2_f64(((double)ref - (double)to) * r.c) : 0.0;
            ref = to;
            limit = to + lead;
          }
        }
#pragma unroll
        for (uint32_t j = 0; j < E; ++j) {
          const double w = exp2_f64(((double)y[j] - (double)ref) * r.c);
          if (!kFiltered || (y[j] >= keep.cut && y[j] > kMaskedRow && w >= keep.min_p)) sum += w;
        }
      },
      [&](uint32_t c) {
        sum = wave_sum_f64(sum);
        if (threadIdx.x % kWave == 0) {
          sums[c] = sum;
          if (!kFiltered) refs[c] = ref;
        }
        sum = 0.0;
      });
  return m;
}

constexpr size_t kTableBytes = (size_t)(kBins + 1) / 2 * 16;

// No filter: the sums of chunks c0 .. c1 - 1 (sums[0] is chunk 0's), and what each is relative to.  Returns the largest of these references, which is
// the largest logit or near it; kMaskedRow if there is no logit.
template <int DT, int W>
__device__ __forceinline__ float sum_plain(Row& r, uint32_t c0, uint32_t c1, unsigned char* lds, double* sums, float* refs, SampleShared<W>& s) {
  const Kept all{-3.402823466e38f, 0.0};
  if constexpr (DT == ESPO_BF16) {
    const float is = block_max<W>(sum_by_table<W>(r, c0, c1, all, true, lds, sums, s), s);
    __syncthreads();
    if (is == 1.0f && (r.m + (double)kBinsBelow) * r.inv_t > 50.0) {
#pragma unroll 1
      for (uint32_t c = c0 + threadIdx.x; c < c1; c += W * kWave) refs[c] = (float)r.m;
      return (float)r.m;
    }
  }
  return block_max<W>(sum_by_powers<DT, W, false>(r, c0, c1, all, sums, refs), s);
}

// Its draw, once the sums are in LDS.
template <int DT, int W>
__device__ __forceinline__ void draw_plain(const SampleArgs& a, int64_t b, Row& r, float top, double* sums, const float* refs, SampleShared<W>& s) {
  const uint32_t chunks = (r.ntiles + kChunk - 1) / kChunk;
  if (!(top > kMaskedRow)) {
    if (threadIdx.x == 0) store_result(a, b, -1, 0.0f);
    return;
  }
  r.m = (double)top;
  __syncthreads();
#pragma unroll 1
  for (uint32_t c = threadIdx.x; c < chunks; c += W * kWave) sums[c] = refs[c] > kMaskedRow ? sums[c] * exp2_f64(((double)refs[c] - r.m) * r.c) : 0.0;
  __syncthreads();
  draw<DT, W>(a, b, r, Kept{-3.402823466e38f, 0.0}, sums, chunks, kChunk * kWave, s, [](uint32_t q) { return q * (kChunk * kWave); });
}

// Of many kept logits: the kept sum of every chunk, with the cut and the largest logit known.
template <int DT, int W>
__device__ __forceinline__ void draw_many(const SampleArgs& a, int64_t b, Row& r, const Kept& keep, unsigned char* lds, SampleShared<W>& s) {
  const uint32_t chunks = (r.ntiles + kChunk - 1) / kChunk;
  double* sums = (double*)(lds + (DT == ESPO_BF16 ? kTableBytes : 0));
  __syncthreads();                          // what was in LDS has been read
  if (DT == ESPO_BF16 && r.m < (double)kBinsBelow && keep.cut > -kBinsBelow)
    sum_by_table<W>(r, 0, chunks, keep, false, lds, sums, s);
  else
    sum_by_powers<DT, W, true>(r, 0, chunks, keep, sums, nullptr);
  __syncthreads();
  draw<DT, W>(a, b, r, keep, sums, chunks, kChunk * kWave, s, [](uint32_t q) { return q * (kChunk * kWave); });
}

// The cut of a row that the bins do not describe.
template <int DT, int W>
__device__ __forceinline__ float cut_by_keys(const Row& r, int32_t k, float p, unsigned char* lds, SampleShared<W>& s) {
  uint32_t floor = 0;
  u64 mass = 0;
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {    // the k largest (or the mass of the whole row), then the nucleus
    if (pass == 1 && p == 0.0f) continue;
    const Goal goal = pass == 1 ? Goal{false, 0, (double)p * (double)mass} : Goal{true, k > 0 ? (u64)k : (u64)r.V + 1, 0.0};
    const uint32_t cut = find_cut<DT, W>(r, floor, goal, lds, s, mass);
    if (pass == 1 || k > 0) floor = cut;
  }
  return of_key(floor);
}

// Collects the logits of one bin, or of it and all above; false if there are more than are ranked.
template <int DT, int W>
__device__ __forceinline__ bool collect_members(const Row& r, int bin, bool above, const float* blocks, uint32_t nblocks, float* members, SampleShared<W>& s) {
  constexpr uint32_t E = vec_elems<DT>(), kStep = W * kWave / kBlockVecs;
  __syncthreads();
  if (threadIdx.x == 0) s.nmembers = 0;
  __syncthreads();
  const float floor = bin_floor(bin);
#pragma unroll 1
  for (uint32_t j = threadIdx.x / kBlockVecs; j < nblocks; j += kAhead * kStep) {
    u32x4 raw[kAhead];
#pragma unroll
    for (int h = 0; h < kAhead; ++h) {      // those that reach the bin, all on their way at once
      const uint32_t q = j + h * kStep;
      raw[h] = vec_masked<DT>();
      if (q < nblocks && blocks[q] >= floor)
        raw[h] = __builtin_nontemporal_load((const u32x4*)(r.x + (size_t)min(q * kBlockVecs + threadIdx.x % kBlockVecs, r.nvec - 1) * 16));
    }
    uint32_t in = 0;
#pragma unroll
    for (int h = 0; h < kAhead; ++h) {
      float y[E];
      vec_unpack<DT>(raw[h], y);
#pragma unroll
      for (uint32_t e = 0; e < E; ++e) in |= y[e] >= floor ? 1u << (h * E + e) : 0u;
    }
    for (; in != 0; in &= in - 1) {
      const uint32_t at_bit = (uint32_t)__builtin_ctz(in), h = at_bit / E, e = at_bit % E;
      u32x4 v = raw[0];
#pragma unroll
      for (uint32_t q = 1; q < kAhead; ++q) v = h == q ? raw[q] : v;
      const float x = logit_in<DT>(v, e);
      const int at_bin = bin_of(__builtin_bit_cast(uint32_t, x));
      const bool beyond = ((j + h * kStep) * kBlockVecs + threadIdx.x % kBlockVecs) * E + e >= r.V;
      if (beyond || !(x > -kBinsBelow) || (above ? at_bin < bin : at_bin != bin)) continue;
      const uint32_t at = atomicAdd(&s.nmembers, 1u);
      if (at < kMostMembers) members[at] = x;
    }
  }
  __syncthreads();
  return s.nmembers <= kMostMembers;
}

// What the filters of a row ask for, and what a pass over it has to leave for them.
struct Filters {
  int32_t k;       // 0: off
  float p;         // 0: off
  double min_p;
  bool few;        // fp32 logits, and so small a k that all of the k largest are ranked
  bool counts, masses;
};

// The bins of tiles t0 .. t1 - 1, and the largest logit of each of their blocks.  Returns the thread's largest logit; next_to_0 is its share
// of the mass of bf16 logits next to 0, relative to e^0.
template <int DT, int W>
__device__ __forceinline__ float fill_bins(const Row& r, uint32_t t0, uint32_t t1, const Filters& f, unsigned char* lds, float* blocks, double& next_to_0) {
  constexpr uint32_t E = vec_elems<DT>();
  constexpr int kThreads = W * kWave;
  constexpr bool kOne = DT == ESPO_BF16;
  const uint32_t lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  uint32_t* count = (uint32_t*)lds;
  u64* mass = (u64*)(lds + kCountBytes);
  const bool counts = f.counts, masses = f.masses;
  const float p = f.p;
  if (counts || masses) {
#pragma unroll 1
    for (int i = threadIdx.x; i < kBins; i += kThreads) {
      count[i] = 0;
      if (masses) mass[i] = 0;
    }
    __syncthreads();
  }
  float m = kMaskedRow;
  bool any_low = false;
  stream_ring(r, t0 + wave, t1, W, [&](uint32_t t, u32x4 raw) {
    float y[E];
    tile_logits<DT>(r, t, raw, y);
    float top = max_of<E>(y);
    m = fmaxf(m, top);
    ESPO_DPP_STEP("v_max_f32", top, "row_shr:1 row_mask:0xf bank_mask:0xf");
    ESPO_DPP_STEP("v_max_f32", top, "row_shr:2 row_mask:0xf bank_mask:0xf");
    ESPO_DPP_STEP("v_max_f32", top, "row_shr:4 row_mask:0xf bank_mask:0xf");
    ESPO_DPP_STEP("v_max_f32", top, "row_shr:8 row_mask:0xf bank_mask:0xf");
    if (lane % kBlockVecs == kBlockVecs - 1) blocks[t * (kWave / kBlockVecs) + lane / kBlockVecs] = top;
    if (counts) {
      float low = y[0], least = fabsf(y[0]);
#pragma unroll
      for (uint32_t j = 1; j < E; ++j) low = fminf(low, y[j]), least = fminf(least, fabsf(y[j]));
      if (kOne && __builtin_amdgcn_ballot_w64(!(low > -kBinsBelow)) == 0) {
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
          const uint32_t at = bins_of_pair<4>(raw[j]);
          atomicAdd((uint32_t*)(lds + (at & 0xffffu)), 1u);
          atomicAdd((uint32_t*)(lds + (at >> 16)), 1u);
        }
      } else {                              // masked logits would all wait for one counter
#pragma unroll
        for (uint32_t j = 0; j < E; ++j)
          if (y[j] > kMaskedRow) atomicAdd(&count[bin_of(__builtin_bit_cast(uint32_t, y[j]))], 1u);
      }
      if (kOne && p > 0.0f && __builtin_amdgcn_ballot_w64(least < 0x1p-10f) != 0) {
#pragma unroll 1
        for (uint32_t j = 0; j < E; ++j) {
          const float v = logit_in<DT>(raw, j);
          if (fabsf(v) < 0x1p-10f && (t * kWave + lane) * E + j < r.V) next_to_0 += exp2_f64((double)v * r.c);
        }
      }
    }
    if (masses) {
#pragma unroll
      for (uint32_t j = 0; j < E; ++j) {
        any_low |= y[j] > kMaskedRow && !(y[j] > -kBinsBelow);
        if (!(y[j] > -kBinsBelow)) continue;
        const int bin = bin_of(__builtin_bit_cast(uint32_t, y[j]));
        const double rel = exp2_f64((double)(y[j] - bin_number(bin)) * r.c);
        atomicAdd(&mass[bin], fixed_point(rel, kBinMass));
      }
    }
  });
  if (any_low) atomicAdd(&mass[kBinLow], (u64)1);  // that there are any is all that counts
  return m;
}

// The sum over the parts of entry i behind `offset` of their bins, all loads on their way at once (one after the other: V = 152064 bf16, B = 64 nucleus
// of 0.7 27.4 us for 26.5, f32, B = 32 50.5 for 44.3).
template <typename T>
__device__ __forceinline__ T over_parts(const SplitLayout& split, int64_t b, size_t offset, uint32_t i) {
  T v[kMostParts], n{};
#pragma unroll
  for (uint32_t q = 0; q < kMostParts; ++q) v[q] = ((const T*)(split.part_bins(b, min(q, split.parts - 1)) + offset))[i];
#pragma unroll
  for (uint32_t q = 0; q < kMostParts; ++q) n += q < split.parts ? v[q] : T{};
  return n;
}

// The parts' bins and blocks put together in LDS; what fill_bins leaves of a whole row.
template <int DT, int W>
__device__ __forceinline__ float join_parts(const SplitLayout& split, int64_t b, const Row& r, const Filters& f, unsigned char* lds, float* blocks,
                                            double& next_to_0) {
  constexpr int kThreads = W * kWave;
  const uint32_t nblocks = r.ntiles * (kWave / kBlockVecs);
  const float* from = (const float*)split.of(b);
  const PartRecord* records = split.records(b);
  float m = kMaskedRow;
#pragma unroll 4
  for (uint32_t j = threadIdx.x; j < nblocks; j += kThreads) blocks[j] = from[j];
  if (threadIdx.x < split.parts) m = records[threadIdx.x].m, next_to_0 = records[threadIdx.x].next_to_0;
  // The counts, and behind them the masses, as 16 bytes at a time: sums of words without a carry, and of pairs with one.
  if (f.counts) {
#pragma unroll 1
    for (uint32_t i = threadIdx.x; i < kCountBytes / 16; i += kThreads) {
      ((u32x4*)lds)[i] = over_parts<u32x4>(split, b, 0, i);
    }
  }
  if (f.masses) {
#pragma unroll 1
    for (uint32_t i = threadIdx.x; i < kBins; i += kThreads) {
      ((u64*)(lds + kCountBytes))[i] = over_parts<u64>(split, b, kCountBytes, i);
    }
  }
  return m;                                 // (block_max has the barrier)
}

template <int DT, int W, bool kJoin>
__device__ __forceinline__ void draw_filtered(const SampleArgs& a, int64_t b, Row& r, const Filters& f, unsigned char* lds, SampleShared<W>& s) {
  constexpr uint32_t E = vec_elems<DT>();
  constexpr int kThreads = W * kWave;
  constexpr bool kOne = DT == ESPO_BF16;    // one value per bin: its mass follows from its count
  const int32_t k = f.k;
  const float p = f.p;
  const double min_p = f.min_p;
  const bool masses = f.masses;
  const uint32_t nblocks = r.ntiles * (kWave / kBlockVecs);
  uint32_t* count = (uint32_t*)lds;
  u64* mass = (u64*)(lds + kCountBytes);
  float* blocks = (float*)(lds + a.lds_blocks);
  float* members = (float*)(lds + a.lds_members);
  double next_to_0 = 0.0;
  float m = kMaskedRow;
  if constexpr (kJoin) {
    m = join_parts<DT, W>(a.split, b, r, f, lds, blocks, next_to_0);
  } else {
    m = fill_bins<DT, W>(r, 0, r.ntiles, f, lds, blocks, next_to_0);
  }
  const float top = block_max<W>(m, s);
  if (!(top > kMaskedRow)) {
    if (threadIdx.x == 0) store_result(a, b, -1, 0.0f);
    return;
  }
  r.m = (double)top;

  // the cut: logits of at least this are kept, as far as top-k and top-p go
  float cut = -3.402823466e38f;
  // The bins must hold all logits that have a say, and e^(x / T) of the logits next to 0 must be a number.  A bin's mass must fit and count: its
  // members lie within 2^-7 of its number, relative to that, or within 2^-10 of 0.  Above 0 the number is the bin's least: none weighs more than
  // e^(300 / 128) = 10.4 times what it does, and 2^19 of them in units of 2^-40 stay below 2^63.  Below 0 it is the largest: those
  // near the top weigh e^(-900 / 128) = 1 / 1130 at least, and half a unit of each is 5e-10 of the mass.
  const double far = fmax(fmax((double)top, 0.125), -1.0 / 3.0 * (double)top);
  bool known = (k == 0 && p == 0.0f) || (top < kBinsBelow && (!masses || far * r.inv_t < 300.0) && (p == 0.0f || r.inv_t < 300000.0));
  constexpr int kEach = (kBinHigh + kThreads - 1) / kThreads;  // bins of a thread, from the top
  const int highest = kBinHigh - (int)threadIdx.x * kEach, lowest = max(highest - kEach + 1, kBinLow);
  int kbin = 0;                             // bins below it are out by top-k
  bool ranked = false;                      // and it has been ranked for top-k: kept_mass is the mass of what is left of it
  if (known && k > 0) {
    uint32_t mine = 0, all;
#pragma unroll 1
    for (int i = highest; i >= lowest; --i) mine += count[i];
    uint32_t before = block_before<W>(mine, s.wave_u32, all);
    uint32_t rank = all;                    // of the k-th largest among the members, from 1
    if ((uint32_t)k <= all) {
      if (before < (uint32_t)k && (uint32_t)k <= before + mine) {
        int i = highest;
#pragma unroll 1
        for (;; --i) {
          const uint32_t c = count[i];
          if (before + c >= (uint32_t)k || i <= lowest) break;
          before += c;
        }
        s.found_bin = (uint32_t)i;
        s.above_count = before;
      }
      __syncthreads();
      kbin = (int)s.found_bin;
      known = kbin != kBinLow;
      rank = (uint32_t)k - (f.few ? 0 : s.above_count);
      ranked = known && !(kOne && kbin != kBinZero);
      if (known && !ranked) cut = bin_number(kbin);
    } else if (f.few) {                     // fewer logits than k: they are all members
      known = count[kBinLow] == 0;
      kbin = kBinLow + 1;
      ranked = known;
    }
    if (ranked) {
      ranked = known = collect_members<DT, W>(r, kbin, f.few, blocks, nblocks, members, s);
      if (known) {
        const uint32_t n = s.nmembers;
        if (threadIdx.x == 0) s.kept_mass = 0;
#pragma unroll 1
        for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
          uint32_t above = 0, level = 0;
          const float mine = members[i];
#pragma unroll 8
          for (uint32_t j = 0; j < n; ++j) above += members[j] > mine, level += members[j] == mine;
          if (above < rank && rank <= above + level) s.cut_key = __builtin_bit_cast(uint32_t, mine);
        }
        __syncthreads();
        cut = __builtin_bit_cast(float, s.cut_key);
        if (p > 0.0f) {
#pragma unroll 1
          for (uint32_t i = threadIdx.x; i < n; i += kThreads)
            if (members[i] >= cut) atomicAdd(&s.kept_mass, fixed_point(r.weight(members[i]), kFixed));
        }
        __syncthreads();
      }
    }
  }
  bool rank_mass = false;                   // the nucleus ends among the members
  double above = 0.0, target = 0.0;         // their mass from the top: what lies above them, and where the nucleus ends
  if (known && p > 0.0f && f.few) {
    rank_mass = true;
    target = (double)p * (double)s.kept_mass * (1.0 / kFixed);
  } else if (known && p > 0.0f) {
    // logits of -128 and less: there are none, or top-k leaves none, or they weigh nothing
    known = kbin > kBinLow || ((double)top + kBinsBelow) * r.inv_t > 50.0 || (kOne ? count[kBinLow] == 0 : mass[kBinLow] == 0);
  }
  if (known && p > 0.0f && !f.few) {
    double zero = 0.0;
    if constexpr (kOne) {
      block_before<W>(next_to_0, s.wave_f64[1], zero);
      zero = zero > 0.0 ? zero * exp2_f64(-r.m * r.c) : 0.0;
    }
    const auto bin_mass = [&](int bin) {
      double n = kOne ? (double)count[bin] : (double)mass[bin] * (1.0 / kBinMass);
      // by a select: above the largest logit, where bins are empty, a weight may be beyond the range of exp2_f64, and no number
      n = n > 0.0 ? n * r.weight(bin_number(bin)) : 0.0;
      if (kOne && bin == kBinZero) n = zero;
      if (ranked && bin == kbin) n = (double)s.kept_mass * (1.0 / kFixed);
      return bin < kbin ? 0.0 : n;
    };
    double mine = 0.0, before = 0.0;
    uint32_t who = threadIdx.x;
#pragma unroll 1
    for (int round = 0; round < 2; ++round) {  // the thread's mass; then, in the thread that the target falls to, its bin
      if (threadIdx.x == who) {
        double upto = before;
#pragma unroll 1
        for (int i = highest; i >= lowest; --i) {
          if (__builtin_amdgcn_ballot_w64(kOne ? count[i] != 0 : mass[i] != 0) == 0) continue;
          const double w = bin_mass(i);
          if (round == 0) {
            mine += w;
          } else if (w > kNoWeight) {
            s.found_bin = (uint32_t)i;
            s.rest = upto;
            upto += w;
            if (upto >= target) break;
          }
        }
      }
      if (round == 0) {
        double all;
        before = block_before<W>(mine, s.wave_f64[0], all);
        target = (double)p * all;
        who = block_pick<W>(before, mine, target, true, s.picks[0]);
      }
    }
    __syncthreads();
    const int bin = (int)s.found_bin;
    above = s.rest;
    if (kOne && bin != kBinZero) {
      cut = bin_number(bin);
    } else {
      rank_mass = true;
      if (!ranked || bin != kbin) known = collect_members<DT, W>(r, bin, false, blocks, nblocks, members, s);
    }
  }
  if (known && rank_mass) {
    const uint32_t n = s.nmembers;
    u64* weights = (u64*)lds;               // over the bins
    __syncthreads();
    if (threadIdx.x == 0) s.cut_key = 0xffffffffu;
#pragma unroll 1
    for (uint32_t i = threadIdx.x; i < n; i += kThreads) weights[i] = fixed_point(r.weight(members[i]), kFixed);
    __syncthreads();
#pragma unroll 1
    for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
      if (members[i] < cut) continue;       // out by top-k
      const float mine = members[i];
      u64 higher = 0;
#pragma unroll 8
      for (uint32_t j = 0; j < n; ++j) higher += members[j] > mine ? weights[j] : 0;
      if (higher == 0 || above + (double)higher * (1.0 / kFixed) < target) atomicMin(&s.cut_key, key_of(members[i]));
    }
    __syncthreads();
    cut = of_key(s.cut_key);
  }
  if (!known) cut = cut_by_keys<DT, W>(r, k, p, lds, s);
  const Kept keep{cut, min_p};

  // the blocks that reach the cut, in the order of the vocabulary, and their kept sums
  float least = cut;
  if (min_p > 0.0) {
    const float down = (float)(log_f64(min_p) / r.inv_t);
    least = fmaxf(least, top + down - 1e-5f * (fabsf(top) + fabsf(down)) - 1e-30f);
  }
  if (known) {
    uint32_t* visit = (uint32_t*)lds;
    double* sums = (double*)(lds + (nblocks + 3) / 4 * 16);
    const uint32_t range = (nblocks + kThreads - 1) / kThreads, from = threadIdx.x * range, to = min(from + range, nblocks);
    uint32_t n = 0, nvisit;
#pragma unroll 1
    for (uint32_t j = from; j < to; ++j) n += blocks[j] >= least && blocks[j] > kMaskedRow;
    __syncthreads();
    uint32_t at = block_before<W>(n, s.wave_u32, nvisit);
    if (nvisit <= kThreads / kBlockVecs * kMostRounds) {
#pragma unroll 1
      for (uint32_t j = from; j < to; ++j)
        if (blocks[j] >= least && blocks[j] > kMaskedRow) visit[at++] = j;
      __syncthreads();
      const uint32_t sub = threadIdx.x % kBlockVecs;
#pragma unroll 1
      for (uint32_t q = threadIdx.x / kBlockVecs; q < nvisit; q += kThreads / kBlockVecs) {
        const u32x4 raw = vec_load<DT>(r.x, visit[q] * kBlockVecs + sub, r.V);
        float y[E];
        vec_unpack<DT>(raw, y);
        uint32_t in = 0;                    // most vectors hold one kept logit or none
#pragma unroll
        for (uint32_t e = 0; e < E; ++e) in |= y[e] >= least ? 1u << e : 0u;
        double w = 0.0;
        for (; in != 0; in &= in - 1) w += keep.weight(r, logit_in<DT>(raw, (uint32_t)__builtin_ctz(in)));
        w += dpp_f64<kDppRowShr1, 0xf>(w);
        w += dpp_f64<kDppRowShr2, 0xf>(w);
        w += dpp_f64<kDppRowShr4, 0xf>(w);
        w += dpp_f64<kDppRowShr8, 0xf>(w);
        if (sub == kBlockVecs - 1) sums[q] = w;
      }
      __syncthreads();
      draw<DT, W>(a, b, r, keep, sums, nvisit, kBlockVecs, s, [&](uint32_t q) { return visit[q] * kBlockVecs; });
      return;
    }
  }
  draw_many<DT, W>(a, b, r, keep, lds, s);
}

// A row's settings.
struct RowPlan {
  float T;
  Filters f;
  __device__ __forceinline__ bool is_greedy() const { return !(T > 0.0f); }
  __device__ __forceinline__ bool is_plain() const { return f.k == 0 && f.p == 0.0f && !(f.min_p > 0.0); }
};
template <int DT>
__device__ __forceinline__ RowPlan row_plan(const SampleArgs& a, int64_t b) {
  RowPlan w;
  // beyond 1e25 the distribution is flat, and masked logits still are 10^5 times T below any other
  w.T = a.temperature ? fminf(a.temperature[b], 1e25f) : 1.0f;
  const int32_t k = a.top_k ? a.top_k[b] : 0;
  const float p = a.top_p ? a.top_p[b] : 0.0f;
  w.f.k = k > 0 && (uint32_t)k < a.V ? k : 0;
  w.f.p = p > 0.0f && p < 1.0f ? p : 0.0f;
  w.f.min_p = a.min_p ? (double)fminf(a.min_p[b], 1.0f) : 0.0;
  w.f.counts = w.f.k > 0 || (DT == ESPO_BF16 && w.f.p > 0.0f);
  w.f.few = DT != ESPO_BF16 && w.f.k > 0 && w.f.k <= kMostFew;
  w.f.masses = DT != ESPO_BF16 && w.f.p > 0.0f && !w.f.few;
  return w;
}
template <int DT>
__device__ __forceinline__ Row row_of(const SampleArgs& a, int64_t b, float T) {
  return Row{row_view<DT>(a.logits + b * a.row_bytes, a.V), 1.4426950408889634 / (double)T, 1.0 / (double)T, 0.0};
}

// kJoin: the passes over the row have been made by espo_sample_part_kernel.
template <int DT, int W, bool kFilters, bool kJoin>
__global__ __launch_bounds__(W* kWave) void espo_sample_kernel(SampleArgs a) {
  __shared__ SampleShared<W> s;
  extern __shared__ __align__(16) unsigned char lds[];
  const int64_t b = blockIdx.x;
  if (a.alive && !a.alive[b]) {
    if (threadIdx.x == 0) store_result(a, b, -1, 0.0f);
    return;
  }
  const RowPlan w = row_plan<DT>(a, b);
  Row r = row_of<DT>(a, b, w.T);
  if (w.is_greedy()) {
    greedy<DT, W>(a, b, r, s);
    return;
  }
  if constexpr (kFilters) {
    if (!w.is_plain()) {
      if (threadIdx.x == 0) s.found_bin = 0;  // where NaN leaves nothing to be found
      draw_filtered<DT, W, kJoin>(a, b, r, w.f, lds, s);
      return;
    }
  }
  const uint32_t chunks = (r.ntiles + kChunk - 1) / kChunk;
  double* sums = (double*)(lds + (DT == ESPO_BF16 ? kTableBytes : 0));
  float* refs = (float*)(sums + chunks);
  float top;
  if constexpr (kJoin) {
    const double* from = (const double*)a.split.of(b);
    const float* from_refs = (const float*)(from + chunks);
#pragma unroll 1
    for (uint32_t c = threadIdx.x; c < chunks; c += W * kWave) sums[c] = from[c], refs[c] = from_refs[c];
    top = block_max<W>(threadIdx.x < a.split.parts ? a.split.records(b)[threadIdx.x].m : kMaskedRow, s);
  } else {
    top = sum_plain<DT, W>(r, 0, chunks, lds, sums, refs, s);
  }
  draw_plain<DT, W>(a, b, r, top, sums, refs, s);
}

// One of the workgroups that a row is split over where there are few rows: its share of the row's chunks.
constexpr int kPartWaves = 16;
template <int DT, bool kFilters>
__global__ __launch_bounds__(kPartWaves* kWave) void espo_sample_part_kernel(SampleArgs a) {
  constexpr int W = kPartWaves, kThreads = W * kWave;
  __shared__ SampleShared<W> s;
  extern __shared__ __align__(16) unsigned char lds[];
  const uint32_t parts = a.split.parts, part = blockIdx.x % parts;
  const int64_t b = blockIdx.x / parts;
  if (a.alive && !a.alive[b]) return;
  const RowPlan w = row_plan<DT>(a, b);
  if (w.is_greedy()) return;                // its draw reads the row itself
  Row r = row_of<DT>(a, b, w.T);
  const uint32_t chunks = (r.ntiles + kChunk - 1) / kChunk, each = (chunks + parts - 1) / parts, c0 = part * each, c1 = min(c0 + each, chunks);  // at least 8 chunks a part, 8 parts at most: none is empty
  PartRecord* record = a.split.records(b) + part;
  if constexpr (kFilters) {
    if (!w.is_plain()) {
      const uint32_t per = kChunk * (kWave / kBlockVecs), t1 = min(c1 * kChunk, r.ntiles);
      float* blocks = (float*)(lds + a.lds_blocks);  // of the whole row, as far as it is this workgroup's
      double next_to_0 = 0.0, all;
      const float top = block_max<W>(fill_bins<DT, W>(r, c0 * kChunk, t1, w.f, lds, blocks, next_to_0), s);
      block_before<W>(next_to_0, s.wave_f64[0], all);
      if (threadIdx.x == 0) *record = PartRecord{all, top, 0.0f};
      float* to = (float*)a.split.of(b);
      for (uint32_t j = c0 * per + threadIdx.x; j < t1 * (kWave / kBlockVecs); j += kThreads) to[j] = blocks[j];
      const uint32_t first = w.f.counts ? 0 : kCountBytes / 16, last = (uint32_t)(w.f.masses ? a.split.bins : w.f.counts ? kCountBytes : 0) / 16;
      for (uint32_t i = first + threadIdx.x; i < last; i += kThreads) ((u32x4*)a.split.part_bins(b, part))[i] = ((const u32x4*)lds)[i];
      return;
    }
  }
  double* sums = (double*)a.split.of(b);
  const float top = sum_plain<DT, W>(r, c0, c1, lds, sums, (float*)(sums + chunks), s);
  if (threadIdx.x == 0) *record = PartRecord{0.0, top, 0.0f};
}

// Dynamic LDS of a draw without filters: the weights of all bins, the chunks' sums and references.
template <int DT>
size_t plain_lds(int64_t V) {
  const size_t tile = kWave * vec_elems<DT>(), chunks = (V + tile * kChunk - 1) / (tile * kChunk);
  return (DT == ESPO_BF16 ? kTableBytes : 0) + (chunks * 12 + 15) / 16 * 16;
}

// Of a filtered one: bins, then (over them) the blocks that are visited and their sums, or the chunks' sums; the blocks' maxima; members.
template <int DT>
size_t filter_lds(int64_t V, uint32_t& blocks, uint32_t& members) {
  const size_t E = vec_elems<DT>(), ntiles = (V + kWave * E - 1) / (kWave * E), nblocks = ntiles * (kWave / kBlockVecs);
  const size_t bins = kCountBytes + (DT == ESPO_BF16 ? 0 : (size_t)kBins * 8), visited = (nblocks + 3) / 4 * 16 + nblocks * 8;
  size_t first = (size_t)kLevelBins * 12;
  for (size_t n : {bins, visited, plain_lds<DT>(V)}) first = n > first ? n : first;
  first = (first + 15) / 16 * 16;
  blocks = (uint32_t)first;
  members = (uint32_t)(first + (nblocks + 3) / 4 * 16);
  return members + (size_t)kMostMembers * 4;
}

// Workgroups that a row is split over: as many as the idle compute units allow, of enough tiles each.  A draw without filters gains from
// 32 tiles each on (two per wave), bf16 logits in rows of 256 tiles; a filtered one, whose parts hand their bins on, in
// rows of 256 tiles and from three parts of 64 tiles on.  Of fp32 logits under top-p, which take longest, three parts pay from 192 tiles on, two from 512.
// us, whole rows / split, at T = 1:
//   V = 152064 bf16  plain           B = 1 21.5 / 14.7   64 23.8 / 18.5   128 24.5 / 22.4
//                    nucleus of 0.7  B = 1 25.6 / 21.7   64 29.5 / 28.1   128 30.3 / 31.5 (two parts: not taken)
//   V = 152064 f32   plain           B = 32 32.8 / 14.2
//                    nucleus of 0.7  B = 32 83 / 44      128 89 / 74 (two parts)
//   V = 50003 bf16   plain           B = 32 14.7 / 16.1 (98 tiles: not taken)
//                    nucleus of 0.7  B = 32 18.5 / 21.0 (not taken)
//   V = 50003 f32    nucleus of 0.7  B = 16 36.3 / 30.9  64 37.1 / 35.8   100 38.2 / 39.2 (two parts: not taken)
//   V = 32768 f32    plain           B = 4 11.5 / 10.3
//                    top-k 50        B = 4 16.1 / 18.8 (two parts: not taken)
// Greedy rows are read by one workgroup all the same.
constexpr int64_t kComputeUnits = 256;
enum Draws { kPlainDraws, kFilteredDraws, kNucleusDraws };  // without filters, with some, with top-p among them
template <int DT>
uint32_t parts_of(int64_t B, int64_t V, Draws draws) {
  const bool filters = draws != kPlainDraws, masses = DT != ESPO_BF16 && draws == kNucleusDraws;
  const int64_t tiles = V / (kWave * vec_elems<DT>());
  if (V > (1 << 19) || ((filters || DT == ESPO_BF16) && tiles < (masses ? 192 : 256))) return 1;
  int64_t n = kComputeUnits / B;
  if (n > tiles / (filters ? 64 : 32)) n = tiles / (filters ? 64 : 32);
  if (n > kMostParts) n = kMostParts;
  return n < (filters && !(masses && tiles >= 512) ? 3 : 2) ? 1u : (uint32_t)n;
}

template <int DT>
SplitLayout split_layout(int64_t B, int64_t V, Draws draws) {
  const size_t tile = kWave * vec_elems<DT>(), ntiles = (V + tile - 1) / tile, chunks = (ntiles + kChunk - 1) / kChunk;
  size_t front = ntiles * (kWave / kBlockVecs) * 4;
  if (front < chunks * 12) front = chunks * 12;
  front = (front + 15) / 16 * 16;
  const size_t bins = draws != kPlainDraws ? kCountBytes + (DT == ESPO_BF16 ? 0 : (size_t)(kBins + 1) / 2 * 16) : 0;
  SplitLayout l{nullptr, 0, bins, parts_of<DT>(B, V, draws), (uint32_t)front};
  l.row = (front + l.parts * (sizeof(PartRecord) + l.bins) + 255) / 256 * 256;
  return l;
}

template <int DT, bool kFilters>
void launch(SampleArgs& a, int64_t B, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  const size_t lds = kFilters ? filter_lds<DT>(a.V, a.lds_blocks, a.lds_members) : plain_lds<DT>(a.V);
  a.split = split_layout<DT>(B, a.V, a.top_p ? kNucleusDraws : kFilters ? kFilteredDraws : kPlainDraws);
  if (a.split.parts > 1 && workspace && workspace_bytes >= (size_t)B * a.split.row && (uintptr_t)workspace % 16 == 0) {
    a.split.base = (char*)workspace;
    hipLaunchKernelGGL((espo_sample_part_kernel<DT, kFilters>), dim3((unsigned)(B * a.split.parts)), dim3(kPartWaves * kWave), lds, stream, a);
    hipLaunchKernelGGL((espo_sample_kernel<DT, 16, kFilters, true>), dim3((unsigned)B), dim3(16 * kWave), lds, stream, a);
  } else if (B <= kComputeUnits) {
    hipLaunchKernelGGL((espo_sample_kernel<DT, 16, kFilters, false>), dim3((unsigned)B), dim3(16 * kWave), lds, stream, a);
  } else {
    hipLaunchKernelGGL((espo_sample_kernel<DT, 8, kFilters, false>), dim3((unsigned)B), dim3(8 * kWave), lds, stream, a);
  }
}

template <int DT>
void launch(SampleArgs& a, int64_t B, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (a.top_k || a.top_p || a.min_p)
    launch<DT, true>(a, B, workspace, workspace_bytes, stream);
  else
    launch<DT, false>(a, B, workspace, workspace_bytes, stream);
}

}  // namespace

size_t sample_workspace(int dt, int64_t B, int64_t V) {
  size_t most = 0;
  for (Draws draws : {kPlainDraws, kFilteredDraws, kNucleusDraws}) {
    const SplitLayout l = dt == ESPO_BF16 ? split_layout<ESPO_BF16>(B, V, draws) : split_layout<ESPO_F32>(B, V, draws);
    if (l.parts > 1 && (size_t)B * l.row > most) most = (size_t)B * l.row;
  }
  return most;
}

int launch_sample(const void* logits, int dt, int64_t B, int64_t V, int64_t row_stride, const float* temperature, const int32_t* top_k,
                  const float* top_p, const float* min_p, const float* u, const uint8_t* alive, int32_t* tokens, float* logprob,
                  void* workspace, size_t workspace_bytes, hipStream_t stream) {
  SampleArgs a{(const char*)logits, row_stride * (dt == ESPO_BF16 ? 2 : 4), (uint32_t)V, temperature, top_k, top_p, min_p, u, alive, tokens, logprob, 0, 0, {}};
  if (dt == ESPO_BF16)
    launch<ESPO_BF16>(a, B, workspace, workspace_bytes, stream);
  else
    launch<ESPO_F32>(a, B, workspace, workspace_bytes, stream);
  return hipGetLastError() == hipSuccess ? ESPO_OK : ESPO_EHIP;
}

}  // namespace espo
