// Device-side access to rows of logits, 16 bytes at a time, and the softmax sum of a row over one workgroup.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/espo.h"
#include "espo_device.h"

namespace espo {

// Logits at or below this are masked like -inf, whatever they are filled with.
constexpr float kMaskedRow = -1e30f;
// Exponents (to base 2) are held above this where they are multiplied by their own power: 2^-200 is 0 in fp32, and so is the product.
constexpr float kLeastExponent = -200.0f;

template <int DT>
constexpr int vec_elems() { return DT == ESPO_BF16 ? 8 : 4; }  // logits in 16 bytes
template <int DT>
constexpr int logit_bytes() { return DT == ESPO_BF16 ? 2 : 4; }

template <int DT>
__device__ __forceinline__ void vec_unpack(u32x4 r, float x[vec_elems<DT>()]) {
  if constexpr (DT == ESPO_BF16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __builtin_bit_cast(float, r[i] << 16);
      x[2 * i + 1] = __builtin_bit_cast(float, r[i] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = r[i];  // a vector's element as the operand of a bit cast is its element 0
      x[i] = __builtin_bit_cast(float, w);
    }
  }
}

// Logit j of a vector.
template <int DT>
__device__ __forceinline__ float logit_in(u32x4 raw, uint32_t j) {
  const uint32_t q = DT == ESPO_BF16 ? j >> 1 : j;
  uint32_t w = raw[0];
#pragma unroll
  for (uint32_t i = 1; i < 4; ++i) {
    const uint32_t wi = raw[i];
    w = q == i ? wi : w;
  }
  if constexpr (DT == ESPO_BF16) w = j & 1 ? w & 0xffff0000u : w << 16;
  return __builtin_bit_cast(float, w);
}

// Rounded once, to the nearest even.
template <int DT>
__device__ __forceinline__ u32x4 vec_pack(const float x[vec_elems<DT>()]) {
  u32x4 r;
  if constexpr (DT == ESPO_BF16) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x[2 * i], x[2 * i + 1]}, bf16x2));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(uint32_t, x[i]);
  }
  return r;
}

// The 16 bytes of a vector that holds no logit: all masked.
template <int DT>
__device__ __forceinline__ u32x4 vec_masked() {
  constexpr uint32_t w = DT == ESPO_BF16 ? 0xFF80FF80u : 0xFF800000u;
  return u32x4{w, w, w, w};
}

// Vector `i` of a row of V logits; what lies at or beyond V (a row's last 16 bytes) becomes masked.  Rows start at multiples of 16 bytes
// and so do their pitches, so that the 16 bytes that a row ends in belong to the row's own pitch.
template <int DT>
__device__ __forceinline__ u32x4 vec_load(const char* row, uint32_t i, uint32_t V) {
  constexpr uint32_t E = vec_elems<DT>();
  if (i * E >= V) return vec_masked<DT>();
  u32x4 r = __builtin_nontemporal_load((const u32x4*)(row + (size_t)i * 16));
  const uint32_t in = V - i * E;
  if (in < E) {
#pragma unroll
    for (uint32_t w = 0; w < 4; ++w) {
      if constexpr (DT == ESPO_BF16) {
        if (2 * w >= in) r[w] = 0xFF80FF80u;
        else if (2 * w + 1 >= in) r[w] = (r[w] & 0xFFFFu) | 0xFF800000u;
      } else {
        if (w >= in) r[w] = 0xFF800000u;
      }
    }
  }
  return r;
}

// Stores vector `i`, and of a row's last one only what lies below V.
template <int DT>
__device__ __forceinline__ void vec_store(char* row, uint32_t i, uint32_t V, u32x4 r) {
  constexpr uint32_t E = vec_elems<DT>();
  if (i * E + E <= V) {
    __builtin_nontemporal_store(r, (u32x4*)(row + (size_t)i * 16));
    return;
  }
#pragma unroll
  for (uint32_t j = 0; j < E; ++j) {
    if (i * E + j >= V) break;
    if constexpr (DT == ESPO_BF16)
      ((uint16_t*)row)[i * E + j] = (uint16_t)(r[j >> 1] >> (16 * (j & 1)));
    else
      ((uint32_t*)row)[i * E + j] = r[j];
  }
}

// A row of V logits as tiles of 64 vectors, one per lane of a wave.
struct RowView {
  const char* x;
  uint32_t V, nvec, ntiles;
};
template <int DT>
__device__ __forceinline__ RowView row_view(const char* x, uint32_t V) {
  const uint32_t nvec = (V + vec_elems<DT>() - 1) / vec_elems<DT>();
  return RowView{x, V, nvec, (nvec + kWave - 1) / kWave};
}

constexpr int kAhead = 4;  // vectors of a lane in flight

// Calls use(t, raw) for tiles t, t + step, t + 2 step, t + 3 step at a time, starting at `first` and below `end`, while the next four
// are loaded.  A vector's index is clamped to the row's last one, so that every load is in bounds and none waits for a branch;
// tile_logits masks what lies beyond V, and `use` leaves out tiles at or beyond `end`.
template <typename Use>
__device__ __forceinline__ void stream_tiles(const RowView& r, uint32_t first, uint32_t end, uint32_t step, Use&& use) {
  const uint32_t lane = threadIdx.x & (kWave - 1);
  const auto load = [&](uint32_t t) {
    return __builtin_nontemporal_load((const u32x4*)(r.x + (size_t)min(t * kWave + lane, r.nvec - 1) * 16));
  };
  if (first >= end) return;
  u32x4 a[kAhead], b[kAhead];
  const auto load_all = [&](u32x4* v, uint32_t t) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) v[j] = load(min(t + j * step, end - 1));
  };
  load_all(a, first);
  for (uint32_t t = first;;) {
    load_all(b, t + kAhead * step);
    use(t, a);
    if ((t += kAhead * step) >= end) return;
    load_all(a, t + kAhead * step);
    use(t, b);
    if ((t += kAhead * step) >= end) return;
  }
}

// The lane's logits of tile t; those at or beyond V are masked.
template <int DT>
__device__ __forceinline__ void tile_logits(const RowView& r, uint32_t t, u32x4 raw, float y[vec_elems<DT>()]) {
  constexpr uint32_t E = vec_elems<DT>();
  vec_unpack<DT>(raw, y);
  if (t + 1 >= r.ntiles) {  // the row's last tile
    const uint32_t i = t * kWave + (threadIdx.x & (kWave - 1));
#pragma unroll
    for (uint32_t j = 0; j < E; ++j)
      if (i * E + j >= r.V) y[j] = kNegInf;
  }
}

template <int DT>
__device__ __forceinline__ float logit_at(const char* row, uint32_t v) {
  if constexpr (DT == ESPO_BF16)
    return __builtin_bit_cast(float, (uint32_t)((const uint16_t*)row)[v] << 16);
  else
    return ((const float*)row)[v];
}

// Softmax sums of the logits seen so far: s = sum 2^t, a = sum t 2^t with t = x k2 + nb, k2 = log2(e) / temperature and nb = -m k2
// rounded, m the largest logit.  One fused operation forms t with one rounding; that nb is rounded moves every t by the same d of up to half a
// step of nb, which scales both sums by one factor, and row_sums takes it out.  m starts at kMaskedRow, and sums over nothing but masked
// logits are dropped.
// Where |nb| is large, so is d.  From kFarRow on (below it d is at most 8) a row's sums are formed again from the differences x - m.  From kFarLane on
// 2^d may be no number (below it d is at most 64), but two logits that differ are 128 powers of 2 and more apart, so that what a lane has summed up relative to
// one that is not the row's largest counts as nothing.
constexpr float kFarRow = 0x1p28f, kFarLane = 0x1p31f;
struct SoftmaxSums {
  float m, nb, s, a;
};
constexpr SoftmaxSums kNoSums = SoftmaxSums{kMaskedRow, 0.0f, 0.0f, 0.0f};

template <bool kEntropy>
__device__ __forceinline__ void rescale(SoftmaxSums& p, float m, float k2) {
#pragma clang fp contract(off)  // the difference of two references is that of their rounded values
  const bool any = p.m > kMaskedRow && fabsf(p.nb) < kFarLane;
  const float nb = -m * k2, d = fmaxf(nb - p.nb, kLeastExponent), f = any ? __builtin_amdgcn_exp2f(d) : 0.0f, s = any ? p.s : 0.0f;
  if constexpr (kEntropy) p.a = f * ((any ? p.a : 0.0f) + d * s);
  p.s = s * f;
  p.m = m;
  p.nb = nb;
}

// The same where one of the lanes needs it: after a row's first vectors hardly any does.
template <bool kEntropy>
__device__ __forceinline__ void follow(SoftmaxSums& p, float m, float k2) {
  if (__builtin_amdgcn_ballot_w64(m > p.m) != 0) rescale<kEntropy>(p, m, k2);
}

template <bool kEntropy>
__device__ __forceinline__ void add_logit(SoftmaxSums& p, float x, float k2) {
  float t = __builtin_fmaf(x, k2, p.nb);
  if constexpr (kEntropy) t = fmaxf(t, kLeastExponent);
  const float e = __builtin_amdgcn_exp2f(t);
  p.s += e;
  if constexpr (kEntropy) p.a = __builtin_fmaf(e, t, p.a);
}

// Merged over a wave, wave-uniform, in a fixed order.
template <bool kEntropy>
__device__ __forceinline__ SoftmaxSums wave_merge(SoftmaxSums p, float k2) {
  rescale<kEntropy>(p, wave_max(p.m), k2);
  p.s = wave_sum(p.s);
  if constexpr (kEntropy) p.a = wave_sum(p.a);
  return p;
}

// Merged over a workgroup of W waves, the same in every thread; lds holds W entries, and a barrier has passed since its last use.
template <int W, bool kEntropy>
__device__ __forceinline__ SoftmaxSums block_merge(SoftmaxSums p, float k2, SoftmaxSums* lds) {
  p = wave_merge<kEntropy>(p, k2);
  const int lane = threadIdx.x & (kWave - 1);
  if (lane == 0) lds[threadIdx.x >> 6] = p;
  __syncthreads();
  return wave_merge<kEntropy>(lane < W ? lds[lane] : kNoSums, k2);
}

// By how much t falls short of (x - m) k2.
__device__ __forceinline__ float exponent_short(float m, float nb, float k2) { return __builtin_fmaf(-m, k2, -nb); }

// The sums relative to m itself, of a row with |nb| below kFarRow.  The largest logit's own term is 1, and 0 in a, by definition: it is taken out
// as it was added and put back as that, so that a row of one logit has the sums 1 and 0.
__device__ __forceinline__ SoftmaxSums exact_sums(const SoftmaxSums& p, float k2) {
  const float d = exponent_short(p.m, p.nb, k2), f = __builtin_amdgcn_exp2f(d), t = __builtin_fmaf(p.m, k2, p.nb), e = __builtin_amdgcn_exp2f(t);
  const float s = p.s - e, a = p.a - e * t;
  return SoftmaxSums{p.m, p.nb, __builtin_fmaf(s, f, 1.0f), f * __builtin_fmaf(d, s, a)};
}

// The same of a row with |nb| of kFarRow and more, from the row itself, by a workgroup of W waves.
template <int DT, int W>
__device__ __forceinline__ SoftmaxSums far_sums(const RowView& r, float m, float k2, SoftmaxSums* lds) {
  float s = 0.0f, a = 0.0f;
#pragma unroll 1
  for (uint32_t i = threadIdx.x; i < r.nvec; i += W * kWave) {
    const u32x4 raw = vec_load<DT>(r.x, i, r.V);
#pragma unroll 1
    for (uint32_t j = 0; j < vec_elems<DT>(); ++j) {
      const float x = logit_in<DT>(raw, j), t = fmaxf((x - m) * k2, kLeastExponent), e = x > kMaskedRow ? __builtin_amdgcn_exp2f(t) : 0.0f;
      s += e;
      a = __builtin_fmaf(e, t, a);
    }
  }
  s = wave_sum(s), a = wave_sum(a);
  if constexpr (W > 1) {
    const int lane = threadIdx.x & (kWave - 1);
    __syncthreads();                          // block_merge's sums have been read
    if (lane == 0) lds[threadIdx.x >> 6] = SoftmaxSums{m, 0.0f, s, a};
    __syncthreads();
    s = wave_sum(lane < W ? lds[lane].s : 0.0f), a = wave_sum(lane < W ? lds[lane].a : 0.0f);
  }
  return SoftmaxSums{m, -m * k2, s, a};
}

// A row's sums relative to its largest logit, from what was merged over its workgroup of W waves (the same in all threads); lds: block_merge's.
template <int DT, int W>
__device__ __forceinline__ SoftmaxSums row_sums(const RowView& r, const SoftmaxSums& p, float k2, SoftmaxSums* lds) {
  const float m = uniform_f32(p.m, 0), nb = uniform_f32(p.nb, 0);
  if (m > kMaskedRow && !(fabsf(nb) < kFarRow)) return far_sums<DT, W>(r, m, k2, lds);
  return exact_sums(p, k2);
}

}  // namespace espo
