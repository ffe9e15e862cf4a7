// Rotary positions: the rotation's table as kernels take it, and the cosine
// and sine of a position's angle.
#pragma once

#include "hsa_device.h"
#include "hsa_kernels.h"

namespace hsa {

// Cosine and sine of t turns (2 pi t). The turns are an fp64 product of
// position and frequency, so that far positions keep their angle: the nearest
// quarter is taken off in fp64, exactly, and what is left, at most an eighth of a
// turn, is small enough for the Taylor series in fp32 (the first terms left
// out are below 2e-9).
__device__ __forceinline__ void cos_sin_turns(double t, float& c, float& s) {
  const double t4 = 4.0 * t, q = rint(t4);
  const float x = (float)(t4 - q) * 1.57079632679489662f;
  const float x2 = x * x;
  float ps = fmaf(x2, 2.75573192e-6f, -1.98412698e-4f);
  ps = fmaf(x2, ps, 8.33333333e-3f);
  ps = fmaf(x2, ps, -1.66666667e-1f);
  const float sn = fmaf(x * x2, ps, x);
  float pc = fmaf(x2, -2.75573192e-7f, 2.48015873e-5f);
  pc = fmaf(x2, pc, -1.38888889e-3f);
  pc = fmaf(x2, pc, 4.16666667e-2f);
  pc = fmaf(x2, pc, -0.5f);
  const float cs = fmaf(x2, pc, 1.f);
  const int n = (int)((long long)q & 3);  // quarters: (c, s) turned by n * 90 degrees
  const float a = n & 1 ? sn : cs, b = n & 1 ? cs : sn;
  c = n == 1 || n == 2 ? -a : a;
  s = n >= 2 ? -b : b;
}

// Cosine and sine, times the amplitude, of pair i of a token at positions pos[0..axes).
__device__ __forceinline__ void rope_cos_sin(const RopeTable& r, const int32_t (&pos)[3], int i, float& c, float& s) {
  const int a = r.axis[i];
  const int32_t x = a == 0 ? pos[0] : (a == 1 ? pos[1] : pos[2]);
  cos_sin_turns((double)x * r.turns[i], c, s);
  c *= r.amplitude;
  s *= r.amplitude;
}

// The positions of token i of batch entry b.
__device__ __forceinline__ void rope_positions(const RopeTable& r, int b, int i, int n, int32_t (&pos)[3]) {
  if (r.pos) {
    const int32_t* p = r.pos + ((size_t)b * n + i) * r.axes;
    pos[0] = p[0];
    pos[1] = r.axes > 1 ? p[1] : 0;
    pos[2] = r.axes > 2 ? p[2] : 0;
  } else {
    pos[0] = (r.first ? r.first[b] : 0) + i;
    pos[1] = pos[2] = 0;
  }
}

// E elements of T (uint16_t: bf16) at an element's alignment, as fp32 and back.
template <typename T>
struct Pack;
template <>
struct Pack<uint16_t> {
  static constexpr int E = 8;
  typedef uint32_t V __attribute__((ext_vector_type(4), aligned(2)));
  static __device__ __forceinline__ void load(const uint16_t* p, float (&x)[8]) {
    const V v = *reinterpret_cast<const V*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = bf16_lo(v[i]);
      x[2 * i + 1] = bf16_hi(v[i]);
    }
  }
  static __device__ __forceinline__ void store(uint16_t* p, const float (&x)[8]) {
    V v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
    *reinterpret_cast<V*>(p) = v;
  }
  static __device__ __forceinline__ float load1(const uint16_t* p) { return bf16_to_f32(*p); }
  static __device__ __forceinline__ void store1(uint16_t* p, float x) { *p = (uint16_t)pack_bf16(x, 0.f); }
};
template <>
struct Pack<float> {
  static constexpr int E = 4;
  static __device__ __forceinline__ void load(const float* p, float (&x)[4]) {
    const f32x4 v = ld4u(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = v[i];
  }
  static __device__ __forceinline__ void store(float* p, const float (&x)[4]) {
    st4u(p, f32x4{x[0], x[1], x[2], x[3]});
  }
  static __device__ __forceinline__ float load1(const float* p) { return *p; }
  static __device__ __forceinline__ void store1(float* p, float x) { *p = x; }
};

// A token's head is cut into items of up to E pairs or E copied dims. Half
// layout: ceil(rot/2 / E) items of pairs (i, i + rot/2), then items of the dims
// from rot on. Interleaved: D / E runs of E dims, whose pairs below rot turn.
// E divides D; the last item of either kind may be short (E pairs at rot/2, or
// E dims at D).
template <typename T>
__host__ __device__ __forceinline__ int rope_items(int layout, int rot, int d) {
  constexpr int E = Pack<T>::E;
  if (layout == HSA_ROPE_INTERLEAVED) return d / E;
  return (rot / 2 + E - 1) / E + (d - rot + E - 1) / E;
}

// What item j covers: n elements from dim a on, and for pairs in halves the same
// number from dim a + rot/2 on.
struct RopeItem {
  int a, n;
  bool pairs;
};
template <typename T>
__device__ __forceinline__ RopeItem rope_item(int layout, int rot, int d, int j) {
  constexpr int E = Pack<T>::E;
  if (layout == HSA_ROPE_INTERLEAVED) return RopeItem{j * E, E, false};
  const int np = (rot / 2 + E - 1) / E;
  if (j < np) return RopeItem{j * E, min(E, rot / 2 - j * E), true};
  return RopeItem{rot + (j - np) * E, min(E, d - rot - (j - np) * E), false};
}

// n <= E elements at p, the rest 0
template <typename T>
__device__ __forceinline__ void load_some(const T* p, int n, float (&x)[Pack<T>::E]) {
  if (n == Pack<T>::E) {
    Pack<T>::load(p, x);
  } else {
#pragma unroll
    for (int i = 0; i < Pack<T>::E; ++i) x[i] = i < n ? Pack<T>::load1(p + i) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store_some(T* p, int n, const float (&x)[Pack<T>::E]) {
  if (n == Pack<T>::E) {
    Pack<T>::store(p, x);
  } else {
#pragma unroll
    for (int i = 0; i < Pack<T>::E; ++i)
      if (i < n) Pack<T>::store1(p + i, x[i]);
  }
}

// Cosines and sines of an item's pairs at one token: E pairs for halves, E / 2 interleaved
// ones. Pairs outside the rotated part get (1, 0).
template <typename T>
__device__ __forceinline__ void rope_item_angles(const RopeTable& r, const RopeItem& it, const int32_t (&pos)[3],
                                                 float (&c)[Pack<T>::E], float (&s)[Pack<T>::E]) {
  constexpr int E = Pack<T>::E;
  const bool inter = r.layout == HSA_ROPE_INTERLEAVED;
  const int first = inter ? it.a / 2 : it.a, n = inter ? E / 2 : (it.pairs ? it.n : 0);
#pragma unroll
  for (int i = 0; i < E; ++i) {
    c[i] = 1.f;
    s[i] = 0.f;
    if (i < n && first + i < r.rot / 2) rope_cos_sin(r, pos, first + i, c[i], s[i]);
  }
}

// Turns x (and y, the other half's elements) of an item.
template <typename T>
__device__ __forceinline__ void rope_turn(const RopeTable& r, const RopeItem& it, const float (&c)[Pack<T>::E],
                                          const float (&s)[Pack<T>::E], float (&x)[Pack<T>::E],
                                          float (&y)[Pack<T>::E]) {
  constexpr int E = Pack<T>::E;
  if (r.layout == HSA_ROPE_INTERLEAVED) {
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
      if (it.a / 2 + i >= r.rot / 2) continue;  // copied: also infinities, which 0 * x would spoil
      const float a = x[2 * i], b = x[2 * i + 1];
      x[2 * i] = a * c[i] - b * s[i];
      x[2 * i + 1] = b * c[i] + a * s[i];
    }
  } else if (it.pairs) {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float a = x[i], b = y[i];
      x[i] = a * c[i] - b * s[i];
      y[i] = b * c[i] + a * s[i];
    }
  }
}

}  // namespace hsa
