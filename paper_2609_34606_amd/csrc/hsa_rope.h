// Rotary positions: the rotation's table as kernels take it, and the cosine
// and sine of a position's angle.
#pragma once

#include "hsa_device.h"
#include "hsa_kernels.h"

namespace hsa {

// Cosine and sine of t4 quarter turns (pi / 2 each). The turns are an fp64 product of
// position and frequency, so that far positions keep their angle: the nearest
// whole number is taken off in fp64, exactly, and what is left, at most half a quarter, is
// small enough for the Taylor series in fp32 (the first terms left out are below 2e-9).
__device__ __forceinline__ void cos_sin_quarters(double t4, float& c, float& s) {
  // adding 1.5 * 2^52 rounds to a whole number, whose low bits are then the sum's
  constexpr double kRound = 6755399441055744.0;
  const double u = t4 + kRound;
  const uint32_t n = (uint32_t)__double2loint(u);
  const float x = (float)(t4 - (u - kRound)) * 1.57079632679489662f;
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
  // (c, s) turned by n quarters
  c = __uint_as_float(__float_as_uint(n & 1 ? sn : cs) ^ ((n + 1) & 2) << 30);
  s = __uint_as_float(__float_as_uint(n & 1 ? cs : sn) ^ (n & 2) << 30);
}

// The positions of token i of batch entry b, on up to three axes.
struct RopePos {
  int x0, x1, x2;
};
__device__ __forceinline__ RopePos rope_positions(const RopeTable& r, int b, int i, int n) {
  if (!r.pos) return RopePos{(r.first ? r.first[b] : 0) + i, 0, 0};
  const int32_t* p = r.pos + ((size_t)b * n + i) * r.axes;
  return RopePos{p[0], r.axes > 1 ? p[1] : 0, r.axes > 2 ? p[2] : 0};
}

// 16 bytes of T (uint16_t: bf16) at an element's alignment, one access.
template <typename T>
struct Vec16;
template <>
struct Vec16<uint16_t> {
  typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2)));
};
template <>
struct Vec16<float> {
  typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4)));
};

// N elements of T (16 bytes, or one) and their fp32 values.
template <typename T, int N>
struct Elems {
  using Raw = typename Vec16<T>::type;
  static __device__ __forceinline__ Raw load(const T* p) { return *reinterpret_cast<const Raw*>(p); }
  static __device__ __forceinline__ void unpack(const Raw& v, float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2) {
        x[2 * i] = bf16_lo(v[i]);
        x[2 * i + 1] = bf16_hi(v[i]);
      } else {
        x[i] = __uint_as_float(v[i]);
      }
    }
  }
  static __device__ __forceinline__ void store(T* p, const float (&x)[N]) {
    Raw v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2) v[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
      else v[i] = __float_as_uint(x[i]);
    }
    *reinterpret_cast<Raw*>(p) = v;
  }
};
template <typename T>
struct Elems<T, 1> {
  using Raw = T;
  static __device__ __forceinline__ Raw load(const T* p) { return *p; }
  static __device__ __forceinline__ void unpack(const Raw& v, float (&x)[1]) {
    if constexpr (sizeof(T) == 2) x[0] = bf16_to_f32(v);
    else x[0] = v;
  }
  static __device__ __forceinline__ void store(T* p, const float (&x)[1]) {
    if constexpr (sizeof(T) == 2) *p = (uint16_t)pack_bf16(x[0], 0.f);
    else *p = x[0];
  }
};

// How a token's head is cut into items, by what the rotated part allows:
//   halves       16 bytes of first elements and the 16 of their partners, rot / 2 dims on
//                (rot / 2 a multiple of the elements in 16 bytes); "part" where dims
//                are left to copy, which takes up to twice the items;
//   interleaved  16 bytes of whole pairs (rot a multiple);
//   single       one pair, of either layout (any rot).
// Items of the copied dims follow, 16 bytes or one element each.
enum RopeMode { kRopeHalves = 0, kRopeInterleaved = 1, kRopeSingle = 2, kRopePart = 3 };

template <typename T>
inline int rope_mode(const RopeTable& r, int d) {
  constexpr int E = 16 / sizeof(T);
  if (r.layout == HSA_ROPE_HALF) return r.rot / 2 % E ? kRopeSingle : (r.rot == d ? kRopeHalves : kRopePart);
  return r.rot % E == 0 ? kRopeInterleaved : kRopeSingle;
}

template <typename T, int kMode>
struct RopeItem {
  static constexpr int N = kMode == kRopeSingle ? 1 : 16 / (int)sizeof(T);  // elements a load
  static constexpr int NP = kMode == kRopeInterleaved ? N / 2 : N;          // pairs an item
  using El = Elems<T, N>;
  int a, b;      // first dims of its two runs
  bool turn;     // its pairs turn (else its first run is copied)
  double f[NP];  // quarter turns per position of its pairs, and their axes
  int axis[NP];

  static __host__ __device__ __forceinline__ int count(int rot, int d) {
    return kMode == kRopeInterleaved ? d / N : (rot / 2 + d - rot) / N;
  }
  __device__ __forceinline__ void set(const RopeTable& r, int j) {
    if constexpr (kMode == kRopeInterleaved) {
      a = j * N;
      b = a;
      turn = a < r.rot;
    } else {
      const int np = r.rot / 2 / N;
      turn = j < np;
      const bool apart = kMode == kRopeSingle && r.layout == HSA_ROPE_INTERLEAVED;
      a = turn ? (apart ? 2 * j : j * N) : r.rot + (j - np) * N;
      b = turn ? (apart ? a + 1 : a + r.rot / 2) : a;
    }
  }
  __device__ __forceinline__ void frequencies(const RopeTable& r) {
    const bool halves = kMode != kRopeInterleaved && r.layout == HSA_ROPE_HALF;
    const int i0 = turn ? (halves ? a : a / 2) : 0;
#pragma unroll
    for (int i = 0; i < NP; ++i) f[i] = r.quarters[i0 + i];
#pragma unroll
    for (int i = 0; i < NP; ++i) axis[i] = r.axes > 1 ? r.axis[i0 + i] : 0;
  }
  __device__ __forceinline__ void load(const T* head, typename El::Raw& ra, typename El::Raw& rb) const {
    ra = El::load(head + a);
    if constexpr (kMode != kRopeInterleaved) rb = El::load(head + b);
  }
  // cosines and sines, times the amplitude, at a token's positions
  __device__ __forceinline__ void angles(const RopeTable& r, RopePos pos, float (&c)[NP], float (&s)[NP]) const {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int x0 = pos.x0, x1 = pos.x1, x2 = pos.x2;
      int x = axis[i] == 1 ? x1 : x0;
      x = axis[i] == 2 ? x2 : x;
      cos_sin_quarters((double)x * f[i], c[i], s[i]);
      c[i] *= r.amplitude;
      s[i] *= r.amplitude;
    }
  }
  // The loaded elements, turned: x its first run, y the second (halves and single).
  // Copied ones are left alone (also infinities, which a product by 0 would spoil).
  __device__ __forceinline__ void result(const typename El::Raw& ra, const typename El::Raw& rb, const float (&c)[NP],
                                         const float (&s)[NP], float (&x)[N], float (&y)[N]) const {
    El::unpack(ra, x);
    if constexpr (kMode != kRopeInterleaved) El::unpack(rb, y);
    if (!turn) return;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if constexpr (kMode == kRopeInterleaved) {
        const float u = x[2 * i], v = x[2 * i + 1];
        x[2 * i] = u * c[i] - v * s[i];
        x[2 * i + 1] = v * c[i] + u * s[i];
      } else {
        const float u = x[i], v = y[i];
        x[i] = u * c[i] - v * s[i];
        y[i] = v * c[i] + u * s[i];
      }
    }
  }
  __device__ __forceinline__ void store(T* head, const float (&x)[N], const float (&y)[N]) const {
    El::store(head + a, x);
    if constexpr (kMode != kRopeInterleaved)
      if (turn) El::store(head + b, y);
  }
};

}  // namespace hsa
