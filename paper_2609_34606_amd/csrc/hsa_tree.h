// What the attention kernels of drafted trees share, over either cache: the bits of the tokens that a node
// sees, and values that are no finite numbers among the nodes'.
#pragma once

#include "hsa_device.h"
#include "hsa_kernels.h"

namespace hsa {

constexpr int kMaskWords = HSA_MAX_TREE / 32;

// All ones where bit x of `on` is set (no condition codes: a tile's hundreds of them would fill the scalar
// registers).
__device__ __forceinline__ uint32_t ones_if(uint32_t on, int x) {
  return (uint32_t)((int32_t)(on << (31 - x)) >> 31);
}
// v, or other where bit x of `on` is not set.
__device__ __forceinline__ uint32_t pick(uint32_t on, int x, uint32_t v, uint32_t other) {
  const uint32_t m = ones_if(on, x);
  return (v & m) | (other & ~m);
}
// A score that bit x of `on` does not let through.
__device__ __forceinline__ float hidden(uint32_t on, int x, float s) {
  return __uint_as_float(pick(on, x, __float_as_uint(s), 0xff800000u));
}
// Two bf16 numbers of each word, eight in all, where bits of `on` are set.
__device__ __forceinline__ u32x4 keep8(u32x4 v, uint32_t on) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] &= (ones_if(on, 2 * i) & 0xffffu) | (ones_if(on, 2 * i + 1) & 0xffff0000u);
  return v;
}
// The low n bits.
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }

// One bit of a word's 8-, 16- or 32-bit lanes, spread over the lane.
__device__ __forceinline__ uint32_t fill8(uint32_t bit7) { return (bit7 >> 7) * 255u; }
__device__ __forceinline__ uint32_t fill16(uint32_t bit15) { return (bit15 >> 15) * 0xffffu; }
// Bits 0 to 3 as the top bits of four bytes; bits 0 and 1 as those of two halves.
__device__ __forceinline__ uint32_t bytes4(uint32_t on) { return (on & 15u) * 0x10204080u & 0x80808080u; }
__device__ __forceinline__ uint32_t halves2(uint32_t on) { return (on << 15 & 0x8000u) | (on << 30 & 0x80000000u); }

// Bit j: whether node i, whose mask row is `row`, sees token t0 + j.
template <typename Params, typename Walk>
__device__ __forceinline__ uint32_t tree_sees(const Params& p, const Walk& w, const uint32_t* row, int i, int t0) {
  if (t0 >= w.len) return 0u;
  const int rel = t0 - w.base;  // (t0 below len: no overflow)
  if (rel <= -8) return 0xffu;
  uint32_t on;
  if (p.mask) {
    const int x = rel >> 5, sh = rel & 31;
    const uint32_t lo = x < 0 ? ~0u : x < p.words ? row[x] : 0u;
    const uint32_t hi = x + 1 < 0 ? ~0u : x + 1 < p.words ? row[x + 1] : 0u;
    on = (uint32_t)(((uint64_t)hi << 32 | lo) >> sh);
  } else {
    on = low_bits(i + 1 - rel);
  }
  return on & low_bits(min(w.len - t0, 8));
}

// Calls add(t0, j, value) for the nodes among the tokens t0 + j of list granules [lo, hi) (t0: a granule's first);
// value(dim) is what the node holds there, 0 for finite numbers (held: a number of the cache). Slow, and rarely called.
template <typename Params, typename Walk, typename Value, typename Add>
__device__ __forceinline__ void tree_wild(const Params& p, const Walk& w, int b, int h, int D, int lo, int hi,
                                          Value&& held, Add&& add) {
  for (int gr = lo; gr < hi; ++gr) {
    const int li = gr / p.gpp;
    if (li >= w.n_list) break;
    const int page = li < w.n_sel ? p.sel[((size_t)b * p.Hk + h) * p.k_max + li] : p.cur_first + li - w.n_sel;
    const int off = 8 * (gr - li * p.gpp), t0 = page * p.P + off;
    if (t0 + 8 <= w.base || t0 >= w.len) continue;
    const size_t slot = clampi(p.page_table[(size_t)b * p.max_pages + page], 0, p.num_slots - 1);
    const size_t head = slot * p.Hk + h;
    for (int j = max(w.base - t0, 0); j < min(w.len - t0, 8); ++j)
      add(t0, j, [&](int dim) {
        const float v = held(head, (head * D + dim) * p.P + off + j, off);
        return fabsf(v) < INFINITY ? 0.f : v;
      });
  }
}

}  // namespace hsa
