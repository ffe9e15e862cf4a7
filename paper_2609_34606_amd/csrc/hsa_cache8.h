// What the kernels of the attention over the 8-bit cache share: the walk of a key
// head's tokens and the output of a row.
#pragma once

#include <algorithm>

#include "hsa_fp8.h"
#include "hsa_kernels.h"

namespace hsa {

// One item (a tile of query rows of one key head): its queries and its 64-key tiles.
// The list is n_sel selected pages, then pages [cur_first, ..). Its tokens are one stream, cut every
// 64 whatever pages they are in (stream), or a page is tpp tiles, its last one shifted back to
// end at the page's end.
struct Cache8Walk {
  int len, q_len;  // tokens and queries of the sequence
  int base;        // causal: query i sees tokens below base + i + 1
  int rows;        // queries of the item that exist, times G (<= 0: none)
  int lim;         // tokens that the item's last query sees
  int n_sel, n_list, n_tiles;
};

// Tokens that query i of the sequence sees (an index below this; 0 for a query before the first
// token, so that differences with a place past the list's end fit 32 bits).
__device__ __forceinline__ int cache8_limit(const Cache8AttnParams& p, const Cache8Walk& w, int i) {
  return p.causal ? max(min(w.len, w.base + i + 1), 0) : w.len;
}

// Every lane of the wave must call it.
__device__ __forceinline__ Cache8Walk cache8_walk(const Cache8AttnParams& p, int b, int h, int row0, int rows,
                                                  int lane) {
  Cache8Walk w;
  const int cap = p.max_pages * p.P;
  const int end = (p.cur_first + p.n_cur) * p.P;
  w.len = p.kv_len ? clampi(ld_const(p.kv_len + b), 0, cap) : (p.causal ? end : cap);
  w.q_len = p.q_len ? clampi(ld_const(p.q_len + b), 0, p.n_q) : p.n_q;
  w.base = w.len - w.q_len;
  const int last = min(row0 + rows, w.q_len * p.G);  // row past the last one
  w.rows = last - row0;
  w.lim = cache8_limit(p, w, __builtin_amdgcn_readfirstlane((last - 1) / p.G));
  w.n_sel = __builtin_amdgcn_readfirstlane(
      min(count_selected(p.sel + ((size_t)b * p.Hk + h) * p.k_max, p.k_max, p.max_pages, lane), (int)p.k_h[h]));
  const int cur = clampi(w.lim - p.cur_first * p.P, 0, p.n_cur * p.P);  // tokens of the run of pages
  // (quotients come from the vector unit: what follows from them is brought back)
  const int full = __builtin_amdgcn_readfirstlane(cur / p.P), rest = cur - full * p.P;
  w.n_list = w.n_sel + full + (rest > 0 ? 1 : 0);
  if (p.stream) w.n_tiles = (int)(((int64_t)w.n_sel * p.P + cur + 63) >> 6);
  else w.n_tiles = w.n_sel * p.tpp + full * p.tpp + (rest + 63) / 64;
  return w;
}

// Granule gr (8 tokens) of a tile of the stream that begins in the page at list position li, at
// the page's granule at: its list position and first token within the page. ok: it is a token of a
// listed page (else it repeats one).
struct Cache8Granule {
  int li, off;
  bool ok;
};
__device__ __forceinline__ Cache8Granule cache8_granule(const Cache8AttnParams& p, const Cache8Walk& w, int li, int at,
                                                        int gr) {
  const int x = at + gr;                // below gpp + 8
  const int pg = (x * p.gmul) >> 16;    // x / gpp: exact while (gpp + 8) gpp is below 2^16
  Cache8Granule a;
  a.off = 8 * (x - pg * p.gpp);
  a.ok = li + pg < w.n_list;
  a.li = min(li + pg, w.n_list - 1);
  return a;
}
// Logical page of list position li and the slot of a page, per lane.
__device__ __forceinline__ int page_v(const Cache8AttnParams& p, const Cache8Walk& w, const int32_t* selrow, int li) {
  return li < w.n_sel ? selrow[li] : p.cur_first + li - w.n_sel;
}
__device__ __forceinline__ int slot_v(const Cache8AttnParams& p, const int32_t* ptrow, int page) {
  return clampi(ptrow[page], 0, p.num_slots - 1);
}

// N dims of a finished row from its sums: o / l, and the log-sum-exp once a row. A
// row that sees no key is 0 with a log-sum-exp of -inf.
template <typename T, int N>
__device__ __forceinline__ void cache8_store(const Cache8AttnParams& p, int b, int i, int head, int d0,
                                             const float (&o)[N], float m, float l, bool lse) {
  const float inv = l > 0.f ? 1.f / l : (l == l ? 0.f : l);
  T* dst = static_cast<T*>(p.o) + (((size_t)b * p.n_q + i) * p.H + head) * p.d + d0;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < N; ++e) dst[e] = o[e] * inv;
  } else if constexpr (N == 1) {
    *dst = (uint16_t)pack_bf16(o[0] * inv, 0.f);
  } else {
    uint32_t* w = reinterpret_cast<uint32_t*>(dst);
#pragma unroll
    for (int e = 0; e < N / 2; ++e) w[e] = pack_bf16(o[2 * e] * inv, o[2 * e + 1] * inv);
  }
  if (lse && p.lse)
    p.lse[((size_t)b * p.H + head) * p.n_q + i] = l > 0.f ? m * p.sm_scale + logf(l) : (l == l ? -INFINITY : l);
}

}  // namespace hsa
