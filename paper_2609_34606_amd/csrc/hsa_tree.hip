// Attention of drafted trees over the paged caches, and the ancestor bits of their nodes.
//
// A step brings up to HSA_MAX_TREE nodes per sequence, appended behind it as its last tokens. With
// base = length - nodes, node i sees every token before base, and token base + j if bit j of its mask
// row is set (without a mask: j <= i):
//
//   o_i = sum_j softmax_j(scale q_i . k_j) v_j over the tokens it sees.
//
// The H / Hk query heads that share a key head are rows of one product (row r of key head h is head
// h G + r % G of node r / G), so that every key and value is read once for up to 64 rows.
#include <limits.h>

#include <algorithm>
#include <type_traits>

#include "hsa_fp8.h"
#include "hsa_kernels.h"

namespace hsa {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kMaskWords = HSA_MAX_TREE / 32;

// ---------------------------------------------------------------- ancestors
// A node's row is its own bit and its parent's row. Rows double the path they hold with every
// round (row |= row of the node at the end of the path), so a chain of n nodes takes log2(n) rounds, through
// shared memory, a thread a node. Bound: a launch's latency.
__global__ __launch_bounds__(HSA_MAX_TREE) void tree_mask_kernel(TreeMaskParams p) {
  __shared__ uint32_t rows[HSA_MAX_TREE][kMaskWords + 1];
  __shared__ int jump[HSA_MAX_TREE];
  const int i = threadIdx.x, b = blockIdx.x;
  const int n = p.count ? clampi(p.count[b], 0, p.n) : p.n;
  const bool node = i < n;
  int at = -1;
  if (node) {
    const int x = p.parent[(size_t)b * p.n + i];
    at = x >= 0 && x < i ? x : -1;
  }
  uint32_t row[kMaskWords];
#pragma unroll
  for (int w = 0; w < kMaskWords; ++w) row[w] = i >> 5 == w ? 1u << (i & 31) : 0u;
  for (int done = 1; done < n; done *= 2) {
#pragma unroll
    for (int w = 0; w < kMaskWords; ++w) rows[i][w] = row[w];
    jump[i] = at;
    __syncthreads();
    if (at >= 0) {
#pragma unroll
      for (int w = 0; w < kMaskWords; ++w) row[w] |= rows[at][w];
      at = jump[at];
    }
    __syncthreads();
  }
  if (!node) return;
  int depth = -1;
#pragma unroll
  for (int w = 0; w < kMaskWords; ++w) {
    if (w < p.words) p.mask[((size_t)b * p.n + i) * p.words + w] = row[w];
    depth += __popc(row[w]);
  }
  if (p.pos) p.pos[(size_t)b * p.n + i] = (p.first ? p.first[b] : 0) + depth;
}

// ---------------------------------------------------------------- attention
// What a cache holds, and the type of queries and outputs: e4m3 codes (bf16 or fp32 queries), or numbers
// in the type of the call.
enum Held { kCodes, kCodesF32, kBf16, kF32 };

// The same of fp32 numbers, A[16x4] * B[4x16], k = l/16.
__device__ __forceinline__ f32x4 mfma4(float a, float b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// Two bf16 numbers of a word where bits 0 and 1 of `on` are set.
__device__ __forceinline__ uint32_t keep2(uint32_t w, uint32_t on) {
  return w & (((on & 1u) ? 0xffffu : 0u) | ((on & 2u) ? 0xffff0000u : 0u));
}
__device__ __forceinline__ u32x4 keep8(u32x4 v, uint32_t on) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = keep2(v[i], on >> (2 * i));
  return v;
}
__device__ __forceinline__ bool wild2(uint32_t w) {
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}
// The low n bits.
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }

// A sequence's tokens as an item's key head lists them: n_sel selected pages, then pages
// [cur_first, ..), one stream cut into tiles whatever pages they are in.
struct TreeWalk {
  int len, q_len, base;
  int n_sel, n_list, n_tiles;
};

// Every lane of the wave must call it.
template <int kTile>
__device__ __forceinline__ TreeWalk tree_walk(const TreeAttnParams& p, int b, int h, int lane) {
  TreeWalk w;
  const int end = (p.cur_first + p.n_cur) * p.P;
  w.len = p.kv_len ? clampi(ld_const(p.kv_len + b), 0, p.max_pages * p.P) : end;
  w.q_len = p.q_len ? clampi(ld_const(p.q_len + b), 0, p.n_q) : p.n_q;
  w.base = w.len - w.q_len;
  w.n_sel = __builtin_amdgcn_readfirstlane(
      min(count_selected(p.sel + ((size_t)b * p.Hk + h) * p.k_max, p.k_max, p.max_pages, lane), (int)p.k_h[h]));
  const int cur = clampi(w.len - p.cur_first * p.P, 0, p.n_cur * p.P);
  w.n_list = w.n_sel + __builtin_amdgcn_readfirstlane((cur + p.P - 1) / p.P);
  w.n_tiles = (w.n_sel * p.P + cur + kTile - 1) / kTile;
  return w;
}

template <int H>
using QType = typename std::conditional<H == kCodes || H == kBf16, uint16_t, float>::type;

// N dims of a finished row: o / l, and the log-sum-exp once a row. A row that sees no token is
// 0 with a log-sum-exp of -inf.
template <typename T, int N>
__device__ __forceinline__ void tree_store(const TreeAttnParams& p, int D, int b, int i, int head, int d0,
                                           const float (&o)[N], float m, float l, bool lse) {
  const float inv = l > 0.f ? 1.f / l : (l == l ? 0.f : l);
  T* dst = static_cast<T*>(p.o) + (((size_t)b * p.n_q + i) * p.H + head) * D + d0;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < N; ++e) dst[e] = o[e] * inv;
  } else {
    static_assert(N % 2 == 0, "pairs");
    uint32_t* w = reinterpret_cast<uint32_t*>(dst);
#pragma unroll
    for (int e = 0; e < N / 2; ++e) w[e] = pack_bf16(o[2 * e] * inv, o[2 * e + 1] * inv);
  }
  if (lse && p.lse)
    p.lse[((size_t)b * p.H + head) * p.n_q + i] = l > 0.f ? m * p.sm_scale + logf(l) : (l == l ? -INFINITY : l);
}

// Up to 16 kCols rows of one key head against a range of its tiles. A wave takes every kWaves-th tile (64
// tokens, fp32 32) and keeps an online softmax of its own; the workgroup joins them at the end.
//
// Products are transposed (keys are the rows of S^T = K Q^T, dims those of O^T = V^T P^T), so a lane
// holds scores of one row r = l % 16. Keys take the places in S^T that give a lane the scores of the
// keys whose values it loads, a granule of eight tokens (which never crosses a page) for each half u
// of the tile: weights become the second product's operand without an exchange between lanes. Tiles go
// from memory to the registers of the wave that uses them; the next tile's keys are asked for once this
// one's scores are done with their registers, the values after its output.
template <int H, int D, int kCols, int kWaves>
__global__ __launch_bounds__(64 * kWaves, kWaves == 8 ? 2 : 1) void tree_attn_kernel(TreeAttnParams p) {
  using T = QType<H>;
  constexpr bool kEight = H == kCodes || H == kCodesF32, kMat32 = H == kF32;
  constexpr int kTile = kMat32 ? 32 : 64, kGran = kTile / 8;  // tokens, granules of a tile
  constexpr int NI = kTile / 16;                              // score blocks
  constexpr int M = D / 16;                                   // blocks of output dims
  constexpr int kParts = H == kCodesF32 ? 3 : 1;              // bf16 parts of a query
  // bf16 parts of a weight. One rounds it by up to 2^-8, about what the result's own rounding adds; two
  // leave 2^-16. fp32 queries take three (2^-24); fp32 caches none (their products are of fp32).
  constexpr int kWParts = H == kCodesF32 ? 3 : (kCols == 1 ? 2 : 1);
  constexpr int KC = H == kF32 ? D / 16 : (kEight ? D / 64 : D / 32);  // 16-byte pieces of a key row a lane
  constexpr int kRows = 16 * kCols, OS = D + 4;
  constexpr int kThreads = 64 * kWaves;
  __shared__ int2 pages[kTreePages];                // slot and first token of the listed pages
  __shared__ uint32_t bits[kRows][kMaskWords + 1];  // mask rows of the item's nodes
  __shared__ __attribute__((aligned(16))) float osm[kWaves * 16 * OS];
  __shared__ float msm[kWaves][kRows], lsm[kWaves][kRows];
  const int tid = threadIdx.x, lane = tid & 63, c16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Workgroup i runs on XCD i % 8: the row tiles of a piece, which read the same pages, follow each
  // other there. Later pieces, which short sequences lack, come last.
  const int per8 = 8 * p.n_rt;
  const int oct = __builtin_amdgcn_readfirstlane(blockIdx.x / per8), in = blockIdx.x - oct * per8;
  const int rt = in >> 3, group = oct * 8 + (in & 7), heads = p.B * p.Hk;
  const int split = __builtin_amdgcn_readfirstlane(group / heads), bh = group - split * heads;
  if (split >= p.n_split) return;
  const int b = __builtin_amdgcn_readfirstlane(bh / p.Hk), h = bh - b * p.Hk;
  const TreeWalk w = tree_walk<kTile>(p, b, h, lane);
  const int row0 = rt * kRows;
  if (row0 >= w.q_len * p.G) return;
  const int t_lo = split * p.split_tiles, t_hi = min(t_lo + p.split_tiles, w.n_tiles);
  if (split > 0 && t_lo >= w.n_tiles) return;
  const bool whole = w.n_tiles <= p.split_tiles;

  const int i0 = __builtin_amdgcn_readfirstlane(row0 / p.G);
  if (p.mask) {
    const int nodes = min((row0 + kRows - 1) / p.G, w.q_len - 1) - i0 + 1;
    const uint32_t* src = p.mask + ((size_t)b * p.n_q + i0) * p.words;
    for (int x = tid; x < nodes * p.words; x += kThreads) bits[x / p.words][x % p.words] = src[x];
  }

  // queries
  u32x4 qf[kCols][kMat32 ? 1 : D / 32][kParts];
  f32x4 qs[kCols][kMat32 ? D / 16 : 1];
  int node[kCols];  // of the column's row
#pragma unroll
  for (int n = 0; n < kCols; ++n) {
    const int r = row0 + 16 * n + c16, i = min(r / p.G, w.q_len - 1);
    node[n] = i;
    const T* q = static_cast<const T*>(p.q) + (((size_t)b * p.n_q + i) * p.H + h * p.G + r % p.G) * D;
    if constexpr (kMat32) {
#pragma unroll
      for (int c = 0; c < D / 16; ++c) qs[n][c] = *reinterpret_cast<const f32x4*>(q + 16 * c + 4 * g);
    } else {
#pragma unroll
      for (int c = 0; c < D / 32; ++c)  // (a lane's 16 codes are dims 16 g.. of 64)
        split_row<T, kParts>(q + (kEight ? 64 * (c >> 1) + 16 * g + 8 * (c & 1) : 32 * c + 8 * g), qf[n][c]);
    }
  }

  f32x4 acc[kCols][M];
  float m_run[kCols], l_run[kCols];
  const float c2 = p.scale_log2;
#pragma unroll
  for (int n = 0; n < kCols; ++n) {
#pragma unroll
    for (int m = 0; m < M; ++m) acc[n][m] = f32x4{0};
    m_run[n] = softmax_floor(c2);
    l_run[n] = 0.f;
  }

  u32x4 kc[NI][KC], vc[M][kEight ? 1 : 2];
  float ksc[2], vsc[2];
  // granules of the lane's key rows and of its values, for half u
  auto key_granule = [&](int u) { return kMat32 ? 2 * u + (c16 >> 3) : kEight ? 2 * (c16 >> 2) + u : 4 * u + (c16 >> 2); };
  auto val_granule = [&](int u) { return kMat32 ? 2 * u + (g >> 1) : kEight ? 2 * g + u : 4 * u + g; };
  // the next tile's places: slots, tokens within the page, first tokens of the value granules (INT_MAX
  // - 8 where no page is listed)
  int ks[2], ko[2], vs[2], vo[2], vt[2];
  auto look_up = [&](int li, int at) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int xk = at + key_granule(u), xv = at + val_granule(u);
      const int pk = p.gpp >= 8 ? (xk >= p.gpp) : (xk * p.gmul) >> 16, pv = p.gpp >= 8 ? (xv >= p.gpp) : (xv * p.gmul) >> 16;
      const int2 ek = pages[li + pk], ev = pages[li + pv];
      ks[u] = ek.x;
      ko[u] = 8 * (xk - pk * p.gpp);
      vs[u] = ev.x;
      vo[u] = 8 * (xv - pv * p.gpp);
      vt[u] = ev.y < 0 ? INT_MAX - 8 : ev.y + vo[u];
    }
  };
  auto load_keys = [&]() {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const size_t head = (size_t)ks[u] * p.Hk + h;
      if constexpr (kMat32) {
        const float* kb = static_cast<const float*>(p.k) + (head * p.P + ko[u] + (c16 & 7)) * D + 4 * g;
#pragma unroll
        for (int c = 0; c < KC; ++c) kc[u][c] = ld_global16(kb + 16 * c);
      } else if constexpr (kEight) {
        const uint8_t* kb = static_cast<const uint8_t*>(p.k) + (head * p.P + ko[u] + (c16 & 3)) * D + 16 * g;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int c = 0; c < KC; ++c) kc[2 * u + i][c] = ld_global16(kb + 4 * i * D + 64 * c);
        ksc[u] = scale_of(p.k_exp[head * p.nb + (ko[u] >> 6)]);
      } else {
        const uint16_t* kb = static_cast<const uint16_t*>(p.k) + (head * p.P + ko[u] + (c16 & 3)) * D + 8 * g;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int c = 0; c < KC; ++c) kc[2 * u + i][c] = ld_global16(kb + 4 * i * D + 32 * c);
      }
    }
  };
  auto load_values = [&]() {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const size_t head = (size_t)vs[u] * p.Hk + h;
      if constexpr (kMat32) {
        const float* vb = static_cast<const float*>(p.v) + (head * D + c16) * p.P + vo[u] + 4 * (g & 1);
#pragma unroll
        for (int m = 0; m < M; ++m) vc[m][u] = ld_global16(vb + (size_t)(16 * m) * p.P);
      } else if constexpr (kEight) {
        const uint8_t* vb = static_cast<const uint8_t*>(p.v) + (head * D + c16) * p.P + vo[u];
#pragma unroll
        for (int m = 0; m < M; ++m) {
          const u32x2a8 x = *reinterpret_cast<const u32x2a8*>(vb + (size_t)(16 * m) * p.P);
          vc[m][0][2 * u] = x[0];
          vc[m][0][2 * u + 1] = x[1];
        }
        vsc[u] = scale_of(p.v_exp[head * p.nb + (vo[u] >> 6)]);
      } else {
        const uint16_t* vb = static_cast<const uint16_t*>(p.v) + (head * D + c16) * p.P + vo[u];
#pragma unroll
        for (int m = 0; m < M; ++m) vc[m][u] = ld_global16(vb + (size_t)(16 * m) * p.P);
      }
    }
  };
  // the value operand of dim block m, half u
  auto values = [&](int m, int u) {
    if constexpr (kEight) return codes_to_bf16(vc[m][0][2 * u], vc[m][0][2 * u + 1], vsc[u]);
    else return vc[m][u];
  };
  // Bit j: whether node i (row `row` of bits) sees token t0 + j.
  auto sees = [&](int row, int i, int t0) -> uint32_t {
    if (t0 >= w.len) return 0u;
    const int rel = t0 - w.base;  // (t0 below len: no overflow)
    if (rel <= -8) return 0xffu;
    uint32_t on;
    if (p.mask) {
      const int x = rel >> 5, sh = rel & 31;
      const uint32_t lo = x < 0 ? ~0u : x < p.words ? bits[row][x] : 0u;
      const uint32_t hi = x + 1 < 0 ? ~0u : x + 1 < p.words ? bits[row][x + 1] : 0u;
      on = (uint32_t)(((uint64_t)hi << 32 | lo) >> sh);
    } else {
      on = low_bits(i + 1 - rel);
    }
    return on & low_bits(min(w.len - t0, 8));
  };

  const int chunk = ((kTreePages - 2) * p.gpp) / kGran;  // tiles whose pages fit the table
  for (int c_lo = t_lo; c_lo < t_hi; c_lo += chunk) {
    const int c_hi = min(c_lo + chunk, t_hi);
    const int li0 = __builtin_amdgcn_readfirstlane(c_lo * kGran / p.gpp), at0 = c_lo * kGran - li0 * p.gpp;
    const int n_pages = (at0 + (c_hi - c_lo) * kGran - 1) / p.gpp + 1;
    if (c_lo > t_lo) __syncthreads();
    for (int x = tid; x < n_pages; x += kThreads) {
      const int li = min(li0 + x, w.n_list - 1);
      const int page = li < w.n_sel ? p.sel[((size_t)b * p.Hk + h) * p.k_max + li] : p.cur_first + li - w.n_sel;
      const int slot = clampi(p.page_table[(size_t)b * p.max_pages + page], 0, p.num_slots - 1);
      pages[x] = int2{slot, li0 + x < w.n_list ? page * p.P : -1};
    }
    __syncthreads();
    int at = at0 + wave * kGran, li = __builtin_amdgcn_readfirstlane(at / p.gpp);
    at -= li * p.gpp;
    const int on_pages = __builtin_amdgcn_readfirstlane(kWaves * kGran / p.gpp), on_rest = kWaves * kGran - on_pages * p.gpp;
    if (c_lo + wave < c_hi) {
      look_up(li, at);
      load_keys();
      load_values();
    }
    for (int t = c_lo + wave; t < c_hi; t += kWaves) {
      const bool more = t + kWaves < c_hi;
      const int tok[2] = {vt[0], vt[1]};
      at += on_rest;
      li += on_pages;
      if (at >= p.gpp) {
        at -= p.gpp;
        ++li;
      }
      if (more) look_up(li, at);
      f32x4 s[kCols][NI];
#pragma unroll
      for (int n = 0; n < kCols; ++n)
#pragma unroll
        for (int i = 0; i < NI; ++i) s[n][i] = f32x4{0};
      if constexpr (kMat32) {
#pragma unroll
        for (int c = 0; c < KC; ++c)
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
              for (int n = 0; n < kCols; ++n) s[n][i] = mfma4(__uint_as_float(kc[i][c][j]), qs[n][c][j], s[n][i]);
      } else {
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
          for (int i = 0; i < NI; ++i) {
            u32x4 a;
            if constexpr (kEight) a = codes_to_bf16(kc[i][c >> 1][2 * (c & 1)], kc[i][c >> 1][2 * (c & 1) + 1], ksc[i >> 1]);
            else a = kc[i][c];
#pragma unroll
            for (int n = 0; n < kCols; ++n)
#pragma unroll
              for (int k = 0; k < kParts; ++k) s[n][i] = mfma16(a, qf[n][c][k], s[n][i]);
          }
      }
      if (more) load_keys();
      // What a node does not see. (tok + 8 does not overflow.)
      bool wild = false;  // some value that not every row sees is no finite number
      uint32_t seen[kCols][2];
      if (__any(max(tok[0], tok[1]) + 8 > w.base)) {
#pragma unroll
        for (int n = 0; n < kCols; ++n)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const uint32_t on = sees(node[n] - i0, node[n], tok[u]);
            seen[n][u] = on;
            if constexpr (kMat32) {
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if (!(on >> (4 * (g & 1) + r) & 1u)) s[n][u][r] = -INFINITY;
            } else {
#pragma unroll
              for (int x = 0; x < 8; ++x)
                if (!(on >> x & 1u)) s[n][2 * u + (x >> 2)][x & 3] = -INFINITY;
            }
          }
        // What lies past the sequence's end may be anything; a weight of 0 would not take a NaN out.
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint32_t in_len = low_bits(clampi(w.len - min(tok[u], w.len), 0, 8));
#pragma unroll
          for (int m = 0; m < M; ++m) {
            if constexpr (kMat32) {
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                if (!(in_len >> (4 * (g & 1) + j) & 1u)) vc[m][u][j] = 0u;
                wild |= (vc[m][u][j] & 0x7f800000u) == 0x7f800000u;
              }
            } else if constexpr (kEight) {
              const uint32_t m4 = ((in_len & 15u) * 0x00204081u & 0x01010101u) * 255u;
              const uint32_t m8 = ((in_len >> 4) * 0x00204081u & 0x01010101u) * 255u;
              vc[m][0][2 * u] &= m4;
              vc[m][0][2 * u + 1] &= m8;
              const u32x4 v = values(m, u);
              wild |= wild2(v[0]) || wild2(v[1]) || wild2(v[2]) || wild2(v[3]);
            } else {
              vc[m][u] = keep8(vc[m][u], in_len);
              wild |= wild2(vc[m][u][0]) || wild2(vc[m][u][1]) || wild2(vc[m][u][2]) || wild2(vc[m][u][3]);
            }
          }
        }
        wild = __any(wild);
      }
      u32x4 pk[kCols][2][kWParts];
#pragma unroll
      for (int n = 0; n < kCols; ++n) {
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[n][i][r]);
        // The reference maximum moves only when a score exceeds it by more than 8 in exp2 units:
        // exponentials stay below 256, and the division by the sum is exact for any reference.
        if (__any(mx * c2 > m_run[n] * c2 + 8.f)) {
          mx = fmaxf(mx, __shfl_xor(mx, 16));
          mx = fmaxf(mx, __shfl_xor(mx, 32));
          const float m_new = mx * c2 > m_run[n] * c2 + 8.f ? mx : m_run[n];
          const float alpha = __builtin_amdgcn_exp2f((m_run[n] - m_new) * c2);
          l_run[n] *= alpha;
#pragma unroll
          for (int m = 0; m < M; ++m) acc[n][m] *= alpha;
          m_run[n] = m_new;
        }
        const float mc = m_run[n] * c2;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
#pragma unroll
          for (int r = 0; r < 4; ++r)
            // (fp32: subtracted before it is scaled, so that large scores lose nothing)
            s[n][i][r] = __builtin_amdgcn_exp2f(sizeof(T) == 2 ? fmaf(s[n][i][r], c2, -mc) : (s[n][i][r] - m_run[n]) * c2);
          sum += (s[n][i][0] + s[n][i][1]) + (s[n][i][2] + s[n][i][3]);
        }
        l_run[n] += sum;
        if constexpr (!kMat32) {
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int k = 0; k < kWParts; ++k)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                f32x4& e = s[n][2 * u + (i >> 1)];
                const uint32_t pair = pack_bf16(e[2 * (i & 1)], e[2 * (i & 1) + 1]);
                pk[n][u][k][i] = pair;
                if (k + 1 < kWParts) {
                  e[2 * (i & 1)] -= bf16_lo(pair);
                  e[2 * (i & 1) + 1] -= bf16_hi(pair);
                }
              }
        }
      }
      if (__builtin_expect(!wild, 1)) {
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            if constexpr (kMat32) {
#pragma unroll
              for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int n = 0; n < kCols; ++n) acc[n][m] = mfma4(__uint_as_float(vc[m][u][j]), s[n][u][j], acc[n][m]);
            } else {
              const u32x4 a = values(m, u);
#pragma unroll
              for (int n = 0; n < kCols; ++n)
#pragma unroll
                for (int k = 0; k < kWParts; ++k) acc[n][m] = mfma16(a, pk[n][u][k], acc[n][m]);
            }
          }
      } else {
        // Row by row, each with the values that it sees (0 times an infinity is NaN).
#pragma unroll
        for (int n = 0; n < kCols; ++n)
          for (int c = 0; c < 16; ++c) {
            const uint32_t on0 = (uint32_t)__shfl((int)seen[n][0], 16 * g + c), on1 = (uint32_t)__shfl((int)seen[n][1], 16 * g + c);
#pragma unroll
            for (int m = 0; m < M; ++m) {
              f32x4 one = f32x4{0};
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                const uint32_t on = u ? on1 : on0;
                if constexpr (kMat32) {
#pragma unroll
                  for (int j = 0; j < 4; ++j)
                    one = mfma4(on >> (4 * (g & 1) + j) & 1u ? __uint_as_float(vc[m][u][j]) : 0.f, s[n][u][j], one);
                } else {
                  const u32x4 a = keep8(values(m, u), on);
#pragma unroll
                  for (int k = 0; k < kWParts; ++k) one = mfma16(a, pk[n][u][k], one);
                }
              }
              if (c16 == c) acc[n][m] += one;
            }
          }
      }
      if (more) load_values();
    }
  }

  // Join the waves: 16 rows at a time through LDS, then kShare threads a row.
#pragma unroll
  for (int n = 0; n < kCols; ++n) {
    l_run[n] += __shfl_xor(l_run[n], 16);
    l_run[n] += __shfl_xor(l_run[n], 32);
    if (g == 0) {
      msm[wave][16 * n + c16] = m_run[n];
      lsm[wave][16 * n + c16] = l_run[n];
    }
  }
  constexpr int kShare = kThreads / 16, N = D / kShare;
  const int col = tid / kShare, d0 = tid % kShare * N;
#pragma unroll
  for (int n = 0; n < kCols; ++n) {
    if (n > 0) __syncthreads();
#pragma unroll
    for (int m = 0; m < M; ++m)
      *reinterpret_cast<f32x4*>(osm + (wave * 16 + c16) * OS + 16 * m + 4 * g) = acc[n][m];
    __syncthreads();
    const int row = 16 * n + col, r = row0 + row, i = r / p.G;
    float m_all = msm[0][row];
#pragma unroll
    for (int x = 1; x < kWaves; ++x) m_all = fmaxf(m_all, msm[x][row]);
    float l = 0.f, o[N] = {};
#pragma unroll
    for (int x = 0; x < kWaves; ++x) {
      const float wt = __builtin_amdgcn_exp2f((msm[x][row] - m_all) * c2);
      l += wt * lsm[x][row];
#pragma unroll
      for (int e = 0; e < N; ++e) o[e] += wt * osm[(x * 16 + col) * OS + d0 + e];
    }
    if (i >= w.q_len) continue;
    if (whole) {
      tree_store<T, N>(p, D, b, i, h * p.G + r % p.G, d0, o, m_all, l, d0 == 0);
    } else {
      const size_t part = ((size_t)bh * p.n_split + split) * p.part_rows + r;
#pragma unroll
      for (int e = 0; e < N; ++e) p.part_o[part * D + d0 + e] = o[e];
      if (d0 == 0) reinterpret_cast<f32x2*>(p.part_ml)[part] = f32x2{m_all, l};
    }
  }
}

// Joins the pieces of a row in an order that does not depend on the launch's timing: kW groups of D / 4
// lanes a row, four dims a lane, each every kW-th piece, then the groups in order.
template <typename T, int D, int kTile, int kW>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeAttnParams p) {
  constexpr int kLanes = D / 4, kRows = 256 / (kLanes * kW);
  __shared__ __attribute__((aligned(16))) float osm[kW == 1 ? 1 : kRows * kW * D];
  __shared__ f32x2 mlsm[kW == 1 ? 1 : kRows * kW];
  const int tid = threadIdx.x, lane = tid & 63;
  const int tiles = (p.part_rows + kRows - 1) / kRows;
  const int bh = __builtin_amdgcn_readfirstlane(blockIdx.x / tiles), b = __builtin_amdgcn_readfirstlane(bh / p.Hk);
  const int h = bh - b * p.Hk;
  const TreeWalk w = tree_walk<kTile>(p, b, h, lane);
  if (w.n_tiles <= p.split_tiles) return;
  const int row = tid / (kLanes * kW), r = (blockIdx.x - bh * tiles) * kRows + row;
  const int grp = tid / kLanes % kW, d0 = 4 * (tid % kLanes), i = r / p.G;
  const bool mine = i < w.q_len && r < p.part_rows;
  const int n = (w.n_tiles + p.split_tiles - 1) / p.split_tiles;
  const size_t part0 = (size_t)bh * p.n_split * p.part_rows + (mine ? r : 0);
  const f32x2* ml = reinterpret_cast<const f32x2*>(p.part_ml);
  float m = -FLT_MAX, l = 0.f, o[4] = {};
#pragma unroll 4
  for (int s = grp; s < n; s += kW) {
    const f32x2 x = ml[part0 + (size_t)s * p.part_rows];
    const f32x4 y = *reinterpret_cast<const f32x4*>(p.part_o + (part0 + (size_t)s * p.part_rows) * D + d0);
    const float top = fmaxf(m, x[0]);
    const float was = __builtin_amdgcn_exp2f((m - top) * p.scale_log2);
    const float add = __builtin_amdgcn_exp2f((x[0] - top) * p.scale_log2);
    l = l * was + add * x[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = o[e] * was + add * y[e];
    m = top;
  }
  if constexpr (kW > 1) {
    *reinterpret_cast<f32x4*>(osm + (row * kW + grp) * D + d0) = f32x4{o[0], o[1], o[2], o[3]};
    if (d0 == 0) mlsm[row * kW + grp] = f32x2{m, l};
    __syncthreads();
    if (grp) return;
    float top = m;
#pragma unroll
    for (int x = 1; x < kW; ++x) top = fmaxf(top, mlsm[row * kW + x][0]);
    l = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = 0.f;
#pragma unroll
    for (int x = 0; x < kW; ++x) {
      const f32x2 y = mlsm[row * kW + x];
      const float wt = __builtin_amdgcn_exp2f((y[0] - top) * p.scale_log2);
      l += wt * y[1];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += wt * osm[(row * kW + x) * D + d0 + e];
    }
    m = top;
  }
  if (mine) tree_store<T, 4>(p, D, b, i, h * p.G + r % p.G, d0, o, m, l, d0 == 0);
}

template <int H, int D, int kCols>
void launch_tree(const TreeAttnParams& p, hipStream_t s) {
  const int groups = p.n_split * p.B * p.Hk;
  tree_attn_kernel<H, D, kCols, 4><<<(groups + 7) / 8 * 8 * p.n_rt, 256, 0, s>>>(p);
}

template <int H, int D>
hipError_t launch_held(const TreeAttnParams& p, hipStream_t s) {
  const int cols = p.rows_per_item / 16;
  if (cols == 1) launch_tree<H, D, 1>(p, s);
  else if (cols == 2) launch_tree<H, D, 2>(p, s);
  else if constexpr (H == kCodes || H == kBf16) launch_tree<H, D, 4>(p, s);
  if (p.n_split > 1) {
    constexpr int kTile = H == kF32 ? 32 : 64;
    // eight groups a row while the rows alone do not fill the chip
    if ((int64_t)p.B * p.Hk * p.part_rows <= 8192) {
      constexpr int kRows = 256 / (D / 4 * (D == 128 ? 8 : 16));
      tree_join_kernel<QType<H>, D, kTile, D == 128 ? 8 : 16><<<p.B * p.Hk * ((p.part_rows + kRows - 1) / kRows), 256, 0, s>>>(p);
    } else {
      constexpr int kRows = 256 / (D / 4);
      tree_join_kernel<QType<H>, D, kTile, 1><<<p.B * p.Hk * ((p.part_rows + kRows - 1) / kRows), 256, 0, s>>>(p);
    }
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_tree_mask(int B, const TreeMaskParams& p, hipStream_t s) {
  tree_mask_kernel<<<B, (p.n + 63) / 64 * 64, 0, s>>>(p);
  return hipGetLastError();
}

int tree_tile(int dtype, bool eight) { return dtype == HSA_DTYPE_F32 && !eight ? 32 : 64; }

int64_t plan_tree(TreeAttnParams& p, int dtype, bool eight, int64_t list) {
  p.nb = (p.P + kScaleTok - 1) / kScaleTok;
  p.gpp = p.P / 8;
  p.gmul = 65536 / p.gpp + 1;
  const int64_t rows = (int64_t)p.n_q * p.G;
  p.rows_per_item = rows <= 16 ? 16 : (rows <= 32 || dtype == HSA_DTYPE_F32 ? 32 : 64);
  p.n_rt = (int)((rows + p.rows_per_item - 1) / p.rows_per_item);
  p.part_rows = p.n_rt * p.rows_per_item;
  const int tile = tree_tile(dtype, eight);
  const int64_t tiles = std::max<int64_t>(1, (list * p.P + tile - 1) / tile);
  const int64_t items = (int64_t)p.B * p.Hk * p.n_rt;
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(kTreeMaxSplit, tiles / 16));
  const int64_t n = std::min((1024 + items - 1) / items, most);
  p.split_tiles = (int)((tiles + n - 1) / n);
  p.n_split = (int)((tiles + p.split_tiles - 1) / p.split_tiles);
  return n * p.part_rows;
}

hipError_t launch_tree_attention(int dtype, int d, bool eight, const TreeAttnParams& p, hipStream_t s) {
  if (eight) {
    if (dtype == HSA_DTYPE_BF16) return d == 128 ? launch_held<kCodes, 128>(p, s) : launch_held<kCodes, 64>(p, s);
    return d == 128 ? launch_held<kCodesF32, 128>(p, s) : launch_held<kCodesF32, 64>(p, s);
  }
  if (dtype == HSA_DTYPE_BF16) return d == 128 ? launch_held<kBf16, 128>(p, s) : launch_held<kBf16, 64>(p, s);
  return d == 128 ? launch_held<kF32, 128>(p, s) : launch_held<kF32, 64>(p, s);
}

}  // namespace hsa
