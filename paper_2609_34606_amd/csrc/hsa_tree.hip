// Attention of drafted trees over the paged caches, and the ancestor bits of their nodes.
//
// A step brings up to HSA_MAX_TREE nodes per sequence, appended behind it as its last tokens. With
// base = length - nodes, node i sees every token before base, and token base + j if bit j of its mask
// row is set (without a mask: j <= i):
//
//   o_i = sum_j softmax_j(scale q_i . k_j) v_j over the tokens it sees.
//
// The H / Hk query heads that share a key head are rows of one product (row r of key head h is head
// h G + r % G of node r / G), so that every key and value is read once for up to 128 rows.
#include <limits.h>

#include <algorithm>
#include <type_traits>

#include "hsa_device.h"
#include "hsa_kernels.h"
#include "hsa_tree.h"

namespace hsa {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------- ancestors
// A node's row is its own bit and its parent's row. Rows double the path they hold with every
// round (row |= row of the node at the end of the path), so a chain of n nodes takes log2(n) rounds, through
// shared memory, a thread a node. Bound: a launch's latency (64 trees of up to 256 nodes: 4.4 us).
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
// The same of fp32 numbers, A[16x4] * B[4x16], k = l/16.
__device__ __forceinline__ f32x4 mfma4(float a, float b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// A sequence's tokens as an item's key head lists them: n_sel selected pages, then pages
// [cur_first, ..), one stream cut into tiles whatever pages they are in.
struct TreeWalk {
  int len, q_len, base;
  int n_sel, n_list, n_tiles;
};

// Every lane of the wave must call it.
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
  w.n_tiles = (w.n_sel * p.P + cur + p.tile - 1) / p.tile;
  return w;
}

// A listed page: where its numbers of the key head begin (of keys and values alike), the page's first token (-1 past
// the list, where it repeats the last page).
struct TreePage {
  int64_t at;
  int first;
};
__device__ __forceinline__ void tree_pages(const TreeAttnParams& p, const TreeWalk& w, int b, int h, int li0, int n,
                                           int D, int tid, int threads, TreePage* pages) {
  for (int x = tid; x < n; x += threads) {
    const int li = min(li0 + x, w.n_list - 1);
    const int page = li < w.n_sel ? p.sel[((size_t)b * p.Hk + h) * p.k_max + li] : p.cur_first + li - w.n_sel;
    const int slot = clampi(p.page_table[(size_t)b * p.max_pages + page], 0, p.num_slots - 1);
    const int64_t head = (int64_t)slot * p.Hk + h;
    pages[x] = TreePage{head * p.P * D, li0 + x < w.n_list ? page * p.P : -1};
  }
}

// A tile's place in the table: list position and granule within the page. Most tiles lie in one page, which is then
// a scalar, as is all that follows from it.
struct TreePlace {
  int li, at;
  bool one;       // the whole tile is in one page
  int64_t base;   // (one) where the page's numbers begin
  int off, first; // (one) the tile's first token, within the page and of the sequence
};
__device__ __forceinline__ void tree_place(const TreeAttnParams& p, const TreePage* pages, int grans, TreePlace& t) {
  t.one = t.at + grans <= p.gpp;
  if (t.one) {
    const TreePage e = pages[t.li];
    t.base = (int64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)e.at) |
             (int64_t)__builtin_amdgcn_readfirstlane((int)(e.at >> 32)) << 32;
    t.off = 8 * t.at;
    t.first = __builtin_amdgcn_readfirstlane(e.first) + t.off;
  }
}
// Granule gr of a tile: its page and token within it.
__device__ __forceinline__ TreePage tree_granule(const TreeAttnParams& p, const TreePage* pages, const TreePlace& t, int gr,
                                                 int& off) {
  const int x = t.at + gr, pg = p.gpp >= 8 ? (x >= p.gpp) : (x * p.gmul) >> 16;
  off = 8 * (x - pg * p.gpp);
  return pages[t.li + pg];
}
__device__ __forceinline__ int tree_token(const TreeAttnParams& p, const TreePage* pages, const TreePlace& t, int gr) {
  if (t.one) return t.first + 8 * gr;
  int off;
  const int first = tree_granule(p, pages, t, gr, off).first;
  return first < 0 ? INT_MAX - 8 : first + off;
}
// 16 bytes at a uniform place plus a thread's own offset (bytes).
__device__ __forceinline__ u32x4 ld_at(const uint8_t* base, uint32_t off) { return ld_global16(base + off); }

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

// A number of the pool.
template <typename T>
__device__ __forceinline__ float pool_value(const TreeAttnParams& p, size_t at) {
  if constexpr (sizeof(T) == 2) return bf16_to_f32(static_cast<const uint16_t*>(p.v)[at]);
  else return static_cast<const float*>(p.v)[at];
}

constexpr int kTreeTile = 32;  // tokens of a tile of up to 32 rows
constexpr int kBriefItems = 256, kBriefTiles = 128;  // little work: most items of 16 rows, tiles of one

// Up to 16 kCols rows of one key head against a range of its tiles. A wave takes every kWaves-th tile and
// keeps an online softmax of its own; the workgroup joins them at the end.
//
// Products are transposed (keys are the rows of S^T = K Q^T, dims those of O^T = V^T P^T), so a lane
// holds scores of one row r = l % 16. Keys take the places in S^T that give a lane the scores of the
// keys whose values it loads, a granule of eight tokens (which never crosses a page) for each part u
// of the tile: weights become the second product's operand without an exchange between lanes. Tiles go
// from memory to the registers of the wave that uses them; the next tile's keys are asked for once this
// one's scores are done with their registers, the values after its output.
//
// Bound: of much work, reading the tokens (32 sequences of 8192 tokens, 8 key heads, d = 128: rows 4 to 32 212 to 248 us,
// 5.1 to 4.3 TB/s; 12 heads, 187200 tokens, 1 and 16 rows 223 and 240 us, 5.2 and 4.8 TB/s); of little, the latency of
// the loads that wait for each other, lengths, page table, tokens (12 heads, one row, 1024 tokens: 10.3 us and the join
// 3.7). Through shared memory, which items of more rows use, each wave would wait for all of them.
template <typename T, int D, int kCols, int kWaves>
__global__ __launch_bounds__(64 * kWaves, kWaves > 4 ? kWaves / 4 : kCols == 1 ? (sizeof(T) == 2 ? 3 : 2) : (sizeof(T) == 2 ? 2 : 1))
void tree_attn_kernel(TreeAttnParams p) {
  constexpr bool kMat32 = sizeof(T) == 4;
  constexpr int kTile = kTreeTile, kGran = kTile / 8;  // tokens, granules of a tile
  constexpr int kU = kMat32 ? 2 : 1;                   // granules of a lane
  constexpr int BU = kMat32 ? 1 : 2;                   // score blocks of 16 keys of a granule
  constexpr int M = D / 16;                            // blocks of output dims
  // bf16 parts of a weight. One rounds it by up to 2^-8, about what the result's own rounding adds; two
  // leave 2^-16. (fp32: none, its products are of fp32.)
  constexpr int kWParts = kCols == 1 ? 2 : 1;
  constexpr int kRows = 16 * kCols, OS = D + 4;
  constexpr int kThreads = 64 * kWaves;
  __shared__ TreePage pages[kTreePages];
  __shared__ uint32_t bits[kRows][kMaskWords + 1];  // mask rows of the item's nodes
  // the queries; at the end 16 rows of each wave's output
  constexpr int QC = kMat32 ? D / 16 : D / 32;  // 16-byte pieces of a row that a lane takes
  constexpr int kSm = std::max(kCols * QC * 64, kWaves * 16 * OS / 4);
  __shared__ u32x4 qsm[kSm];
  float* osm = reinterpret_cast<float*>(qsm);
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
  const TreeWalk w = tree_walk(p, b, h, lane);
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

  // Queries, as the operands that the lanes of every wave take each tile. (In registers they would cost
  // those that hold a tile.)
  int node[kCols];  // of the column's row
#pragma unroll
  for (int n = 0; n < kCols; ++n) node[n] = min((row0 + 16 * n + c16) / p.G, w.q_len - 1);
  for (int x = wave; x < kCols * QC; x += kWaves) {
    const int n = x / QC, c = x % QC, r = row0 + 16 * n + c16, i = min(r / p.G, w.q_len - 1);
    const T* q = static_cast<const T*>(p.q) + (((size_t)b * p.n_q + i) * p.H + h * p.G + r % p.G) * D;
    qsm[x * 64 + lane] = ld_global16(q + (kMat32 ? 16 * c + 4 * g : 32 * c + 8 * g));
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

  u32x4 kc[kU * BU][QC], vc[M][kU];
  // granules of the lane's key rows and of its values
  auto key_granule = [&](int u) { return kMat32 ? 2 * u + (c16 >> 3) : c16 >> 2; };
  auto val_granule = [&](int u) { return kMat32 ? 2 * u + (g >> 1) : g; };
  // the next tile, and a lane's bytes within one page: its key rows of part u, its value row's granules
  TreePlace to;
  constexpr int E = (int)sizeof(T);
  const uint8_t *const kp = static_cast<const uint8_t*>(p.k), *const vp = static_cast<const uint8_t*>(p.v);
  const int sub = kMat32 ? c16 & 7 : c16 & 3, kcol = (kMat32 ? 4 : 8) * g, vsub = kMat32 ? 4 * (g & 1) : 0;
  auto load_keys = [&](int u) {
    const uint8_t* kb;
    uint32_t mine;
    if (to.one) {
      kb = kp + (to.base + (int64_t)to.off * D) * E;
      mine = ((8 * key_granule(u) + sub) * D + kcol) * E;
    } else {
      int off;
      const TreePage e = tree_granule(p, pages, to, key_granule(u), off);
      kb = kp + (e.at + (int64_t)off * D) * E;
      mine = (sub * D + kcol) * E;
    }
#pragma unroll
    for (int i = 0; i < BU; ++i)
#pragma unroll
      for (int c = 0; c < QC; ++c) kc[BU * u + i][c] = ld_at(kb, mine + 4 * i * D * E + 64 * c);
  };
  auto load_values = [&]() {
    const int64_t next = (int64_t)16 * p.P * E;  // to the next block of dims
    if (to.one) {
      const uint8_t* vb = vp + (to.base + to.off) * E;
      const uint32_t row = (uint32_t)c16 * p.P;
#pragma unroll
      for (int m = 0; m < M; ++m) {
#pragma unroll
        for (int u = 0; u < kU; ++u) vc[m][u] = ld_at(vb, (row + 8 * val_granule(u) + vsub) * E);
        vb += next;
      }
    } else {
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        int off;
        const TreePage e = tree_granule(p, pages, to, val_granule(u), off);
        const uint8_t* vb = vp + (e.at + (int64_t)c16 * p.P + off + vsub) * E;
#pragma unroll
        for (int m = 0; m < M; ++m) {
          vc[m][u] = ld_global16(vb);
          vb += next;
        }
      }
    }
  };
  // Values of a granule's tokens that are not in `in_len` become 0, and those of `nodes` that are no finite
  // numbers, which are noted.
  uint32_t wild = 0;
  auto clean_values = [&](int m, int u, uint32_t in_len, uint32_t nodes) {
    if constexpr (kMat32) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t x = vc[m][u][j];
        const uint32_t bad = ((x & 0x7f800000u) + 0x00800000u) & (nodes >> (4 * (g & 1)) << (31 - j) & 0x80000000u);
        wild |= bad;
        vc[m][u][j] = x & ones_if(in_len >> (4 * (g & 1)), j) & ~ones_if(bad, 31);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t x = vc[m][u][j];
        const uint32_t bad = ((x & 0x7f807f80u) + 0x00800080u) & halves2(nodes >> (2 * j));
        wild |= bad;
        vc[m][u][j] = x & fill16(halves2(in_len >> (2 * j))) & ~fill16(bad);
      }
    }
  };
  auto sees = [&](int n, int t0) { return tree_sees(p, w, bits[node[n] - i0], node[n], t0); };

  // A tile whose granules begin at tokens tok (partly: which some row may not see): scores, softmax, output.
  // `after` runs once the keys are done with.
  auto step = [&](bool partly, const int (&tok)[kU], auto&& after) __attribute__((always_inline)) {
    f32x4 s[kCols][kU * BU];
#pragma unroll
    for (int n = 0; n < kCols; ++n)
#pragma unroll
      for (int i = 0; i < kU * BU; ++i) s[n][i] = f32x4{0};
#pragma unroll
    for (int c = 0; c < QC; ++c) {
#pragma unroll
      for (int n = 0; n < kCols; ++n) {
        const u32x4 q = qsm[(n * QC + c) * 64 + lane];
#pragma unroll
        for (int i = 0; i < kU * BU; ++i) {
          if constexpr (kMat32) {
#pragma unroll
            for (int j = 0; j < 4; ++j) s[n][i] = mfma4(__uint_as_float(kc[i][c][j]), __uint_as_float(q[j]), s[n][i]);
          } else {
            s[n][i] = mfma16(kc[i][c], q, s[n][i]);
          }
        }
      }
    }
    // The reference maximum moves only when a score exceeds it by more than 8 in exp2 units:
    // exponentials stay below 256, and the division by the sum is exact for any reference.
    auto raise = [&](int n) __attribute__((always_inline)) {
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < kU * BU; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[n][i][r]);
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
    };
    // What a node does not see. (tok + 8 does not overflow.)
    if (__builtin_expect(partly, 0)) {
#pragma unroll
      for (int n = 0; n < kCols; ++n)
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          const uint32_t on = sees(n, tok[u]) >> (kMat32 ? 4 * (g & 1) : 0);
#pragma unroll
          for (int x = 0; x < 4 * BU; ++x) s[n][u * BU + (x >> 2)][x & 3] = hidden(on, x, s[n][u * BU + (x >> 2)][x & 3]);
        }
      // What lies past the sequence's end may be anything, and becomes 0 (a weight of 0 would not take a NaN
      // out); so does what not every row sees and is no finite number: it reaches its rows at the end.
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const uint32_t in_len = low_bits(clampi(w.len - min(tok[u], w.len), 0, 8));
        const uint32_t node_bits = in_len & ~low_bits(clampi(w.base - min(tok[u], w.base), 0, 8));
#pragma unroll
        for (int m = 0; m < M; ++m) {
          __builtin_amdgcn_sched_barrier(0);  // (one block at a time: registers)
          clean_values(m, u, in_len, node_bits);
        }
      }
    }
    after();
#pragma unroll
    for (int n = 0; n < kCols; ++n) raise(n);
    u32x4 pk[kCols][kU][kWParts];
#pragma unroll
    for (int n = 0; n < kCols; ++n) {
      const float mc = m_run[n] * c2;
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < kU * BU; ++i) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          // (fp32: subtracted before it is scaled, so that large scores lose nothing)
          s[n][i][r] = __builtin_amdgcn_exp2f(sizeof(T) == 2 ? fmaf(s[n][i][r], c2, -mc) : (s[n][i][r] - m_run[n]) * c2);
        sum += (s[n][i][0] + s[n][i][1]) + (s[n][i][2] + s[n][i][3]);
      }
      l_run[n] += sum;
      if constexpr (!kMat32) {
#pragma unroll
        for (int u = 0; u < kU; ++u)
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
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        if constexpr (kMat32) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int n = 0; n < kCols; ++n) acc[n][m] = mfma4(__uint_as_float(vc[m][u][j]), s[n][u][j], acc[n][m]);
        } else {
#pragma unroll
          for (int n = 0; n < kCols; ++n)
#pragma unroll
            for (int k = 0; k < kWParts; ++k) acc[n][m] = mfma16(vc[m][u], pk[n][u][k], acc[n][m]);
        }
      }
  };

  const int chunk = ((kTreePages - 2) * p.gpp) / kGran;  // tiles whose pages fit the table
  for (int c_lo = t_lo; c_lo < t_hi; c_lo += chunk) {
    const int c_hi = min(c_lo + chunk, t_hi);
    const int li0 = __builtin_amdgcn_readfirstlane(c_lo * kGran / p.gpp), at0 = c_lo * kGran - li0 * p.gpp;
    const int n_pages = (at0 + (c_hi - c_lo) * kGran - 1) / p.gpp + 1;
    if (c_lo > t_lo) __syncthreads();
    tree_pages(p, w, b, h, li0, n_pages, D, tid, kThreads, pages);
    __syncthreads();
    to.at = at0 + wave * kGran;
    to.li = __builtin_amdgcn_readfirstlane(to.at / p.gpp);
    to.at -= to.li * p.gpp;
    const int on_pages = __builtin_amdgcn_readfirstlane(kWaves * kGran / p.gpp), on_rest = kWaves * kGran - on_pages * p.gpp;
    if (c_lo + wave < c_hi) {
      tree_place(p, pages, kGran, to);
#pragma unroll
      for (int u = 0; u < kU; ++u) load_keys(u);
      load_values();
    }
    for (int t = c_lo + wave; t < c_hi; t += kWaves) {
      const bool more = t + kWaves < c_hi;
      const TreePlace now = to;
      to.at += on_rest;
      to.li += on_pages;
      if (to.at >= p.gpp) {
        to.at -= p.gpp;
        ++to.li;
      }
      if (more) tree_place(p, pages, kGran, to);
      const bool partly = !now.one || now.first + kTile > w.base;  // (some row may not see all of it)
      int tok[kU];
      if (partly) {
#pragma unroll
        for (int u = 0; u < kU; ++u) tok[u] = tree_token(p, pages, now, val_granule(u));
      }
      step(partly, tok, [&]() __attribute__((always_inline)) {
        if (more) {
#pragma unroll
          for (int u = 0; u < kU; ++u) load_keys(u);
        }
      });
      if (more) load_values();
    }
  }

  // (the waves' tiles are not each other's: any of them may have seen one)
  if (__syncthreads_or(wild != 0) && wave == 0)
    tree_wild(p, w, b, h, D, t_lo * kGran, t_hi * kGran, [&](size_t, size_t at, int) { return pool_value<T>(p, at); }, [&](int t0, int j, auto&& value) {
#pragma unroll
      for (int n = 0; n < kCols; ++n)
        if (sees(n, t0) >> j & 1u) {
#pragma unroll
          for (int m = 0; m < M; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[n][m][r] += value(16 * m + 4 * g + r);
        }
    });
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
      for (int e = 0; e < N; ++e) o[e] = add_share(o[e], osm[(x * 16 + col) * OS + d0 + e], wt);
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

// More rows: 32 kRG rows of one key head (kRG = 2 or 4) against a range of its tiles of 64 tokens. Four waves, two
// workgroups a CU; a tile goes once from the registers that it arrived in to LDS, and is read from
// there by all waves: with kRG = 4 each takes 32 rows, with two 32 rows and half of the tile's tokens.
//
// Products are transposed as above, 32x32x16, with key rows in an order that makes a lane's scores the
// weights' operand. A tile's loads are two tiles ahead of its products (three spilled registers: 159 and 288 us for the
// calls below).
// Bound: up to 64 rows, reading the tokens (64 rows, 12 heads over 187200 tokens: 203 to 222 us, 5.7 to 5.2 TB/s; a ragged
// batch of up to 64 rows over up to 8192 tokens 127 to 134 us, 4.4 TB/s, the first kernel here, whose waves each
// loaded 64 rows' tiles for themselves, 250); of more, the matrix and vector instructions, which the two
// workgroups of a CU overlap in part (256 rows, 32 sequences of 8192 tokens, 8 key heads: with lengths given, in
// pieces of 16 tiles, 440 to 450 us, 610 to 625 TFLOP/s; without 343 us, 800).
// A weight is one bf16 part, rounded by up to 2^-8 of it (their sum is of the fp32 ones): the result is off by 2.1e-3 of its
// norm for the ragged batch and 1.7e-3 for the long list, its own rounding alone by 1.7e-3 and 1.6e-3. A second part would
// be half as many matrix instructions again.
template <int D, int kRG>
struct TreeWide {
  static constexpr int kThreads = 256, kRows = 32 * kRG;
  static constexpr int kRowK = 2 * D, kTileK = 64 * kRowK, kRowV = 128, kTileV = D * kRowV;  // bytes
  static constexpr int kBytes = 2 * (kTileK + kTileV);
  // 16-byte pieces of a tile that a thread loads, keys and values alike
  static constexpr int kPieces = 64 * D * 2 / 16 / kThreads;
  // 16-byte chunks of a row, permuted so that rows read together fall on their own banks
  static __device__ __forceinline__ int swz_k(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
  static __device__ __forceinline__ int swz_v(int row) { return (row >> 1) & 7; }
};

template <int D, int kRG>
__global__ __launch_bounds__(256, 2) void tree_wide_kernel(TreeAttnParams p) {
  using L = TreeWide<D, kRG>;
  constexpr int KK = D / 16, NM = D / 32, NP = L::kPieces, kRows = L::kRows;
  constexpr int KH = kRG / 2;  // halves of a tile that a wave takes
  __shared__ __attribute__((aligned(1024))) uint8_t smem[L::kBytes];
  __shared__ TreePage pages[kTreePages];
  __shared__ uint32_t bits[kRows][kMaskWords + 1];
  __shared__ int wild;  // whether a value that not every row sees is no finite number
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int per8 = 8 * p.n_rt;
  const int oct = __builtin_amdgcn_readfirstlane(blockIdx.x / per8), in = blockIdx.x - oct * per8;
  // (Neighbours on an XCD go round its four shader engines: a ragged batch's last row tiles and pieces take turns
  // at which engine has them: 32 sequences of up to 256 rows over up to 8192 tokens 231 us and, so, 207; 100 of up to 160
  // over up to 4096 317 and 261. The register kernel gains nothing by it: one node each 132
  // and 136.)
  const int rt = __builtin_amdgcn_readfirstlane(((in >> 3) + oct + (oct >> 1)) % p.n_rt);
  const int group = oct * 8 + (in & 7), heads = p.B * p.Hk;
  const int split = __builtin_amdgcn_readfirstlane(group / heads);
  if (split >= p.n_split) return;
  const int bh = __builtin_amdgcn_readfirstlane((group - split * heads + 8 * split) % heads);
  const int b = __builtin_amdgcn_readfirstlane(bh / p.Hk), h = bh - b * p.Hk;
  const TreeWalk w = tree_walk(p, b, h, lane);
  const int row0 = rt * kRows, rows = w.q_len * p.G;
  if (row0 >= rows) return;
  const int t_lo = split * p.split_tiles, t_hi = min(t_lo + p.split_tiles, w.n_tiles);
  if (split > 0 && t_lo >= w.n_tiles) return;
  const bool whole = w.n_tiles <= p.split_tiles;

  const int i0 = __builtin_amdgcn_readfirstlane(row0 / p.G);
  if (p.mask) {
    const int nodes = min((row0 + kRows - 1) / p.G, w.q_len - 1) - i0 + 1;
    const uint32_t* src = p.mask + ((size_t)b * p.n_q + i0) * p.words;
    for (int x = tid; x < nodes * p.words; x += 256) bits[x / p.words][x % p.words] = src[x];
  }
  if (tid == 0) wild = 0;

  // the wave's rows, and with kRG = 2 its half of a tile
  const int wrow = row0 + 32 * (wave % kRG), kh0 = kRG == 2 ? wave >> 1 : 0;
  const bool active = wrow < rows;
  const int r = wrow + l32, node = min(r / p.G, w.q_len - 1);
  u32x4 qf[KK];
  {
    const uint16_t* q =
        static_cast<const uint16_t*>(p.q) + (((size_t)b * p.n_q + node) * p.H + h * p.G + min(r, rows - 1) % p.G) * D + 8 * half;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) qf[kk] = ld_global16(q + 16 * kk);
  }
  f32x16 acc[NM];
#pragma unroll
  for (int m = 0; m < NM; ++m) acc[m] = f32x16{0};
  const float c2 = p.scale_log2;
  float m_run = softmax_floor(c2), l_run = 0.f;

  // Bit j: whether the lane's row sees token t0 + j.
  auto sees = [&](int t0) __attribute__((always_inline)) { return tree_sees(p, w, bits[p.mask ? node - i0 : 0], node, t0); };

  // A thread's pieces of a tile: key row and chunk, value row and granule.
  u32x4 kc[NP], vc[NP];
  auto krow_of = [&](int i) { return (tid + 256 * i) / (D / 8); };
  const int kcol = tid % (D / 8);
  const int vgran = tid & 7;
  auto vrow_of = [&](int i) { return (tid + 256 * i) / 8; };
  constexpr int E = 2;
  const uint8_t *const kp = static_cast<const uint8_t*>(p.k), *const vp = static_cast<const uint8_t*>(p.v);
  const uint32_t vrow = vrow_of(0) * (uint32_t)p.P * E + 8 * vgran * E;  // (within one page)
  auto load = [&](const TreePlace& t) __attribute__((always_inline)) {
    const int64_t next = (int64_t)32 * p.P * E;  // to the thread's next value row
    if (t.one) {
      const uint8_t *kb = kp + (t.base + (int64_t)t.off * D) * E, *vb = vp + (t.base + t.off) * E;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        kc[i] = ld_at(kb, 16 * (tid + 256 * i));
      }
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        vc[i] = ld_at(vb, vrow);
        vb += next;
      }
    } else {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        int off;
        const int row = krow_of(i);
        const TreePage e = tree_granule(p, pages, t, row >> 3, off);
        kc[i] = ld_global16(kp + (e.at + (int64_t)(off + (row & 7)) * D + kcol * 8) * E);
      }
      int off;
      const TreePage e = tree_granule(p, pages, t, vgran, off);
      const uint8_t* vb = vp + (e.at + (int64_t)vrow_of(0) * p.P + off) * E;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        vc[i] = ld_global16(vb);
        vb += next;
      }
    }
  };
  // What lies past the sequence's end may be anything, and becomes 0; so does what not every row sees and
  // is no finite number (it reaches the rows that see it at the end).
  auto clean = [&](u32x4 v, int t0) __attribute__((always_inline)) {
    uint32_t on = low_bits(clampi(w.len - min(t0, w.len), 0, 8));
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      const bool bad = (v[x >> 1] >> (16 * (x & 1)) & 0x7f80u) == 0x7f80u;
      if (bad && t0 + x >= w.base && (on >> x & 1u)) {
        on &= ~(1u << x);
        wild = 1;
      }
    }
    return keep8(v, on);
  };
  auto put = [&](int buf, const TreePlace& t) __attribute__((always_inline)) {
    uint8_t* ksm = smem + buf * (L::kTileK + L::kTileV);
    uint8_t* vsm = ksm + L::kTileK;
    const bool some = !t.one || t.first + 64 > w.base;  // (some row may not see all of it)
    const int t0 = some ? tree_token(p, pages, t, vgran) : 0;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int row = krow_of(i), dim = vrow_of(i);
      uint8_t* kd = ksm + row * L::kRowK;
      uint8_t* vd = vsm + dim * L::kRowV;
      *reinterpret_cast<u32x4*>(kd + ((kcol ^ L::swz_k(row)) << 4)) = kc[i];
      *reinterpret_cast<u32x4*>(vd + ((vgran ^ L::swz_v(dim)) << 4)) = __builtin_expect(some, 0) ? clean(vc[i], t0) : vc[i];
    }
  };

  const int krow = (l32 & ~12) | ((l32 & 4) << 1) | ((l32 & 8) >> 1);  // bits 2 and 3 swapped
  auto compute = [&](const TreePlace& t, int buf) __attribute__((always_inline)) {
    const uint8_t* ksm = smem + buf * (L::kTileK + L::kTileV);
    const uint8_t* vsm = ksm + L::kTileK;
    f32x16 s[KH];
#pragma unroll
    for (int x = 0; x < KH; ++x) {
      s[x] = f32x16{0};
      const uint8_t* row = ksm + (32 * (kh0 + x) + krow) * L::kRowK;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) s[x] = mfma32(ld_lds16(row + (((2 * kk + half) ^ L::swz_k(krow)) << 4)), qf[kk], s[x]);
    }
    if (__builtin_expect(!t.one || t.first + 64 > w.base, 0)) {
#pragma unroll
      for (int x = 0; x < KH; ++x)
#pragma unroll
        for (int gr = 0; gr < 2; ++gr) {
          const uint32_t on = sees(tree_token(p, pages, t, 4 * (kh0 + x) + 2 * gr + half));
#pragma unroll
          for (int j = 0; j < 8; ++j) s[x][8 * gr + j] = hidden(on, j, s[x][8 * gr + j]);
        }
    }
    // The reference maximum moves only when a score exceeds it by more than 8 in exp2 units.
    float mx = s[0][0];
#pragma unroll
    for (int x = 0; x < KH; ++x)
#pragma unroll
      for (int j = 0; j < 16; ++j) mx = fmaxf(mx, s[x][j]);
    if (__any(mx * c2 > m_run * c2 + 8.f)) {
      const float top = fmaxf(mx, __shfl_xor(mx, 32));
      const float m_new = top * c2 > m_run * c2 + 8.f ? top : m_run;
      const float alpha = __builtin_amdgcn_exp2f((m_run - m_new) * c2);
      l_run *= alpha;
#pragma unroll
      for (int m = 0; m < NM; ++m) acc[m] *= alpha;
      m_run = m_new;
    }
    const float mc = m_run * c2;
    u32x4 pk[KH][2];
#pragma unroll
    for (int x = 0; x < KH; ++x)
#pragma unroll
      for (int gr = 0; gr < 2; ++gr) {
        float sum[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float e = __builtin_amdgcn_exp2f(fmaf(s[x][8 * gr + 2 * j], c2, -mc));
          const float f = __builtin_amdgcn_exp2f(fmaf(s[x][8 * gr + 2 * j + 1], c2, -mc));
          sum[j] = e + f;
          pk[x][gr][j] = pack_bf16(e, f);
        }
        l_run += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      }
#pragma unroll
    for (int x = 0; x < KH; ++x)
#pragma unroll
      for (int gr = 0; gr < 2; ++gr)
#pragma unroll
        for (int m = 0; m < NM; ++m)
          acc[m] = mfma32(ld_lds16(vsm + (32 * m + l32) * L::kRowV +
                                   (((4 * (kh0 + x) + 2 * gr + half) ^ L::swz_v(l32)) << 4)), pk[x][gr], acc[m]);
  };

  const int chunk = ((kTreePages - 2) * p.gpp) / 8;  // tiles whose pages fit the table
  for (int c_lo = t_lo; c_lo < t_hi; c_lo += chunk) {
    const int n = min(chunk, t_hi - c_lo);
    const int li0 = __builtin_amdgcn_readfirstlane(c_lo * 8 / p.gpp), at0 = c_lo * 8 - li0 * p.gpp;
    if (c_lo > t_lo) __syncthreads();
    tree_pages(p, w, b, h, li0, (at0 + n * 8 - 1) / p.gpp + 1, D, tid, 256, pages);
    __syncthreads();
    const int on_pages = __builtin_amdgcn_readfirstlane(8 / p.gpp), on_rest = 8 - on_pages * p.gpp;
    auto next = [&](const TreePlace& from) {
      TreePlace t = from;
      t.at += on_rest;
      t.li += on_pages;
      if (t.at >= p.gpp) {
        t.at -= p.gpp;
        ++t.li;
      }
      tree_place(p, pages, 8, t);
      return t;
    };
    TreePlace now, ahead;  // the tile computed, the one after it (its loads are on their way)
    now.li = 0;
    now.at = at0;
    tree_place(p, pages, 8, now);
    load(now);
    put(0, now);
    if (n > 1) {
      ahead = next(now);
      load(ahead);
    }
    lds_barrier();
    for (int t = 0; t < n; ++t) {
      if (active) compute(now, t & 1);
      if (t + 1 < n) {
        put((t + 1) & 1, ahead);
        now = ahead;
      }
      if (t + 2 < n) {
        ahead = next(now);
        load(ahead);
      }
      lds_barrier();
    }
  }
  __syncthreads();
  if (wild && active && kh0 == 0) {
    // (what was taken out of the tiles, for the rows that see it)
    tree_wild(p, w, b, h, D, t_lo * 8, t_hi * 8, [&](size_t, size_t at, int) { return pool_value<uint16_t>(p, at); }, [&](int t0, int j, auto&& value) {
      if (sees(t0) >> j & 1u) {
#pragma unroll
        for (int m = 0; m < NM; ++m)
#pragma unroll
          for (int x = 0; x < 16; ++x) acc[m][x] += value(32 * m + 8 * (x >> 2) + 4 * half + (x & 3));
      }
    });
  }
  const int row = wrow + l32, i = row / p.G;
  float l = l_run + __shfl_xor(l_run, 32);
  if constexpr (kRG == 2) {
    // join the two halves of the tiles: the second one's sums go through LDS
    __syncthreads();
    float* osm = reinterpret_cast<float*>(smem) + (wave & 1) * (32 * D + 64);
    if (kh0 == 1) {
#pragma unroll
      for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int x = 0; x < 4; ++x)  // [dims / 4][row], so that lanes write side by side
          *reinterpret_cast<f32x4*>(osm + ((8 * m + 2 * x + half) * 32 + l32) * 4) =
              f32x4{acc[m][4 * x], acc[m][4 * x + 1], acc[m][4 * x + 2], acc[m][4 * x + 3]};
      if (half == 0) {
        osm[32 * D + l32] = m_run;
        osm[32 * D + 32 + l32] = l;
      }
    }
    __syncthreads();
    if (kh0 == 1) return;
    const float m_other = osm[32 * D + l32], top = fmaxf(m_run, m_other);
    const float a = __builtin_amdgcn_exp2f((m_run - top) * c2), c = __builtin_amdgcn_exp2f((m_other - top) * c2);
    l = a * l + c * osm[32 * D + 32 + l32];
    // (a choice for each number instead: the ragged batch above 144 us for 139)
    if (__builtin_expect(__any(fminf(a, c) == 0.f), 0)) {
#pragma unroll
      for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int x = 0; x < 16; ++x)
          acc[m][x] = add_share(add_share(0.f, acc[m][x], a), osm[((8 * m + 2 * (x >> 2) + half) * 32 + l32) * 4 + (x & 3)], c);
    } else {
#pragma unroll
      for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const f32x4 y = *reinterpret_cast<const f32x4*>(osm + ((8 * m + 2 * x + half) * 32 + l32) * 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[m][4 * x + e] = a * acc[m][4 * x + e] + c * y[e];
        }
    }
    m_run = top;
  }
  if (!active || i >= w.q_len) return;
  if (whole) {
    const int head = h * p.G + row % p.G;
#pragma unroll
    for (int m = 0; m < NM; ++m)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const float o[4] = {acc[m][4 * x], acc[m][4 * x + 1], acc[m][4 * x + 2], acc[m][4 * x + 3]};
        tree_store<uint16_t, 4>(p, D, b, i, head, 32 * m + 8 * x + 4 * half, o, m_run, l, m == 0 && x == 0 && half == 0);
      }
  } else {
    const size_t part = ((size_t)bh * p.n_split + split) * p.part_rows + row;
#pragma unroll
    for (int m = 0; m < NM; ++m)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        *reinterpret_cast<f32x4*>(p.part_o + part * D + 32 * m + 8 * x + 4 * half) =
            f32x4{acc[m][4 * x], acc[m][4 * x + 1], acc[m][4 * x + 2], acc[m][4 * x + 3]};
    if (half == 0) reinterpret_cast<f32x2*>(p.part_ml)[part] = f32x2{m_run, l};
  }
}

// Joins the pieces of a row in an order that does not depend on the launch's timing: kW groups of D / 4
// lanes a row, four dims a lane, each every kW-th piece, then the groups in order. Bound: reading the pieces
// (16384 rows of up to 8: 9.1 us), of few rows a launch and a few loads after another (12 rows of 6: 2.8 us).
template <typename T, int D, int kW>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeAttnParams p) {
  constexpr int kLanes = D / 4, kRows = 256 / (kLanes * kW);
  __shared__ __attribute__((aligned(16))) float osm[kW == 1 ? 1 : kRows * kW * D];
  __shared__ f32x2 mlsm[kW == 1 ? 1 : kRows * kW];
  const int tid = threadIdx.x, lane = tid & 63;
  const int tiles = (p.part_rows + kRows - 1) / kRows;
  const int bh = __builtin_amdgcn_readfirstlane(blockIdx.x / tiles), b = __builtin_amdgcn_readfirstlane(bh / p.Hk);
  const int h = bh - b * p.Hk;
  const TreeWalk w = tree_walk(p, b, h, lane);
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
  if (__builtin_expect(mine && !all_finite(o), 0)) {
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = 0.f;
#pragma unroll 1
    for (int s = 0; s < n; ++s) {
      const float share = __builtin_amdgcn_exp2f((ml[part0 + (size_t)s * p.part_rows][0] - m) * p.scale_log2);
      const float* y = p.part_o + (part0 + (size_t)s * p.part_rows) * D + d0;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = add_share(o[e], y[e], share);
    }
  }
  if (mine) tree_store<T, 4>(p, D, b, i, h * p.G + r % p.G, d0, o, m, l, d0 == 0);
}

// Waves of a workgroup where the whole call is little work: as many as the registers allow (12 heads, one query, 1024
// tokens, d = 128: 8 waves 14.1 us, 16, which spill, 24.7).
constexpr int brief_waves(size_t size, int d) { return size == 4 || d == 128 ? 8 : 16; }

// Tiles of 32 tokens up to which items of 16 rows are little work. (Up to 16 rows a key head the other workgroups read
// every token once too.) In us, as little work and not: 12 heads, one row, 1024 tokens 13.8 and 15.8; 8 key heads, 64
// rows, 1024 and 4096 tokens 13.6 and 24.0, 22.7 and 27.8; 4 sequences of 2000, 4 key heads, 240 rows, d = 64 21.6 and
// 30.9; fp32, 2 sequences of 2000, 8 heads, one row 20.8 and 25.9.
int64_t brief_tiles(int64_t items16, int64_t rows) {
  return items16 > kBriefItems ? 0 : rows <= 16 ? 4096 / items16 : std::min<int64_t>(kBriefTiles, 16384 / items16);
}
// Rows of an item otherwise, and the most pieces that its list is cut into: of 16 tiles, which balance ragged lists (up to
// 64 rows, up to 8192 tokens: pieces of 16 tiles 139 us, of 8 154), while they make fewer than 4096 workgroups (1024:
// 149 us; 2048 to 8192: 139). fp32 has registers for 32 rows.
int tree_rows(int dtype, int64_t rows) {
  return rows <= 16 ? 16 : (rows <= 32 || dtype == HSA_DTYPE_F32 ? 32 : (rows <= 64 ? 64 : 128));
}
int64_t tree_pieces(int64_t items, int64_t tiles) {
  return std::max<int64_t>(1, std::min<int64_t>({kTreeMaxSplit, tiles / 16, (4096 + items - 1) / items}));
}

template <typename T, int D>
hipError_t launch_pool(const TreeAttnParams& p, hipStream_t s) {
  const int grid = (p.n_split * p.B * p.Hk + 7) / 8 * 8 * p.n_rt;
  if (p.waves > 4) tree_attn_kernel<T, D, 1, brief_waves(sizeof(T), D)><<<grid, 64 * brief_waves(sizeof(T), D), 0, s>>>(p);
  else if (p.rows_per_item == 16) tree_attn_kernel<T, D, 1, 4><<<grid, 256, 0, s>>>(p);
  else if (p.rows_per_item == 32) tree_attn_kernel<T, D, 2, 4><<<grid, 256, 0, s>>>(p);
  else if constexpr (sizeof(T) == 2) {
    if (p.rows_per_item == 64) tree_wide_kernel<D, 2><<<grid, 256, 0, s>>>(p);
    else tree_wide_kernel<D, 4><<<grid, 256, 0, s>>>(p);
  }
  if (p.n_split > 1) {
    // several groups of lanes a row while the rows alone do not fill the chip (12 heads, 187200 tokens, 16 and 1 rows, in
    // us of both kernels: 240 and 223, with one group 255 and 238; 4096 rows of 16 pieces 35.0 and 30.6)
    constexpr int kMost = 256 / (D / 4);  // rows of a workgroup
    if ((int64_t)p.B * p.Hk * p.part_rows <= 2048)
      tree_join_kernel<T, D, kMost><<<p.B * p.Hk * p.part_rows, 256, 0, s>>>(p);
    else
      tree_join_kernel<T, D, 1><<<p.B * p.Hk * ((p.part_rows + kMost - 1) / kMost), 256, 0, s>>>(p);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_tree_mask(int B, const TreeMaskParams& p, hipStream_t s) {
  tree_mask_kernel<<<B, (p.n + 63) / 64 * 64, 0, s>>>(p);
  return hipGetLastError();
}

void plan_tree(TreeAttnParams& p, int dtype, int d, int64_t list, bool ragged) {
  p.gpp = p.P / 8;
  p.gmul = 65536 / p.gpp + 1;
  const int64_t rows = (int64_t)p.n_q * p.G;
  auto tiles_of = [&](int tile) { return std::max<int64_t>(1, (list * p.P + tile - 1) / tile); };
  // Little work: what counts is how many tiles a wave does after one another, and a second launch if they
  // are cut.
  const int64_t items16 = (int64_t)p.B * p.Hk * ((rows + 15) / 16), tiles32 = tiles_of(kTreeTile);
  const bool brief = tiles32 <= brief_tiles(items16, rows);
  p.waves = brief ? brief_waves(dtype == HSA_DTYPE_BF16 ? 2 : 4, d) : 4;
  p.rows_per_item = brief ? 16 : tree_rows(dtype, rows);
  p.n_rt = (int)((rows + p.rows_per_item - 1) / p.rows_per_item);
  p.part_rows = p.n_rt * p.rows_per_item;
  p.tile = p.rows_per_item > 32 ? 64 : kTreeTile;
  const int64_t tiles = tiles_of(p.tile), items = (int64_t)p.B * p.Hk * p.n_rt;
  // pieces that little work may be cut into
  auto may = [&](int64_t k) { return k <= kTreeMaxSplit && k * items16 <= 512 && p.waves * (k - 1) < tiles32; };
  int64_t n = 1;
  if (brief) {
    // in us: a tile after another 1.7, the join 4.5
    double best = 1e300;
    for (int64_t k = 1; k == 1 || may(k); ++k) {
      const double t = 1.7 * (double)((tiles + p.waves * k - 1) / (p.waves * k)) + (k > 1 ? 4.5 : 0.0);
      if (t < best) {
        best = t;
        n = k;
      }
    }
  } else {
    n = tree_pieces(items, tiles);
    if (!ragged && p.rows_per_item > 32) {
      // Equal lists, two workgroups a CU: rounds of them, each of its tiles and about eight more for its start, end and
      // part of the join (64 nodes of 12 heads over 187200 tokens: 42 pieces, one round, 217 us, 85 241, 128 249; of
      // 32 heads, 8 key heads, over 65536, 106 and, in 64, 116). Pieces of ragged lists end at different times
      // anyway, and many short ones balance.
      int64_t best = INT64_MAX;
      for (int64_t k = 1, most = n; k <= most; ++k) {
        const int64_t t = (items * k + 511) / 512 * ((tiles + k - 1) / k + 8);
        if (t < best) {
          best = t;
          n = k;
        }
      }
    }
  }
  p.split_tiles = (int)((tiles + n - 1) / n);
  p.n_split = (int)((tiles + p.split_tiles - 1) / p.split_tiles);
}

int64_t tree_part_rows(int dtype, int d, int P, int64_t heads, int64_t rows, int64_t list) {
  const int64_t items16 = heads * ((rows + 15) / 16), tiles32 = (list * P + kTreeTile - 1) / kTreeTile;
  int64_t most = 0;
  auto take = [&](int64_t pieces, int64_t per_item) {
    if (pieces > 1) most = std::max(most, pieces * ((rows + per_item - 1) / per_item * per_item));
  };
  if (items16 <= kBriefItems) {  // as many pieces as the longest list of little work may be cut into
    const int64_t longest = std::min(tiles32, brief_tiles(items16, rows)), waves = brief_waves(dtype == HSA_DTYPE_BF16 ? 2 : 4, d);
    take(std::min<int64_t>({kTreeMaxSplit, 512 / items16, (longest - 1) / waves + 1}), 16);
  }
  if (tiles32 > brief_tiles(items16, rows)) {
    const int64_t per = tree_rows(dtype, rows), tile = per > 32 ? 64 : kTreeTile;
    take(tree_pieces(heads * ((rows + per - 1) / per), (list * P + tile - 1) / tile), per);
  }
  return most;
}

hipError_t launch_tree_attention(int dtype, int d, const TreeAttnParams& p, hipStream_t s) {
  if (dtype == HSA_DTYPE_BF16) return d == 128 ? launch_pool<uint16_t, 128>(p, s) : launch_pool<uint16_t, 64>(p, s);
  return d == 128 ? launch_pool<float, 128>(p, s) : launch_pool<float, 64>(p, s);
}

}  // namespace hsa
