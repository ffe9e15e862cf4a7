// Attention over the 8-bit cache: exact softmax attention of a step's queries over
// the tokens of the listed pages (selected pages, then a run of pages), up to each
// sequence's length and, with the causal mask, up to each query's own token.
//
//   o_i = sum_j softmax_j(scale q_i . k_j) v_j,  k_j = 2^(e of its block) code_j, v_j alike.
//
// The H / Hk query heads that share a key head are rows of one product: row r of
// key head h is head h G + r % G of query r / G, so a step of one token
// reads every code once. Codes become bf16 matrix operands on the way (exactly:
// see hsa_fp8.h), so keys and values are never in HBM in more than 8 bits.
#include <limits.h>

#include <type_traits>

#include "hsa_cache8.h"

namespace hsa {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kMaxSplit = 256;  // pieces of one item

// D[16x16] += A[16x32] * B[32x16]. Lane l supplies A row (l % 16), k =
// 8*(l/16)..+8, and B column (l % 16), same k range. Result register r of
// lane l holds row 4*(l/16) + r, column l % 16.
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
}

// Byte masks that keep the first n (0..16) of 16 codes.
__device__ __forceinline__ u32x4 keep_codes(u32x4 v, int n) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = clampi(n - 4 * i, 0, 4);
    v[i] = m == 4 ? v[i] : v[i] & ((1u << (8 * m)) - 1u);
  }
  return v;
}

// Eight elements of T in kParts bf16 operands whose sum is the element: one for
// bf16, three for fp32 (3 x 8 significant bits).
template <typename T, int kParts>
__device__ __forceinline__ void split_row(const T* p, u32x4 (&f)[kParts]) {
  if constexpr (kParts == 1) {
    f[0] = ld_global16(p);
  } else {
    float x[8];
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = a[i];
      x[4 + i] = b[i];
    }
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[k][i] = pack_bf16(x[2 * i], x[2 * i + 1]);
        x[2 * i] -= bf16_lo(f[k][i]);
        x[2 * i + 1] -= bf16_hi(f[k][i]);
      }
      // an infinity is its first part alone
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = fabsf(x[i]) < INFINITY ? x[i] : 0.f;
    }
  }
}

// Few query rows: 16 kCols rows of one key head against a range of its tokens. A wave takes
// every kWaves-th 64-key tile and keeps an online softmax of its own; the workgroup
// joins them at the end. Four waves, or eight where the whole call is little work (plan_cache8).
//
// Products are transposed (keys are the rows of S^T = K Q^T, dims those of O^T = V^T P^T),
// so a lane holds scores of one query and the 16 keys of its quarter. Row m of
// score block i is key 16 (m / 4) + 4 i + m % 4: a quarter of lanes then
// holds 16 consecutive keys, in the order in which the value operand, 16 consecutive codes
// of a d-major row, has them, and the weights need no exchange between lanes. Codes go
// from HBM to the registers of the wave that uses them, 16 bytes a lane; a
// score block's rows are read in 64-byte pieces, a value block's too. The keys of a wave's next
// tile are asked for once this one's scores are done with their registers, the values after its
// output; other waves of the CU (three workgroups of 168 registers) cover the rest.
// Bound: HBM (2 d bytes a token and key head): 32 sequences of 1 to 16384 tokens, 32 query and 8 key
// heads, 560 MB in 124 us, 4.6 TB/s; one token over 187200 of 12 heads, 575 MB in 127 us.
// A kernel that only reads a cache in this pattern takes 115 to 126 us for the latter: value
// rows of pages of 1560 tokens begin at any multiple of 8 bytes (a copy's reads: 6.1 TB/s). For short
// lists, latency: 3.2 us a tile that a wave does after another, 9 us for a whole call of one.
template <typename T, int D, int kCols, int kParts, bool kStream, int kWaves>
__global__ __launch_bounds__(64 * kWaves, kCols == 1 && kParts == 1 && kWaves == 4 && !kStream ? 3 : 1)
void few_rows_kernel(Cache8AttnParams p) {
  constexpr int C = D / 64;   // 64-dim groups of a key row
  constexpr int M = D / 16;   // 16-dim blocks of the output
  constexpr int kRows = 16 * kCols;
  // Parts of a weight. One bf16 part rounds it by up to 2^-8, what the result's own rounding
  // adds too; two leave 2^-16. Items of 16 rows wait for memory and take two (1 to 3% of
  // their time); with more rows the second part would cost 7 to 10%. fp32 takes three.
  constexpr int kWParts = kParts == 3 ? 3 : (kCols == 1 ? 2 : 1);
  constexpr int OS = D + 4;   // floats per row of the join buffer
  __shared__ __attribute__((aligned(16))) float osm[kWaves * 16 * OS];
  __shared__ float msm[kWaves][kRows], lsm[kWaves][kRows];
  const int tid = threadIdx.x, lane = tid & 63, c16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Workgroup i runs on XCD i % 8. Pieces of one sequence and head come n_items apart, and
  // sequences begin one apart, so that no XCD gets only last pieces, which short
  // sequences lack (32 sequences of 1 to 16384 tokens, 8 pieces each: 129 us, pieces together 164).
  const int n_items = p.Hk * p.n_rt, b = blockIdx.y;
  const int x0 = __builtin_amdgcn_readfirstlane((int)((blockIdx.x + blockIdx.y) % gridDim.x));
  // (a quotient comes from the vector unit, and its uses would stay there)
  const int split = __builtin_amdgcn_readfirstlane(x0 / n_items), item = x0 - split * n_items;
  const int rt = __builtin_amdgcn_readfirstlane(item / p.Hk), h = item - rt * p.Hk;
  const Cache8Walk w = cache8_walk(p, b, h, rt * kRows, kRows, lane);
  if (w.rows <= 0) return;
  const int t_lo = split * p.split_tiles, t_hi = min(t_lo + p.split_tiles, w.n_tiles);
  if (split > 0 && t_lo >= w.n_tiles) return;
  const bool whole = w.n_tiles <= p.split_tiles;

  u32x4 qf[kCols][C][2][kParts];
  int lim[kCols];  // tokens that the column's query sees
#pragma unroll
  for (int n = 0; n < kCols; ++n) {
    const int r = rt * kRows + 16 * n + c16, i = min(r / p.G, w.q_len - 1);
    lim[n] = cache8_limit(p, w, i);
    const T* q = static_cast<const T*>(p.q) + (((size_t)b * p.n_q + i) * p.H + h * p.G + r % p.G) * D;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int u = 0; u < 2; ++u) split_row<T, kParts>(q + 64 * c + 16 * g + 8 * u, qf[n][c][u]);
  }
  const int lim_first = cache8_limit(p, w, __builtin_amdgcn_readfirstlane(rt * kRows / p.G));  // the least of them

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

  const int32_t* selrow = p.sel + ((size_t)b * p.Hk + h) * p.k_max;
  const int32_t* ptrow = p.page_table + (size_t)b * p.max_pages;
  // logical page of list position li, and its slot
  auto page_of = [&](int li) {
    return li < w.n_sel ? ld_const(selrow + li) : p.cur_first + min(li - w.n_sel, p.n_cur - 1);
  };
  auto slot_of = [&](int lp) { return clampi(ld_const(ptrow + lp), 0, p.num_slots - 1); };

  u32x4 kc[4][C], vc[M];  // codes of a tile's keys and values
  float ksc[2], vsc[2];   // their scales (granules of 8 keys: two a lane)
  int tok[2];             // logical token of the lane's keys 0..7 and 8..15; none
                          // (INT_MAX) where they are no token of a listed page
  bool masked;            // whether some query does not see all of the tile

  const int rho = 4 * (c16 >> 2);  // key row of the lane in score block i: 4 rho + 4 i + c16 % 4
  // The tile's first page (list position) and tile, or granule of the stream, within it. A
  // wave's next tile is kWaves on.
  const int per_page = kStream ? p.gpp : p.tpp, on = kStream ? 8 * kWaves : kWaves;
  int li = __builtin_amdgcn_readfirstlane((t_lo + wave) * (kStream ? 8 : 1) / per_page);
  int kt = (t_lo + wave) * (kStream ? 8 : 1) - li * per_page, li_next = 0, kt_next = 0;
  const int on_pages = __builtin_amdgcn_readfirstlane(on / per_page), on_rest = on - on_pages * per_page;
  // The tile's page, and that of the wave's next tile: looked up a tile ahead. Stream: the
  // slots of the lane's two key and two value granules, and the values' first tokens.
  int lp = 0, slot = 0, lp_next = 0, slot_next = 0;
  int ks[2], vs[2], vt[2], ks_next[2], vs_next[2], vt_next[2];
  auto look_up = [&](int l0, int at, int (&k)[2], int (&v)[2], int (&first)[2]) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {  // keys 4 rho + 8 u + 0..7: score blocks 2 u and 2 u + 1
      const Cache8Granule a = cache8_granule(p, w, l0, at, (rho >> 1) + u), c = cache8_granule(p, w, l0, at, 2 * g + u);
      k[u] = slot_v(p, ptrow, page_v(p, w, selrow, a.li));
      const int page = page_v(p, w, selrow, c.li);
      v[u] = slot_v(p, ptrow, page);
      first[u] = c.ok ? page * p.P + c.off : INT_MAX - 8;
    }
  };
  auto look_ahead = [&](int t) {
    kt_next = kt + on_rest;
    li_next = li + on_pages;
    if (kt_next >= per_page) {
      kt_next -= per_page;
      ++li_next;
    }
    if (t + kWaves < t_hi) {
      if constexpr (kStream) {
        look_up(li_next, kt_next, ks_next, vs_next, vt_next);
      } else {
        lp_next = page_of(li_next);
        slot_next = slot_of(lp_next);
      }
    }
  };
  auto load_keys = [&]() {
    if constexpr (!kStream) {
      const size_t head = (size_t)slot * p.Hk + h;
      const int w0 = min(kt * 64, p.P - 64);
      const uint8_t* kb = p.k + (head * p.P + w0 + 4 * rho + (c16 & 3)) * D + 16 * g;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < C; ++c) kc[i][c] = *reinterpret_cast<const u32x4*>(kb + 4 * i * D + 64 * c);
      ksc[0] = ksc[1] = scale_of(p.k_exp[head * p.nb + kt]);
    } else {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const Cache8Granule a = cache8_granule(p, w, li, kt, (rho >> 1) + u);
        const size_t head = (size_t)ks[u] * p.Hk + h;
        ksc[u] = scale_of(p.k_exp[head]);
        const uint8_t* kb = p.k + (head * p.P + a.off + (c16 & 3)) * D + 16 * g;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int c = 0; c < C; ++c)
            kc[2 * u + i][c] = *reinterpret_cast<const u32x4*>(kb + 4 * i * D + 64 * c);
      }
    }
  };
  auto load_values = [&]() {
    if constexpr (!kStream) {
      const size_t head = (size_t)slot * p.Hk + h;
      const int w0 = min(kt * 64, p.P - 64);
      const uint8_t* vb = p.v + (head * D + c16) * p.P + w0 + 16 * g;
#pragma unroll
      for (int m = 0; m < M; ++m) {
        const u32x4a8 x = *reinterpret_cast<const u32x4a8*>(vb + (size_t)(16 * m) * p.P);
        vc[m] = u32x4{x[0], x[1], x[2], x[3]};
      }
      vsc[0] = vsc[1] = scale_of(p.v_exp[head * p.nb + kt]);
    } else {
#pragma unroll
      for (int u = 0; u < 2; ++u)
        vsc[u] = scale_of(p.v_exp[(size_t)vs[u] * p.Hk + h]);  // (a page below 64 tokens is one block)
      if (p.P % 16 == 0) {  // both granules are of one page
        const uint8_t* vb = p.v + (((size_t)vs[0] * p.Hk + h) * D + c16) * p.P + cache8_granule(p, w, li, kt, 2 * g).off;
#pragma unroll
        for (int m = 0; m < M; ++m) {
          const u32x4a8 x = *reinterpret_cast<const u32x4a8*>(vb + (size_t)(16 * m) * p.P);
          vc[m] = u32x4{x[0], x[1], x[2], x[3]};
        }
      } else {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const Cache8Granule a = cache8_granule(p, w, li, kt, 2 * g + u);
          const uint8_t* vb = p.v + (((size_t)vs[u] * p.Hk + h) * D + c16) * p.P + a.off;
#pragma unroll
          for (int m = 0; m < M; ++m) {
            const u32x2a8 x = *reinterpret_cast<const u32x2a8*>(vb + (size_t)(16 * m) * p.P);
            vc[m][2 * u] = x[0];
            vc[m][2 * u + 1] = x[1];
          }
        }
      }
    }
  };
  // what the mask of the tile needs, once its place is known
  auto place = [&]() {
    if constexpr (!kStream) {
      const int w0 = min(kt * 64, p.P - 64), first = lp * p.P + w0 + 16 * g;
      // a tile that the page's end shifts back repeats keys of the one before
      tok[0] = w0 + 16 * g >= kt * 64 ? first : INT_MAX - 8;
      tok[1] = w0 + 16 * g + 8 >= kt * 64 ? first + 8 : INT_MAX - 8;
      masked = kt * 64 > p.P - 64 || lp * p.P + kt * 64 + 64 > lim_first;
    } else {
      tok[0] = vt[0];
      tok[1] = vt[1];
      masked = __any(max(vt[0], vt[1]) + 8 > lim_first);
    }
  };

  if (t_lo + wave < t_hi) {
    if constexpr (kStream) {
      look_up(li, kt, ks, vs, vt);
    } else {
      lp = page_of(li);
      slot = slot_of(lp);
    }
    load_keys();
    load_values();
  }
  for (int t = t_lo + wave; t < t_hi; t += kWaves) {
    look_ahead(t);
    place();
    const bool more = t + kWaves < t_hi;
    f32x4 s[kCols][4];
#pragma unroll
    for (int n = 0; n < kCols; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[n][i] = f32x4{0};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const u32x4 a = codes_to_bf16(kc[i][c][2 * u], kc[i][c][2 * u + 1], ksc[i >> 1]);
#pragma unroll
          for (int n = 0; n < kCols; ++n)
#pragma unroll
            for (int k = 0; k < kParts; ++k) s[n][i] = mfma16(a, qf[n][c][u][k], s[n][i]);
        }
    // the next tile's keys take the registers of these
    if constexpr (kStream) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        ks[u] = ks_next[u];
        vs[u] = vs_next[u];
        vt[u] = vt_next[u];
      }
    }
    lp = lp_next;
    slot = slot_next;
    li = li_next;
    kt = kt_next;
    if (more) load_keys();
    if (masked) {
#pragma unroll
      for (int n = 0; n < kCols; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (tok[i >> 1] >= lim[n] - (4 * (i & 1) + r)) s[n][i][r] = -INFINITY;
      // Codes past the last token any row sees may be anything; a weight of 0 would
      // not take a NaN out.
#pragma unroll
      for (int m = 0; m < M; ++m) {
        const int n0 = clampi(w.lim - min(tok[0], w.lim), 0, 8), n1 = clampi(w.lim - min(tok[1], w.lim), 0, 8);
        const u32x4 lo = keep_codes(vc[m], n0), hi = keep_codes(u32x4{0, 0, vc[m][2], vc[m][3]}, 8 + n1);
        vc[m] = u32x4{lo[0], lo[1], hi[2], hi[3]};
      }
    }
    u32x4 pk[kCols][2][kWParts];
#pragma unroll
    for (int n = 0; n < kCols; ++n) {
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[n][i][r]);
      // The reference maximum moves only when a score exceeds it by more than 8 in
      // exp2 units: exponentials stay below 256, and the division by the
      // sum is exact for any reference.
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
      for (int u = 0; u < 2; ++u) {
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          // (fp32: subtracted before it is scaled, so that large scores lose nothing)
          const float x = s[n][2 * u + (j >> 2)][j & 3];
          e[j] = __builtin_amdgcn_exp2f(kParts == 1 ? fmaf(x, c2, -mc) : (x - m_run[n]) * c2);
        }
        sum += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
#pragma unroll
        for (int k = 0; k < kWParts; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t x = pack_bf16(e[2 * i], e[2 * i + 1]);
            pk[n][u][k][i] = x;
            if (k + 1 < kWParts) {
              e[2 * i] -= bf16_lo(x);
              e[2 * i + 1] -= bf16_hi(x);
            }
          }
      }
      l_run[n] += sum;
    }
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const u32x4 a = codes_to_bf16(vc[m][2 * u], vc[m][2 * u + 1], vsc[u]);
#pragma unroll
        for (int n = 0; n < kCols; ++n)
#pragma unroll
          for (int k = 0; k < kWParts; ++k) acc[n][m] = mfma16(a, pk[n][u][k], acc[n][m]);
      }
    if (more) load_values();
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
  constexpr int kShare = 4 * kWaves;  // threads a row
  constexpr int N = D / kShare;       // dims each
  const int col = tid / kShare, d0 = tid % kShare * N;
#pragma unroll
  for (int n = 0; n < kCols; ++n) {
    if (n > 0) __syncthreads();
#pragma unroll
    for (int m = 0; m < M; ++m)
      *reinterpret_cast<f32x4*>(osm + (wave * 16 + c16) * OS + 16 * m + 4 * g) = acc[n][m];
    __syncthreads();
    const int row = 16 * n + col, r = rt * kRows + row, i = r / p.G;
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
      cache8_store<T, N>(p, b, i, h * p.G + r % p.G, d0, o, m_all, l, d0 == 0);
    } else {
      const size_t part = (((size_t)b * p.Hk + h) * p.n_split + split) * p.part_rows + r;
#pragma unroll
      for (int e = 0; e < N; ++e) p.part_o[part * D + d0 + e] = o[e];
      if (d0 == 0) reinterpret_cast<f32x2*>(p.part_ml)[part] = f32x2{m_all, l};
    }
  }
}

// Many query rows: 256 rows of one key head with d = 128 (eight waves of 32, a workgroup a CU), 128
// with d = 64 (four waves, three workgroups), against a range of its tokens. Each 64-key tile is
// turned into bf16 once, on its way from the registers that its codes arrived in
// to LDS, and read from there by all waves.
//
// Products are transposed as in the page walk of the bf16 pool (S^T = K Q^T, O^T +=
// V^T P^T, 32x32x16), with key rows in an order that makes a lane's scores the
// weights' operand. A step does the softmax and the value product of half a tile and the scores
// of the next half, matrix instructions between the exponentials.
// A weight is one bf16 part, rounded by up to 2^-8 of it, as in that walk (their sum is of the fp32 ones):
// the result is off by 1.9e-3 of its norm, its own rounding alone by 1.7e-3. A second part would be half
// as many matrix instructions again.
// Bound: the matrix and the vector pipe one after the other. 4680 queries over 10920 tokens, 12 heads
// (314 GFLOP): 334 to 340 us, 924 to 940 TFLOP/s, once 100 to 150 launches in a row have brought the clock
// from 1.8 to 2.3 GHz (the first ten 425 to 450 us, one every 20 ms 420 to 440). Of the cycles of a CU that
// has a workgroup the matrix pipe is busy in 44%, and vector instructions (exponentials, their packing, the
// maximum; 16 codes of each operand a thread and tile) issue in 51%, matrix instructions' own issue among
// them; the two hardly overlap, neither within a wave nor between the two of a SIMD. A large library product
// goes from 1140 to 1430 TFLOP/s over the same launches (275 to 220 us). Waves of 64 rows need more
// registers than a wave has (spills); 512 rows a workgroup was no faster, and d = 64 with 256 rows slower
// (55.9 us and 49.5 for causal prompts of up to 1001 tokens; 42 now).
template <int D>
struct ManyLayout {
  static constexpr int kRowK = 2 * D, kTileK = 64 * kRowK;  // bytes
  static constexpr int kRowV = 128, kTileV = D * kRowV;
  static constexpr int kVBase = 3 * kTileK;  // three key tiles, two value tiles
  static constexpr int kBytes = kVBase + 2 * kTileV;
  // 16-byte chunks of a row, permuted so that rows read together fall on their own banks
  static __device__ __forceinline__ int swz_k(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
  static __device__ __forceinline__ int swz_v(int row) { return (row >> 1) & 7; }
};

constexpr int many_rows(int d) { return d == 128 ? 256 : 128; }  // query rows of a many-rows item

template <int D, bool kSmallP>
__global__ __launch_bounds__(4 * D, D == 128 ? 1 : (kSmallP ? 2 : 3)) void many_rows_kernel(Cache8AttnParams p) {
  using L = ManyLayout<D>;
  constexpr int KK = D / 16, NM = D / 32;
  constexpr int kRows = many_rows(D);  // (32 a wave; 4 D threads: 16 codes of a tile's keys each, 16 of its values)
  __shared__ __attribute__((aligned(1024))) uint8_t smem[L::kBytes];
  __shared__ int2 first_sm[kSmallP ? 8 : 1][4];  // first tokens of the granules of eight tiles
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // workgroup i runs on XCD i % 8: an XCD takes an eighth of the items in a row, which share
  // their pages in its L2, first pieces first (a causal item's last pieces may be empty: the
  // workgroups of a CU, 32 apart, should not all be first pieces)
  const int n_wg = gridDim.x, x8 = blockIdx.x & 7;
  const int id = x8 * (n_wg >> 3) + min(x8, n_wg & 7) + (blockIdx.x >> 3);
  const int n_items = p.Hk * p.n_rt, share = (n_items + 7) >> 3;
  // (a quotient comes from the vector unit, and its uses would stay there)
  const int group = __builtin_amdgcn_readfirstlane(id / (share * p.n_split)), in = id - group * share * p.n_split;
  const int members = min(share, n_items - group * share);
  const int split = __builtin_amdgcn_readfirstlane(in / members), item = group * share + in - split * members;
  const int b = blockIdx.y;
  const int h = __builtin_amdgcn_readfirstlane(item / p.n_rt);
  const int rt = p.n_rt - 1 - (item - h * p.n_rt);  // (causal: the longest first)
  const Cache8Walk w = cache8_walk(p, b, h, rt * kRows, kRows, lane);
  if (w.rows <= 0) return;
  const int t_lo = split * p.split_tiles, t_hi = min(t_lo + p.split_tiles, w.n_tiles);
  if (split > 0 && t_lo >= w.n_tiles) return;
  const bool whole = w.n_tiles <= p.split_tiles;
  const int n = t_hi - t_lo;

  // queries
  u32x4 qf[KK];
  int lim;
  const int row0 = rt * kRows + wave * 32;
  {
    const int r = row0 + l32, i = min(r / p.G, w.q_len - 1);
    lim = cache8_limit(p, w, i);
    const uint16_t* q =
        static_cast<const uint16_t*>(p.q) + (((size_t)b * p.n_q + i) * p.H + h * p.G + r % p.G) * D + 8 * half;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) qf[kk] = ld_global16(q + 16 * kk);
  }
  const int lim_first = cache8_limit(p, w, min(__builtin_amdgcn_readfirstlane(row0 / p.G), w.q_len - 1));
  const bool active = row0 < rt * kRows + w.rows;

  // The listed pages are one stream of tokens, cut into tiles of 64; a tile lies in one page or
  // in two (pages hold 64 tokens or more). off: the next tile's first token within its
  // page. Slots are looked up with vector loads, a page ahead (logical pages: two), so that
  // they never wait and leave the LDS counter alone.
  const int32_t* selrow = p.sel + ((size_t)b * p.Hk + h) * p.k_max;
  const int32_t* ptrow = p.page_table + (size_t)b * p.max_pages;
  int zero = 0;
  asm volatile("" : "+v"(zero));  // (keeps the lookups vector loads)
  auto page_at = [&](int li) __attribute__((always_inline)) {
    if (li >= w.n_list) return -1 + zero;  // past the end
    return li < w.n_sel ? selrow[li + zero] : p.cur_first + li - w.n_sel + zero;
  };
  auto slot_at = [&](int lp) __attribute__((always_inline)) {
    return clampi(ptrow[clampi(lp, 0, p.max_pages - 1)], 0, p.num_slots - 1);
  };
  int kbuf = 0;  // key buffer of tile t
  int li = __builtin_amdgcn_readfirstlane((int)((int64_t)t_lo * 64 / p.P));
  int off = (int)((int64_t)t_lo * 64 - (int64_t)li * p.P);
  int lp_cur = 0, lp_nxt = 0, lp_nx2 = 0, slot_cur = 0, slot_nxt = 0;
  if constexpr (!kSmallP) {
    lp_cur = page_at(li), lp_nxt = page_at(li + 1), lp_nx2 = page_at(li + 2);
    slot_cur = slot_at(lp_cur), slot_nxt = slot_at(lp_nxt);
  }

  // What a tile is read and masked by: its first page's slot, the one after, its first token within
  // the first; and the logical tokens: key j is token ta + j below cut, tb + j from there on.
  // Small pages: off is in granules, ta and tb say whether the wave's first query, or the item's last, does not
  // see all of it, and cut is its place in first_sm.
  struct Tile {
    int slot_a, slot_b, off, ta, tb, cut;
  };
  // the tiles t, t + 1, .. t + 3, once load_k has moved on
  Tile ring[4];
  u32x4 kc, vc;  // the codes of the next tiles, 16 a thread
  uint32_t ke = 0, ve0 = 0, ve1 = 0;
  const int krow_ld = tid / (D / 16), vtok_ld = 16 * (tid & 3);
  const uint32_t vplace = (uint32_t)(tid >> 2) * (uint32_t)p.P + vtok_ld;
  // the page's slot and token of the tile's token x
  auto place = [&](const Tile& t, int x, int& at) __attribute__((always_inline)) {
    const bool second = x >= t.cut;
    at = second ? x - t.cut : t.off + x;
    return (size_t)(second ? t.slot_b : t.slot_a) * p.Hk + h;
  };
  // Small pages: a thread looks up the pages of its key row and of its two runs of values, slots
  // a tile ahead and pages two.
  int pages[3], slots[3], v_slots[2], next_at = 0, next_first = 0, next_lim = 0, staged = 0;
  int at = off >> 3;  // of the tile whose pages are looked up next
  const int on_pages = kSmallP ? __builtin_amdgcn_readfirstlane(8 / p.gpp) : 0, on_rest = 8 - on_pages * p.gpp;
  auto within = [&](int x, int& pg) __attribute__((always_inline)) {  // token of a granule x in its page, pg on
    pg = (x * p.gmul) >> 16;
    return 8 * (x - pg * p.gpp);
  };
  const int granules[3] = {krow_ld >> 3, 2 * (tid & 3), 2 * (tid & 3) + 1};
  auto stage_pages = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      int pg;
      within(at + granules[i], pg);
      pages[i] = page_at(li + pg);
    }
  };
  auto stage = [&]() __attribute__((always_inline)) {
    int first[2];
    next_at = at;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      int pg;
      const int x = within(at + granules[i], pg);
      slots[i] = slot_at(pages[i]);
      if (i > 0) first[i - 1] = pages[i] < 0 ? INT_MAX - 8 : pages[i] * p.P + x;
    }
    if (tid < 4) first_sm[staged & 7][tid] = int2{first[0], first[1]};
    const int end = max(first[0], first[1]) + 8;
    next_first = __any(end > lim_first);
    next_lim = __any(end > w.lim);
    ++staged;
    at += on_rest;
    li += on_pages;
    if (at >= p.gpp) {
      at -= p.gpp;
      ++li;
    }
    stage_pages();
  };
  auto load_k = [&]() __attribute__((always_inline)) {  // the next tile's keys; the stream moves on
    ring[0] = ring[1];
    ring[1] = ring[2];
    ring[2] = ring[3];
    Tile& t = ring[3];
    if constexpr (kSmallP) {
      t.off = next_at;
      t.ta = next_first;
      t.tb = next_lim;
      t.cut = (staged - 1) & 7;
      int pg;
      const int x = within(next_at + granules[0], pg);
      const size_t head = (size_t)slots[0] * p.Hk + h;
      kc = ld_global16(p.k + (head * p.P + x + (krow_ld & 7)) * D + 16 * (tid % (D / 16)));
      ke = p.k_exp[head];
      v_slots[0] = slots[1];
      v_slots[1] = slots[2];
      stage();
      return;
    }
    const int lp = __builtin_amdgcn_readfirstlane(lp_cur), lp2 = __builtin_amdgcn_readfirstlane(lp_nxt);
    t.slot_a = __builtin_amdgcn_readfirstlane(slot_cur);
    t.slot_b = __builtin_amdgcn_readfirstlane(slot_nxt);
    t.off = off;
    t.cut = p.P - off;
    t.ta = lp >= 0 ? lp * p.P + off : INT_MAX - 128;
    t.tb = lp2 >= 0 ? lp2 * p.P - t.cut : INT_MAX - 128;
    if (t.cut >= 64) {  // one page: its place is scalar
      const size_t head = (size_t)t.slot_a * p.Hk + h;
      kc = ld_global16(p.k + (head * p.P + t.off) * D + 16 * tid);
      ke = p.k_exp[head * p.nb + ((uint32_t)(t.off + krow_ld) >> 6)];
    } else {
      int at;
      const size_t head = place(t, krow_ld, at);
      kc = ld_global16(p.k + (head * p.P + at) * D + 16 * (tid % (D / 16)));
      ke = p.k_exp[head * p.nb + (at >> 6)];
    }
    off += 64;
    if (off >= p.P) {
      off -= p.P;
      ++li;
      lp_cur = lp_nxt;
      slot_cur = slot_nxt;
      slot_nxt = slot_at(lp_nx2);
      lp_nxt = lp_nx2;
      lp_nx2 = page_at(li + 2);
    }
  };
  auto load_v = [&](const Tile& t) __attribute__((always_inline)) {
    if constexpr (kSmallP) {
      int pg;
      const int x0 = within(t.off + granules[1], pg), x1 = within(t.off + granules[2], pg);
      const size_t h0 = (size_t)v_slots[0] * p.Hk + h, h1 = (size_t)v_slots[1] * p.Hk + h;
      const u32x2a8 x = *reinterpret_cast<const u32x2a8*>(p.v + (h0 * D + (tid >> 2)) * p.P + x0);
      const u32x2a8 y = *reinterpret_cast<const u32x2a8*>(p.v + (h1 * D + (tid >> 2)) * p.P + x1);
      vc = u32x4{x[0], x[1], y[0], y[1]};
      ve0 = p.v_exp[h0];
      ve1 = p.v_exp[h1];
      return;
    }
    if (t.cut >= 64) {
      const size_t head = (size_t)t.slot_a * p.Hk + h;
      const u32x4a8 x = *reinterpret_cast<const u32x4a8*>(p.v + head * D * p.P + t.off + vplace);
      vc = u32x4{x[0], x[1], x[2], x[3]};
      ve0 = p.v_exp[head * p.nb + ((uint32_t)(t.off + vtok_ld) >> 6)];
      ve1 = p.v_exp[head * p.nb + ((uint32_t)(t.off + vtok_ld + 8) >> 6)];
      return;
    }
    int at0, at1;
    const size_t h0 = place(t, vtok_ld, at0), h1 = place(t, vtok_ld + 8, at1);
    const u32x2a8 x = *reinterpret_cast<const u32x2a8*>(p.v + (h0 * D + (tid >> 2)) * p.P + at0);
    const u32x2a8 y = *reinterpret_cast<const u32x2a8*>(p.v + (h1 * D + (tid >> 2)) * p.P + at1);
    vc = u32x4{x[0], x[1], y[0], y[1]};
    ve0 = p.v_exp[h0 * p.nb + (at0 >> 6)];
    ve1 = p.v_exp[h1 * p.nb + (at1 >> 6)];
  };
  auto put_k = [&](int buf) __attribute__((always_inline)) {
    const float s = scale_of(ke);
    const int row = krow_ld, c0 = 2 * (tid % (D / 16));
    uint8_t* dst = smem + buf * L::kTileK + row * L::kRowK;
    *reinterpret_cast<u32x4*>(dst + ((c0 ^ L::swz_k(row)) << 4)) = codes_to_bf16(kc[0], kc[1], s);
    *reinterpret_cast<u32x4*>(dst + (((c0 + 1) ^ L::swz_k(row)) << 4)) = codes_to_bf16(kc[2], kc[3], s);
  };
  // whether some query of limit `most` does not see some token of a tile
  auto beyond = [&](const Tile& t, int most) __attribute__((always_inline)) {
    if constexpr (kSmallP) return (most == w.lim ? t.tb : t.ta) != 0;
    return t.ta + min(t.cut, 64) > most || (t.cut < 64 && t.tb + 64 > most);
  };
  auto put_v = [&](int buf, const Tile& t) __attribute__((always_inline)) {
    if (beyond(t, w.lim)) {
      // codes past the last token any row sees may be anything
      int t0 = (vtok_ld < t.cut ? t.ta : t.tb) + vtok_ld, t1 = (vtok_ld + 8 < t.cut ? t.ta : t.tb) + vtok_ld + 8;
      if constexpr (kSmallP) {
        t0 = first_sm[t.cut][tid & 3].x;
        t1 = first_sm[t.cut][tid & 3].y;
      }
      const u32x4 lo = keep_codes(vc, clampi(w.lim - min(t0, w.lim), 0, 8));
      const u32x4 hi = keep_codes(u32x4{0, 0, vc[2], vc[3]}, 8 + clampi(w.lim - min(t1, w.lim), 0, 8));
      vc = u32x4{lo[0], lo[1], hi[2], hi[3]};
    }
    const int row = tid >> 2, c0 = 2 * (tid & 3);
    uint8_t* dst = smem + L::kVBase + buf * L::kTileV + row * L::kRowV;
    *reinterpret_cast<u32x4*>(dst + ((c0 ^ L::swz_v(row)) << 4)) = codes_to_bf16(vc[0], vc[1], scale_of(ve0));
    *reinterpret_cast<u32x4*>(dst + (((c0 + 1) ^ L::swz_v(row)) << 4)) = codes_to_bf16(vc[2], vc[3], scale_of(ve1));
  };

  f32x16 acc[NM], sa, sb;
  const float c2 = p.scale_log2;
  float m_run = softmax_floor(c2), l_run = 0.f;
#pragma unroll
  for (int m = 0; m < NM; ++m) acc[m] = f32x16{0};
  const int krow = (l32 & ~12) | ((l32 & 4) << 1) | ((l32 & 8) >> 1);  // bits 2 and 3 swapped
  // Operands: slice j of key half kh in key buffer buf; dim block m of 16-key group ks. A
  // lane's chunks of a row are its first one's place with bits 5 to 7 turned.
  const uint32_t kfirst = krow * L::kRowK + ((half ^ L::swz_k(krow)) << 4);
  const uint32_t vfirst = l32 * L::kRowV + ((half ^ L::swz_v(l32)) << 4);
  auto kop = [&](uint32_t at, int kh, int j) __attribute__((always_inline)) {
    return ld_lds16(smem + (at ^ (j << 5)) + kh * 32 * L::kRowK);
  };
  auto vop = [&](uint32_t at, int ks, int m) __attribute__((always_inline)) {
    return ld_lds16(smem + (at ^ (ks << 5)) + m * 32 * L::kRowV);
  };
  // Two weights of 16-key group g (score registers 8 g + 2 i, + 1), packed.
  auto weigh = [&](const f32x16& s, float mc, int g, int i) __attribute__((always_inline)) {
    const float x = __builtin_amdgcn_exp2f(fmaf(s[8 * g + 2 * i], c2, -mc));
    const float y = __builtin_amdgcn_exp2f(fmaf(s[8 * g + 2 * i + 1], c2, -mc));
    l_run += x + y;
    return pack_bf16(x, y);
  };
  // keys of half kh that a query does not see (the eight keys of a group are of one page)
  auto mask = [&](const Tile& t, int kh, f32x16& s) __attribute__((always_inline)) {
    int mine = 32 * kh + 8 * half;
    asm volatile("" : "+v"(mine));  // (nothing of this is kept through the walk)
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int key = mine + 16 * g;
      int sees = lim - (key + (key < t.cut ? t.ta : t.tb));  // of the group's keys
      if constexpr (kSmallP) sees = lim - (half ? first_sm[t.cut][2 * kh + g].y : first_sm[t.cut][2 * kh + g].x);
#pragma unroll
      for (int x = 0; x < 8; ++x)
        if (x >= sees) s[8 * g + x] = -INFINITY;
    }
  };
  // The largest of a half's scores, and the reference that follows it as in the few-rows kernel.
  auto largest = [&](const f32x16& s) __attribute__((always_inline)) {
    float mx = s[0];
#pragma unroll
    for (int x = 1; x < 16; ++x) mx = fmaxf(mx, s[x]);
    return mx;
  };
  auto raise = [&](float mx) __attribute__((always_inline)) {
    if (__any(mx * c2 > m_run * c2 + 8.f)) {
      const float top = fmaxf(mx, __shfl_xor(mx, 32));
      const float m_new = top * c2 > m_run * c2 + 8.f ? top : m_run;
      const float alpha = __builtin_amdgcn_exp2f((m_run - m_new) * c2);
      l_run *= alpha;
#pragma unroll
      for (int m = 0; m < NM; ++m) acc[m] *= alpha;
      m_run = m_new;
    }
  };
  // Half a step: the softmax and value product of key half kh (scores s, value buffer vb), and
  // the scores sn of the half after it: half nh of tile nt, in key buffer kb. An operand is
  // read four matrix instructions before its use; between them go the weights (those of the first 16 keys
  // spread so that their products can begin, then those of the second), the conversion of
  // the tiles to come, and the maximum. The order is the source's: left to itself the
  // compiler reads operands right before their use.
  auto half_step = [&](int vb, int kh, const f32x16& s, int kb, int nh, const Tile& nt, f32x16& sn,
                       auto&& tail) __attribute__((always_inline)) {
    constexpr int NP = KK + 2 * NM;            // matrix instructions
    constexpr int kFirst = KK / 2;             // of them, beside the weights of the first 16 keys
    constexpr int kSecond = KK + NM - kFirst;  // and of the second
    float mc = m_run * c2, mx = -INFINITY;
    u32x4 pk[2], f[4];
    sn = f32x16{0};
    uint32_t k_at = kfirst + kb * L::kTileK, v_at = L::kVBase + vfirst + vb * L::kTileV;
    asm volatile("" : "+v"(k_at), "+v"(v_at));  // (a place each, not one for every operand)
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = kop(k_at, nh, i);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      // (what an instruction computes from is opaque before it, and what it leaves is used in it)
      __builtin_amdgcn_sched_barrier(0);
      u32x4 a = f[i & 3];
      asm volatile("" : "+v"(a));
      asm volatile("" : "+v"(mc));
      const int n = i + 4;
      if (i < KK) sn = mfma32(a, qf[i], sn);
      else acc[(i - KK) % NM] = mfma32(a, pk[(i - KK) / NM], acc[(i - KK) % NM]);
      if (n < KK) f[i & 3] = kop(k_at, nh, n);
      else if (n < NP) f[i & 3] = vop(v_at, 2 * kh + (n - KK) / NM, (n - KK) % NM);
#pragma unroll
      for (int x = 0; x < 4; ++x) {  // packed weights: four of each 16 keys
        uint32_t e;
        if (i < kFirst && x * kFirst / 4 == i) {
          e = weigh(s, mc, 0, x);
          asm volatile("" : "+v"(e), "+v"(l_run));
          pk[0][x] = e;
        }
        if (i >= kFirst && i < kFirst + kSecond && x * kSecond / 4 == i - kFirst) {
          e = weigh(s, mc, 1, x);
          asm volatile("" : "+v"(e), "+v"(l_run));
          pk[1][x] = e;
        }
      }
      if (i >= KK + NM) {  // (the scores were complete NM instructions ago)
#pragma unroll
        for (int x = (i - KK - NM) * 16 / NM; x < (i - KK - NM + 1) * 16 / NM; ++x) mx = fmaxf(mx, sn[x]);
        asm volatile("" : "+v"(mx));
      }
      if (i == KK) tail();
    }
    __builtin_amdgcn_sched_barrier(0);
    if (__builtin_expect(beyond(nt, lim_first), 0)) {
      mask(nt, nh, sn);
      mx = largest(sn);
    }
    raise(mx);
  };
  // One step: tile t (scores of its first half in sa on entry), with the first half of tile
  // t + 1 at its end. par: t's parity, which buffers hold it.
  auto step = [&](auto parity) __attribute__((always_inline)) {
    constexpr int par = decltype(parity)::value;
    __builtin_amdgcn_sched_barrier(0);
    lds_barrier();
    __builtin_amdgcn_sched_barrier(0);
    // V(t + 1) goes over V(t - 1), K(t + 2) over K(t - 1), three key buffers on; the loads
    // after them start as soon as their registers are free
    const int k0 = kbuf, k1 = kbuf == 2 ? 0 : kbuf + 1, k2 = k1 == 2 ? 0 : k1 + 1;
    kbuf = k1;
    auto next_v = [&]() __attribute__((always_inline)) {
      put_v(1 - par, ring[2]);
      load_v(ring[3]);
    };
    auto next_k = [&]() __attribute__((always_inline)) {
      put_k(k2);
      load_k();
    };
    if (!active) {
      next_v();
      next_k();
      return;
    }
    // (tile t is ring[1] before load_k, ring[0] after it)
    half_step(par, 0, sa, k0, 1, ring[1], sb, next_v);
    const Tile ahead = ring[2];
    half_step(par, 1, sb, k1, 0, ahead, sa, next_k);
  };

  if (n > 0) {
    if constexpr (kSmallP) {
      stage_pages();
      stage();
      lds_barrier();  // (first_sm of tile 0, which every wave may read below)
    }
    // K(0), K(1) and V(0) to LDS; K(2) and V(1) on their way
    load_k();
    load_v(ring[3]);
    put_k(0);
    load_k();
    put_v(0, ring[2]);
    put_k(1);
    load_v(ring[3]);
    load_k();
    // (ring[1] is tile 0 now)
    lds_barrier();
    if (active) {
      sa = f32x16{0};
#pragma unroll
      for (int j = 0; j < KK; ++j) sa = mfma32(kop(kfirst, 0, j), qf[j], sa);
      if (beyond(ring[1], lim_first)) mask(ring[1], 0, sa);
      raise(largest(sa));
    }
    for (int t = 0; t < n; t += 2) {
      step(std::integral_constant<int, 0>{});
      if (t + 1 < n) step(std::integral_constant<int, 1>{});
    }
  }
  if (!active) return;
  const int r = row0 + l32, i = r / p.G;
  const float l = l_run + __shfl_xor(l_run, 32);
  if (i >= w.q_len) return;
  if (whole) {
    const int head = h * p.G + r % p.G;
#pragma unroll
    for (int m = 0; m < NM; ++m)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float o[4] = {acc[m][4 * g], acc[m][4 * g + 1], acc[m][4 * g + 2], acc[m][4 * g + 3]};
        cache8_store<uint16_t, 4>(p, b, i, head, 32 * m + 8 * g + 4 * half, o, m_run, l, m == 0 && g == 0 && half == 0);
      }
  } else {
    const size_t part = (((size_t)b * p.Hk + h) * p.n_split + split) * p.part_rows + r;
#pragma unroll
    for (int m = 0; m < NM; ++m)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4*>(p.part_o + part * D + 32 * m + 8 * g + 4 * half) =
            f32x4{acc[m][4 * g], acc[m][4 * g + 1], acc[m][4 * g + 2], acc[m][4 * g + 3]};
    if (half == 0) reinterpret_cast<f32x2*>(p.part_ml)[part] = f32x2{m_run, l};
  }
}

// Joins the pieces of a row whose tokens were split, in an order that does not depend on
// the launch's timing. The pieces' maxima and sums are on their way before the row's
// number of pieces is known (a piece that does not exist holds anything, and is
// not used).
// Up to 1024 rows: a workgroup of eight waves a row, each every eighth piece (1024 rows of up to 16
// pieces: 7.0 us).
template <typename T, int D>
__global__ __launch_bounds__(512) void join_row_kernel(Cache8AttnParams p) {
  constexpr int E = D / 64, kW = 8;  // dims per lane, waves
  __shared__ float osm[kW][D];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = blockIdx.x / p.Hk, h = blockIdx.x - r * p.Hk, b = blockIdx.y;
  const size_t part0 = ((size_t)b * p.Hk + h) * p.n_split * p.part_rows + r;
  const f32x2* ml = reinterpret_cast<const f32x2*>(p.part_ml);
  f32x2 x[kMaxSplit / 64];
#pragma unroll
  for (int k = 0; k < kMaxSplit / 64; ++k)
    x[k] = 64 * k < p.n_split ? ml[part0 + (size_t)min(64 * k + lane, p.n_split - 1) * p.part_rows] : f32x2{0.f, 0.f};
  const Cache8Walk w = cache8_walk(p, b, h, r / p.rows_per_item * p.rows_per_item, p.rows_per_item, lane);
  const int i = r / p.G;
  if (w.rows <= 0 || i >= w.q_len || w.n_tiles <= p.split_tiles) return;
  const int n = (w.n_tiles + p.split_tiles - 1) / p.split_tiles;
  float m_all = -FLT_MAX;
#pragma unroll
  for (int k = 0; k < kMaxSplit / 64; ++k)
    if (64 * k + lane < n) m_all = fmaxf(m_all, x[k][0]);
#pragma unroll
  for (int y = 1; y < 64; y <<= 1) m_all = fmaxf(m_all, __shfl_xor(m_all, y));
  float l = 0.f, o[E] = {};
#pragma unroll
  for (int k = 0; k < kMaxSplit / 64; ++k) {
    if (64 * k >= n) break;
    const bool in = 64 * k + lane < n;
    const float wt = in ? __builtin_amdgcn_exp2f((x[k][0] - m_all) * p.scale_log2) : 0.f;
    float sum = in ? wt * x[k][1] : 0.f;
#pragma unroll
    for (int y = 1; y < 64; y <<= 1) sum += __shfl_xor(sum, y);
    l += sum;
    // (a piece past the last one repeats that with weight 0: no branch between the loads)
    const int last = min(63, n - 64 * k - 1);
    constexpr int kAtOnce = 4;
    for (int s0 = wave; s0 <= last; s0 += kW * kAtOnce) {
      float src[kAtOnce][E];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e)
          src[j][e] = p.part_o[(part0 + (size_t)(64 * k + min(s0 + kW * j, last)) * p.part_rows) * D + E * lane + e];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const int s = s0 + kW * j;
        const float ws = s <= last ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wt), s)) : 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] += ws * src[j][e];
      }
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e) osm[wave][E * lane + e] = o[e];
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    o[e] = osm[0][E * lane + e];
#pragma unroll
    for (int y = 1; y < kW; ++y) o[e] += osm[y][E * lane + e];
  }
  cache8_store<T, E>(p, b, i, h * p.G + r % p.G, E * lane, o, m_all, l, lane == 0);
}

// Many rows: D / 4 lanes a row, four dims each, the pieces one after another.
template <typename T, int D>
__global__ __launch_bounds__(256) void join_rows_kernel(Cache8AttnParams p) {
  constexpr int kLanes = D / 4, kPerWg = 256 / kLanes;
  const int tid = threadIdx.x, lane = tid & 63;
  const int tiles = (p.part_rows + kPerWg - 1) / kPerWg;  // workgroups a key head
  const int h = blockIdx.x / tiles, b = blockIdx.y;
  const int row0 = (blockIdx.x - h * tiles) * kPerWg, r = row0 + tid / kLanes;
  const size_t part0 = ((size_t)b * p.Hk + h) * p.n_split * p.part_rows + r;
  const f32x2* ml = reinterpret_cast<const f32x2*>(p.part_ml);
  // (items are 16 rows or a multiple: a workgroup's are of one item)
  const Cache8Walk w = cache8_walk(p, b, h, row0 / p.rows_per_item * p.rows_per_item, p.rows_per_item, lane);
  const int i = r / p.G, d0 = 4 * (tid % kLanes);
  if (w.rows <= 0 || i >= w.q_len || w.n_tiles <= p.split_tiles) return;
  const int n = (w.n_tiles + p.split_tiles - 1) / p.split_tiles;
  float m = -FLT_MAX, l = 0.f, o[4] = {};
#pragma unroll 4
  for (int s = 0; s < n; ++s) {
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
  cache8_store<T, 4>(p, b, i, h * p.G + r % p.G, d0, o, m, l, d0 == 0);
}

template <typename T, int D, int kCols, int kParts>
void launch_rows(const Cache8AttnParams& p, int B, hipStream_t s) {
  const dim3 grid(p.n_split * p.Hk * p.n_rt, B);
  if (kCols == 1 && p.waves == 8) {
    if (p.stream) few_rows_kernel<T, D, 1, kParts, true, 8><<<grid, 512, 0, s>>>(p);
    else few_rows_kernel<T, D, 1, kParts, false, 8><<<grid, 512, 0, s>>>(p);
  } else {
    if (p.stream) few_rows_kernel<T, D, kCols, kParts, true, 4><<<grid, 256, 0, s>>>(p);
    else few_rows_kernel<T, D, kCols, kParts, false, 4><<<grid, 256, 0, s>>>(p);
  }
}

template <int D>
hipError_t launch_for(int dtype, int B, const Cache8AttnParams& p, hipStream_t s) {
  const int cols = p.rows_per_item / 16;
  if (dtype == HSA_DTYPE_BF16) {
    if (p.many)
      p.P < 64 ? many_rows_kernel<D, true><<<dim3(p.n_split * p.Hk * p.n_rt, B), 4 * D, 0, s>>>(p)
               : many_rows_kernel<D, false><<<dim3(p.n_split * p.Hk * p.n_rt, B), 4 * D, 0, s>>>(p);
    else if (cols == 1) launch_rows<uint16_t, D, 1, 1>(p, B, s);
    else if (cols == 2) launch_rows<uint16_t, D, 2, 1>(p, B, s);
    else if constexpr (D == 64) launch_rows<uint16_t, D, 4, 1>(p, B, s);
  } else {
    if (cols == 1) launch_rows<float, D, 1, 3>(p, B, s);
    else launch_rows<float, D, 2, 3>(p, B, s);
  }
  if (p.n_split > 1) {
    // a workgroup a row while the rows alone do not fill the chip
    if ((int64_t)p.n_q * p.H * B <= 1024) {
      const dim3 grid(p.n_q * p.H, B);
      if (dtype == HSA_DTYPE_BF16) join_row_kernel<uint16_t, D><<<grid, 512, 0, s>>>(p);
      else join_row_kernel<float, D><<<grid, 512, 0, s>>>(p);
    } else {
      const int per = 256 / (D / 4);
      const dim3 grid((p.part_rows + per - 1) / per * p.Hk, B);
      if (dtype == HSA_DTYPE_BF16) join_rows_kernel<uint16_t, D><<<grid, 256, 0, s>>>(p);
      else join_rows_kernel<float, D><<<grid, 256, 0, s>>>(p);
    }
  }
  return hipGetLastError();
}

// 64-token tiles of a list, walked by the page or, of small pages, as a stream.
int64_t cache8_tiles(int64_t list, int P) { return P < 64 ? (list * P + 63) / 64 : list * ((P + 63) / 64); }
// Calls that the many-rows kernel may take, and the work (items of 16 rows times tiles) up to which a
// call is little.
bool cache8_large(int dtype, int64_t rows) { return dtype == HSA_DTYPE_BF16 && rows > 64; }
int64_t cache8_little(bool large, int d) { return large ? (d == 64 ? 32768 : 8192) : 4096; }
bool cache8_brief(int64_t items16, int64_t tiles, int64_t rows, bool large, int d) {
  return items16 <= (large || rows <= 16 ? 4096 : 256) && items16 * tiles <= cache8_little(large, d);
}
// Rows of an item of the four-wave workgroups.
int cache8_few_rows(int dtype, int d, int64_t rows) {
  return rows <= 16 ? 16 : (rows > 32 && dtype == HSA_DTYPE_BF16 && d == 64 ? 64 : 32);
}
// Workgroups of the many-rows kernel that a call is planned for.
int64_t cache8_slots(int d, int P, bool ragged) { return d == 128 ? 256 : (ragged || P < 64 ? 512 : 768); }
// Most pieces of such a call, their ends counted (see plan_cache8).
constexpr int kManyPieces = 16;
constexpr double kManyEnds = 6.0, kManyJoin = 4.0, kManyGain = 0.97;

}  // namespace

void plan_cache8(Cache8AttnParams& p, int dtype, int B, int max_list_sel, bool ragged) {
  p.nb = (p.P + 63) / 64;
  p.tpp = p.nb;
  p.gpp = p.P / 8;
  p.gmul = 65536 / p.gpp + 1;
  const int64_t list = (int64_t)max_list_sel + p.n_cur;
  const int64_t rows = (int64_t)p.n_q * p.G;
  // Little work: eight waves a workgroup and 16 rows an item. Up to two tiles for each wave of every CU,
  // what counts is how many tiles a wave does after one another, and a second launch if they are
  // cut. The many-rows kernel starts slower still, so calls of more than 64 bf16 rows come here up to
  // four tiles a wave (d = 128: 2048 queries of 4 heads, 2 key heads, over 1024 tokens 25 us and 31;
  // twice the tokens 38 and 36) or sixteen (d = 64: 4096 over 2048 31 us and 35; three ragged
  // prompts, 2.3 times the work, 50 and 46).
  const int64_t items16 = (int64_t)B * p.Hk * ((rows + 15) / 16);
  const int64_t by_page = cache8_tiles(list, p.P);
  const bool large = cache8_large(dtype, rows);
  const bool brief = cache8_brief(items16, by_page, rows, large, p.d);
  // More than 64 rows of bf16 otherwise (8 sequences of 8192 tokens, 8 heads, d = 128: 96 rows 66 us,
  // in items of 32 rows 86; d = 64, 64 rows: 39 us, in one item of 64 rows 30). fp32 has three
  // parts of everything, and its registers hold 32 rows.
  const bool many = !brief && large;
  p.many = many;
  // Pages below 64 tokens are walked as a stream. Larger ones are not, though their last tile repeats
  // tokens: the stream looks up two pages a lane (32 sequences of up to 16384 tokens, 8 key heads:
  // pages of 72, 161 us as a stream and 143 by the page; of 200, 182 and 145; of 16, 140).
  p.stream = many || p.P < 64;
  const int64_t tiles = std::max<int64_t>(1, many ? (list * p.P + 63) / 64 : by_page);
  p.rows_per_item = many ? many_rows(p.d) : (brief ? 16 : cache8_few_rows(dtype, p.d, rows));
  p.waves = brief ? 8 : 4;
  p.n_rt = (int)((rows + p.rows_per_item - 1) / p.rows_per_item);
  p.part_rows = p.n_rt * p.rows_per_item;
  const int64_t items = (int64_t)B * p.Hk * p.n_rt;
  int64_t n = 1;
  if (many) {
    // Rounds of as many workgroups as are resident (one a CU, with d = 64 three, of small pages
    // two), each of its tiles and about six more for its start and end; pieces cost a
    // partial output written and read again (four). 8 causal sequences of 8192 tokens,
    // d = 128, 128 queries: 74 us in four pieces. Calls with kv_len, d = 64, are planned for two workgroups a
    // CU, which leaves more items whole: right for prompts (three of up to 1001 tokens, 16 query and 4 key
    // heads, of drawn, nearly equal and equal lengths 28, 34 and 35 us, for three a CU 34, 40 and 40; two of 3000
    // tokens 117 and 127), not for queries over a longer history (4096 of 4 heads over 8192 tokens 67 us and 63;
    // 4680 of 12 heads over 10920, 265 and 254) or short ones over small pages (four of 900 tokens, pages
    // of 136, 29 and 28).
    const int64_t slots = cache8_slots(p.d, p.P, ragged);
    double best = 1e300;
    for (int64_t k = 1; k <= kManyPieces && k * 4 <= std::max<int64_t>(tiles, 4); ++k) {
      const double each = (double)((tiles + k - 1) / k) + kManyEnds + (k > 1 ? kManyJoin : 0.0);
      const double t = (double)((items * k + slots - 1) / slots) * each;
      if (t < kManyGain * best) {
        best = t;
        n = k;
      }
    }
  } else if (brief) {
    // In us (12 key heads, one sequence): a tile after another 3.2, the join 3.5; 16 tiles whole
    // 12.0, cut in two 12.4; 32 whole 19, cut in four 12.2; 128 cut in 16 13.0, in 8 16.4.
    double best = 1e300;
    for (int64_t k = 1; k == 1 || (k * items16 <= 256 && 8 * (k - 1) < tiles); ++k) {
      const double t = 3.2 * (double)((tiles + 8 * k - 1) / (8 * k)) + (k > 1 ? 3.5 : 0.0);
      if (t < best) {
        best = t;
        n = k;
      }
    }
  } else {
    const int64_t most_n = std::max<int64_t>(1, std::min<int64_t>(kMaxSplit, tiles / (ragged ? 16 : 8)));
    if (ragged) {
      // Sequences of different lengths: short pieces balance (32 of 1 to 16384 tokens, 8 key
      // heads: pieces of 16 tiles 124 us, of 32 128; 8 of them 42 and 49).
      n = std::min((4096 + items - 1) / items, most_n);
    } else {
      // Equal pieces: at least two workgroups a CU (one of more than 16 rows: its registers leave no
      // room for another; 4 sequences of 8192, 32 rows: 8 pieces 25 us, 16 30), and as even a
      // number on each as can be
      // (8 sequences of 16384: 8 pieces, 512 workgroups, 57 us; 10 pieces 65, 12 61; 8 of 4096 and
      // 12 key heads: 8 pieces of 8 tiles 26, 4 of 16 29). A piece's start and end take
      // about four tiles.
      n = std::min(((p.rows_per_item > 16 ? 256 : 512) + items - 1) / items, most_n);
      double best = 1e300;
      for (int64_t k = n, stop = std::min((2048 + items - 1) / items, most_n); k <= stop; ++k) {
        const double t = (double)((items * k + 255) / 256) * ((double)((tiles + k - 1) / k) + 4.0);
        if (t < 0.99 * best) {
          best = t;
          n = k;
        }
      }
    }
  }
  int64_t c = (tiles + n - 1) / n;
  if (!many) c = (c + p.waves - 1) / p.waves * p.waves;
  p.split_tiles = (int)c;
  p.n_split = (int)((tiles + c - 1) / c);
}

int64_t cache8_most_part_rows(int dtype, int d, int P, int B, int Hk, int64_t rows, int64_t list) {
  const int64_t tiles = cache8_tiles(list, P), items16 = (int64_t)B * Hk * ((rows + 15) / 16);
  const bool large = cache8_large(dtype, rows);
  int64_t most = 0;
  auto take = [&](int64_t pieces, int64_t per_item) {
    if (pieces > 1) most = std::max(most, pieces * ((rows + per_item - 1) / per_item * per_item));
  };
  // Lists up to some length are little work: as many pieces as workgroups, of at least a tile a wave.
  if (cache8_brief(items16, cache8_tiles(1, P), rows, large, d)) {
    const int64_t longest = std::min(tiles, cache8_little(large, d) / items16);
    take(std::min(256 / items16, (longest - 1) / 8 + 1), 16);
  }
  if (cache8_brief(items16, tiles, rows, large, d)) return most;
  if (large) {
    // k pieces of T tiles (4 k or more) have to be faster than any fewer. With r the rounds of workgroups
    // and e their ends and the join: r(k) (ceil(T / k) + e) < r(j) (ceil(T / j) + e), 1 < j < k (a j that did not
    // gain enough itself leaves no less to beat), and below the gain times r(1) (T + ends). With T / k for the
    // left side and T / j + 1 for the right one, both are linear in T: a range [lo, hi] of it.
    const int64_t all = (list * P + 63) / 64, per = many_rows(d), items = (int64_t)B * Hk * ((rows + per - 1) / per);
    constexpr double e = kManyEnds + kManyJoin, kSlack = 1.0 + 1e-9;
    for (const bool ragged : {false, true}) {
      const int64_t slots = cache8_slots(d, P, ragged);
      auto rounds = [&](int64_t k) { return (double)((items * k + slots - 1) / slots); };
      for (int64_t k = kManyPieces; k > 1; --k) {
        double lo = 4.0 * (double)k, hi = (double)all;
        for (int64_t j = 1; j < k; ++j) {
          const double r = rounds(j) * kSlack * (j > 1 ? 1.0 : kManyGain);
          const double slope = rounds(k) / (double)k - r / (double)j;  // slope T <= room
          const double room = r * (j > 1 ? e + 1.0 : kManyEnds) - rounds(k) * e;
          if (slope > 0.0) hi = std::min(hi, room / slope);
          else if (slope < 0.0) lo = std::max(lo, room / slope);
          else if (room < 0.0) hi = -1.0;
        }
        if (lo > hi) continue;
        take(k, per);
        break;
      }
    }
  } else {
    const int64_t per = cache8_few_rows(dtype, d, rows), items = (int64_t)B * Hk * ((rows + per - 1) / per);
    take(std::min((4096 + items - 1) / items, std::min<int64_t>(kMaxSplit, tiles / 16)), per);  // ragged
    take(std::min((2048 + items - 1) / items, std::min<int64_t>(kMaxSplit, tiles / 8)), per);
  }
  return most;
}

hipError_t launch_cache8_attention(int dtype, int d, int B, const Cache8AttnParams& p, hipStream_t s) {
  return d == 128 ? launch_for<128>(dtype, B, p, s) : launch_for<64>(dtype, B, p, s);
}

}  // namespace hsa
