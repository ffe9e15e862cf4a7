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
#include "hsa_cache8.h"

namespace hsa {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;  // waves of a few-rows workgroup

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

// Few query rows: 16 kCols rows of one key head against a range of its tokens. Each
// of the four waves takes every fourth 64-key tile and keeps an online softmax
// of its own; the workgroup joins them at the end.
//
// Products are transposed (keys are the rows of S^T = K Q^T, dims those of O^T = V^T P^T),
// so a lane holds scores of one query and the 16 keys of its quarter. Row m of
// score block i is key 16 (m / 4) + 4 i + m % 4: a quarter of lanes then
// holds 16 consecutive keys, in the order in which the value operand, 16 consecutive codes
// of a d-major row, has them, and the weights need no exchange between lanes. Codes go
// from HBM to the registers of the wave that uses them, 16 bytes a lane; a
// score block's rows are read in 64-byte pieces, a value block's too.
// Bound: HBM (2 d bytes a token and key head).
template <typename T, int D, int kCols, int kParts, bool kSmallP>
__global__ __launch_bounds__(64 * kWaves) void few_rows_kernel(Cache8AttnParams p) {
  constexpr int C = D / 64;   // 64-dim groups of a key row
  constexpr int M = D / 16;   // 16-dim blocks of the output
  constexpr int kRows = 16 * kCols;
  constexpr int OS = D + 4;   // floats per row of the join buffer
  __shared__ __attribute__((aligned(16))) float osm[kWaves * 16 * OS];
  __shared__ float msm[kWaves][kRows], lsm[kWaves][kRows];
  const int tid = threadIdx.x, lane = tid & 63, c16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int item = blockIdx.x / p.n_split, split = blockIdx.x - item * p.n_split, b = blockIdx.y;
  const int rt = item / p.Hk, h = item - rt * p.Hk;
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
  const int lim_first = cache8_limit(p, w, rt * kRows / p.G);  // the least of them

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
  int tok[2];             // logical token of the lane's keys 0..7 and 8..15
  bool ok[2];             // whether they are tokens of a listed page

  const int rho = 4 * (c16 >> 2);  // key row of the lane in score block i: 4 rho + 4 i + c16 % 4
  int li = 0, kt = 0;              // list position and tile within its page
  if constexpr (!kSmallP) {
    li = (t_lo + wave) / p.tpp;
    kt = (t_lo + wave) - li * p.tpp;
  }
  int lp = 0, slot = 0;
  auto locate = [&](int t) {
    if constexpr (!kSmallP) {
      lp = page_of(li);
      slot = slot_of(lp);
    }
  };
  auto load_keys = [&](int t) {
    if constexpr (!kSmallP) {
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
      for (int u = 0; u < 2; ++u) {  // keys 4 rho + 8 u + 0..7: score blocks 2 u and 2 u + 1
        const int gr = (rho >> 1) + u;
        const Cache8Granule a = cache8_granule(p, w, t, gr);
        const size_t head = (size_t)slot_v(p, ptrow, page_v(p, w, selrow, a.li)) * p.Hk + h;
        ksc[u] = scale_of(p.k_exp[head * p.nb]);
        const uint8_t* kb = p.k + (head * p.P + a.off + (c16 & 3)) * D + 16 * g;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int c = 0; c < C; ++c)
            kc[2 * u + i][c] = *reinterpret_cast<const u32x4*>(kb + 4 * i * D + 64 * c);
      }
    }
  };
  auto load_values = [&](int t) {
    if constexpr (!kSmallP) {
      const size_t head = (size_t)slot * p.Hk + h;
      const int w0 = min(kt * 64, p.P - 64);
      const uint8_t* vb = p.v + (head * D + c16) * p.P + w0 + 16 * g;
#pragma unroll
      for (int m = 0; m < M; ++m) {
        const u32x4a8 x = *reinterpret_cast<const u32x4a8*>(vb + (size_t)(16 * m) * p.P);
        vc[m] = u32x4{x[0], x[1], x[2], x[3]};
      }
      vsc[0] = vsc[1] = scale_of(p.v_exp[head * p.nb + kt]);
      const int first = lp * p.P + w0 + 16 * g;
      tok[0] = first;
      tok[1] = first + 8;
      // a tile that the page's end shifts back repeats keys of the one before
      ok[0] = w0 + 16 * g >= kt * 64;
      ok[1] = w0 + 16 * g + 8 >= kt * 64;
    } else {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const Cache8Granule a = cache8_granule(p, w, t, 2 * g + u);
        const int page = page_v(p, w, selrow, a.li);
        const size_t head = (size_t)slot_v(p, ptrow, page) * p.Hk + h;
        vsc[u] = scale_of(p.v_exp[head * p.nb]);
        tok[u] = page * p.P + a.off;
        ok[u] = a.ok;
        const uint8_t* vb = p.v + (head * D + c16) * p.P + a.off;
#pragma unroll
        for (int m = 0; m < M; ++m) {
          const u32x2a8 x = *reinterpret_cast<const u32x2a8*>(vb + (size_t)(16 * m) * p.P);
          vc[m][2 * u] = x[0];
          vc[m][2 * u + 1] = x[1];
        }
      }
    }
  };
  auto advance = [&]() {
    if constexpr (!kSmallP) {
      kt += kWaves;
      while (kt >= p.tpp) {
        kt -= p.tpp;
        ++li;
      }
    }
  };

  for (int t = t_lo + wave; t < t_hi; t += kWaves) {
    locate(t);
    load_keys(t);
    load_values(t);
    bool masked = true;
    if constexpr (!kSmallP)
      masked = kt * 64 > p.P - 64 || lp * p.P + kt * 64 + 64 > lim_first;
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
    if (masked) {
#pragma unroll
      for (int n = 0; n < kCols; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int u = i >> 1, j = 4 * (i & 1) + r;
            if (!ok[u] || tok[u] + j >= lim[n]) s[n][i][r] = -INFINITY;
          }
      // Codes past the last token any row sees may be anything; a weight of 0 would
      // not take a NaN out.
#pragma unroll
      for (int m = 0; m < M; ++m) {
        const int n0 = ok[0] ? clampi(w.lim - tok[0], 0, 8) : 0, n1 = ok[1] ? clampi(w.lim - tok[1], 0, 8) : 0;
        const u32x4 lo = keep_codes(vc[m], n0), hi = keep_codes(u32x4{0, 0, vc[m][2], vc[m][3]}, 8 + n1);
        vc[m] = u32x4{lo[0], lo[1], hi[2], hi[3]};
      }
    }
    u32x4 pk[kCols][2][kParts];
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
        for (int k = 0; k < kParts; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t x = pack_bf16(e[2 * i], e[2 * i + 1]);
            pk[n][u][k][i] = x;
            if (k + 1 < kParts) {
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
          for (int k = 0; k < kParts; ++k) acc[n][m] = mfma16(a, pk[n][u][k], acc[n][m]);
      }
    advance();
  }

  // Join the waves: 16 rows at a time through LDS, then 16 threads a row.
#pragma unroll
  for (int n = 0; n < kCols; ++n) {
    l_run[n] += __shfl_xor(l_run[n], 16);
    l_run[n] += __shfl_xor(l_run[n], 32);
    if (g == 0) {
      msm[wave][16 * n + c16] = m_run[n];
      lsm[wave][16 * n + c16] = l_run[n];
    }
  }
  const int col = tid >> 4, d0 = (tid & 15) * (D / 16);
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
    float l = 0.f, o[D / 16] = {};
#pragma unroll
    for (int x = 0; x < kWaves; ++x) {
      const float wt = __builtin_amdgcn_exp2f((msm[x][row] - m_all) * c2);
      l += wt * lsm[x][row];
#pragma unroll
      for (int e = 0; e < D / 16; ++e) o[e] += wt * osm[(x * 16 + col) * OS + d0 + e];
    }
    if (i >= w.q_len) continue;
    if (whole) {
      cache8_store<T, D / 16>(p, b, i, h * p.G + r % p.G, d0, o, m_all, l, (tid & 15) == 0);
    } else {
      const size_t part = (((size_t)b * p.Hk + h) * p.n_split + split) * p.part_rows + r;
#pragma unroll
      for (int e = 0; e < D / 16; e += 4)
        *reinterpret_cast<f32x4*>(p.part_o + part * D + d0 + e) = f32x4{o[e], o[e + 1], o[e + 2], o[e + 3]};
      if ((tid & 15) == 0) reinterpret_cast<f32x2*>(p.part_ml)[part] = f32x2{m_all, l};
    }
  }
}

// Joins the pieces of a row whose tokens were split: a workgroup a row, each wave
// every fourth piece, in an order that does not depend on the launch's timing.
template <typename T, int D>
__global__ __launch_bounds__(256) void join_kernel(Cache8AttnParams p) {
  constexpr int E = D / 64;  // dims per lane
  __shared__ float osm[4][D], lsm[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r = blockIdx.x / p.Hk, h = blockIdx.x - r * p.Hk, b = blockIdx.y;
  const Cache8Walk w = cache8_walk(p, b, h, r / p.rows_per_item * p.rows_per_item, p.rows_per_item, lane);
  const int i = r / p.G;
  if (w.rows <= 0 || i >= w.q_len || w.n_tiles <= p.split_tiles) return;
  const int n = (w.n_tiles + p.split_tiles - 1) / p.split_tiles;
  const size_t part0 = ((size_t)b * p.Hk + h) * p.n_split * p.part_rows + r;
  const f32x2* ml = reinterpret_cast<const f32x2*>(p.part_ml);
  float m_all = -FLT_MAX;
  for (int s = lane; s < n; s += 64) m_all = fmaxf(m_all, ml[part0 + (size_t)s * p.part_rows][0]);
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) m_all = fmaxf(m_all, __shfl_xor(m_all, x));
  float l = 0.f, o[E] = {};
#pragma unroll 4
  for (int s = wave; s < n; s += 4) {
    const size_t part = part0 + (size_t)s * p.part_rows;
    const f32x2 x = ml[part];
    const float wt = __builtin_amdgcn_exp2f((x[0] - m_all) * p.scale_log2);
    l += wt * x[1];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] += wt * p.part_o[part * D + E * lane + e];
  }
#pragma unroll
  for (int e = 0; e < E; ++e) osm[wave][E * lane + e] = o[e];
  if (lane == 0) lsm[wave] = l;
  __syncthreads();
  if (wave) return;
  l = (lsm[0] + lsm[1]) + (lsm[2] + lsm[3]);
#pragma unroll
  for (int e = 0; e < E; ++e)
    o[e] = (osm[0][E * lane + e] + osm[1][E * lane + e]) + (osm[2][E * lane + e] + osm[3][E * lane + e]);
  cache8_store<T, E>(p, b, i, h * p.G + r % p.G, E * lane, o, m_all, l, lane == 0);
}

template <typename T, int D, int kCols, int kParts>
void launch_rows(const Cache8AttnParams& p, int B, hipStream_t s) {
  const dim3 grid(p.n_split * p.Hk * p.n_rt, B);
  if (p.P < 64) few_rows_kernel<T, D, kCols, kParts, true><<<grid, 64 * kWaves, 0, s>>>(p);
  else few_rows_kernel<T, D, kCols, kParts, false><<<grid, 64 * kWaves, 0, s>>>(p);
}

template <int D>
hipError_t launch_for(int dtype, int B, const Cache8AttnParams& p, hipStream_t s) {
  const int cols = p.rows_per_item / 16;
  if (dtype == HSA_DTYPE_BF16) {
    if (cols == 1) launch_rows<uint16_t, D, 1, 1>(p, B, s);
    else if (cols == 2) launch_rows<uint16_t, D, 2, 1>(p, B, s);
    else launch_rows<uint16_t, D, 4, 1>(p, B, s);
  } else {
    if (cols == 1) launch_rows<float, D, 1, 3>(p, B, s);
    else launch_rows<float, D, 2, 3>(p, B, s);
  }
  if (p.n_split > 1) {
    const dim3 grid(p.n_q * p.H, B);
    if (dtype == HSA_DTYPE_BF16) join_kernel<uint16_t, D><<<grid, 256, 0, s>>>(p);
    else join_kernel<float, D><<<grid, 256, 0, s>>>(p);
  }
  return hipGetLastError();
}

}  // namespace

void plan_cache8(Cache8AttnParams& p, int dtype, int B, int max_list_sel) {
  const int64_t rows = (int64_t)p.n_q * p.G;
  const int most = dtype == HSA_DTYPE_BF16 ? 4 : 2;
  p.rows_per_item = 16 * (rows <= 16 ? 1 : (rows <= 32 ? 2 : most));
  p.n_rt = (int)((rows + p.rows_per_item - 1) / p.rows_per_item);
  p.part_rows = p.n_rt * p.rows_per_item;
  p.nb = (p.P + 63) / 64;
  p.tpp = p.P < 64 ? 1 : p.nb;
  p.ppt = p.P < 64 && 64 % p.P == 0 ? 64 / p.P : 1;
  const int64_t list = (int64_t)max_list_sel + p.n_cur;
  const int64_t tiles = p.ppt > 1 ? (list + p.ppt - 1) / p.ppt : list * p.tpp;
  const int64_t items = (int64_t)B * p.Hk * p.n_rt;
  // about four workgroups a CU, pieces of at least eight tiles (two a wave)
  int64_t n = (1024 + items - 1) / items;
  n = std::max<int64_t>(1, std::min<int64_t>(n, (tiles + 7) / 8));
  int64_t c = std::max<int64_t>(1, (tiles + n - 1) / n);
  c = (c + kWaves - 1) / kWaves * kWaves;
  p.split_tiles = (int)c;
  p.n_split = (int)std::max<int64_t>(1, (tiles + c - 1) / c);
}

size_t cache8_part_bytes(int64_t B, int64_t Hk, int64_t n_split, int64_t part_rows, int64_t d) {
  return n_split > 1 ? (size_t)(B * Hk * n_split * part_rows * (d + 2)) * 4 : 0;
}

hipError_t launch_cache8_attention(int dtype, int d, int B, const Cache8AttnParams& p, hipStream_t s) {
  return d == 128 ? launch_for<128>(dtype, B, p, s) : launch_for<64>(dtype, B, p, s);
}

}  // namespace hsa
