// Token append: the keys and values of a step, token-major as a projection
// writes them, go to any run of a sequence's tokens in the paged cache, keys rotated by their
// position on the way: into the pool in its own type, or into the 8-bit cache.
//
// A workgroup takes one block of up to 64 tokens of a page (the tokens that share
// a scale) of one head: its keys turn in registers, its values are transposed through LDS into
// the d-major rows. For the 8-bit cache the turned keys wait in LDS in fp32 for the block's
// largest magnitude. A block that holds older tokens keeps its scale or
// grows it by a power of two; then, and only then, the older codes are read and
// written again (exact unless they become subnormal).
// Bound: HBM (the step's tokens read once, the codes written once); few
// tokens: the launch's latency.
#include "hsa_fp8.h"
#include "hsa_rope.h"

namespace hsa {
namespace {

constexpr int kTok = kScaleTok;  // tokens per workgroup

// n bits of largest finite magnitude seen so far
__device__ __forceinline__ float finite_max(float m, float x) {
  x = fabsf(x);
  return x < INFINITY ? fmaxf(m, x) : m;
}

template <typename T>
struct Vec16u;
template <>
struct Vec16u<uint16_t> {
  typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2)));
};
template <>
struct Vec16u<float> {
  typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4)));
};

template <typename T, int D, bool kEight>
__global__ __launch_bounds__(256) void token_write_kernel(TokenWriteParams p) {
  using V16 = typename Vec16u<T>::type;
  constexpr int E = Pack<T>::E;
  constexpr int CPR = D / E;                      // 16-byte chunks per token
  constexpr int NLD = kTok * CPR / 256;           // value chunks per thread
  constexpr int RW = D * (int)sizeof(T) / 4 + 1;  // dwords per value row: one more than d, so that rows fall on their own banks
  constexpr int KS = D + 4;                       // floats per key row
  __shared__ uint32_t vs[kTok * RW];
  __shared__ __attribute__((aligned(16))) float ks[kEight ? kTok * KS : 4];
  __shared__ float amax[2][4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int unit = blockIdx.x / p.H, h = blockIdx.x % p.H, b = blockIdx.y;
  // the step's tokens that fall into the table: [t0, t1) of the sequence
  const int64_t f = p.first ? p.first[b] : 0;
  const int64_t c = p.count ? min(p.count[b], p.n) : p.n;
  const int64_t t0 = f > 0 ? f : 0, cap = (int64_t)p.max_pages * p.P;
  const int64_t t1 = f + c < cap ? f + c : cap;
  if (t0 >= t1) return;
  // this unit's block, and the tokens [o0, o1) of it that the step brings
  const int nb = (p.P + kTok - 1) / kTok;
  const int64_t g = t0 / p.P * nb + t0 % p.P / kTok + unit;
  const int64_t page = g / nb;
  const int blk = (int)(g % nb), boff = blk * kTok;
  const int64_t base = page * p.P + boff;
  if (base >= t1) return;
  const int len = min(kTok, p.P - boff);
  const int o0 = t0 > base ? (int)(t0 - base) : 0;
  const int o1 = t1 - base < len ? (int)(t1 - base) : len;
  const int ntok = o1 - o0;
  if (ntok <= 0) return;
  const int i0 = (int)(base + o0 - f);            // first of them within the step
  const int slot = clampi(ld_const(p.page_table + (size_t)b * p.max_pages + page), 0, p.num_slots - 1);
  const size_t head = (size_t)slot * p.H + h;
  const T* ksrc = static_cast<const T*>(p.k_src) + (int64_t)b * p.k_batch + (int64_t)i0 * p.k_token + h * D;
  const T* vsrc = static_cast<const T*>(p.v_src) + (int64_t)b * p.v_batch + (int64_t)i0 * p.v_token + h * D;
  int ek_old = kScaleMin, ev_old = kScaleMin;
  if constexpr (kEight) {
    if (o0 > 0) {
      ek_old = (int)p.k_exp[head * nb + blk] - 127;
      ev_old = (int)p.v_exp[head * nb + blk] - 127;
    }
  }

  // values: all loads in flight, then the raw rows to LDS
  V16 v[NLD];
#pragma unroll
  for (int l = 0; l < NLD; ++l) {
    const int t = min((tid + 256 * l) / CPR, ntok - 1);
    v[l] = *reinterpret_cast<const V16*>(vsrc + (int64_t)t * p.v_token + tid % CPR * E);
  }
  // keys: two items (rope_items) at a time
  float mk = 0.f, mv = 0.f;
  const RopeTable& r = p.table;
  const int n_items = rope_items<T>(r.layout, r.rot, D);
  T* kdst = static_cast<T*>(p.k) + (head * p.P + boff) * D;
  for (int x0 = tid; x0 < ntok * n_items; x0 += 512) {
    RopeItem it[2];
    int t[2];
    float a[2][E], w[2][E];
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int x = min(x0 + 256 * y, ntok * n_items - 1);
      t[y] = x / n_items;
      it[y] = rope_item<T>(r.layout, r.rot, D, x - t[y] * n_items);
      const T* src = ksrc + (int64_t)t[y] * p.k_token + it[y].a;
      load_some<T>(src, it[y].n, a[y]);
      if (it[y].pairs) load_some<T>(src + r.rot / 2, it[y].n, w[y]);
    }
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      if (x0 + 256 * y >= ntok * n_items) break;
      int32_t pos[3];
      rope_positions(r, b, i0 + t[y], p.n, pos);
      float cs[E], sn[E];
      rope_item_angles<T>(r, it[y], pos, cs, sn);
      rope_turn<T>(r, it[y], cs, sn, a[y], w[y]);
      const int row = o0 + t[y];
      if constexpr (kEight) {
        float* dst = ks + row * KS + it[y].a;
#pragma unroll
        for (int i = 0; i < E; ++i) {
          if (i >= it[y].n) break;
          dst[i] = a[y][i];
          mk = finite_max(mk, a[y][i]);
          if (it[y].pairs) {
            dst[r.rot / 2 + i] = w[y][i];
            mk = finite_max(mk, w[y][i]);
          }
        }
      } else {
        T* dst = kdst + (size_t)row * D + it[y].a;
        store_some<T>(dst, it[y].n, a[y]);
        if (it[y].pairs) store_some<T>(dst + r.rot / 2, it[y].n, w[y]);
      }
    }
  }
#pragma unroll
  for (int l = 0; l < NLD; ++l) {
    const int t = (tid + 256 * l) / CPR;
    if (t >= ntok) continue;
    uint32_t* dst = vs + (o0 + t) * RW + tid % CPR * 4;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      dst[w] = v[l][w];
      if constexpr (kEight) {
        if constexpr (sizeof(T) == 2) {
          mv = finite_max(finite_max(mv, bf16_lo(v[l][w])), bf16_hi(v[l][w]));
        } else {
          mv = finite_max(mv, __uint_as_float(v[l][w]));
        }
      }
    }
  }
  if constexpr (!kEight) {
    __syncthreads();
    // value rows: runs of E tokens (16 bytes of a row), a dword of dims each
    constexpr int EPW = 4 / sizeof(T);
    constexpr int TG = kTok / E;
#pragma unroll 2
    for (int x = tid; x < TG * (RW - 1); x += 256) {
      const int g0 = x % TG * E, w = x / TG;
      if (g0 + E <= o0 || g0 >= o1) continue;
      uint32_t e[E];
#pragma unroll
      for (int i = 0; i < E; ++i) e[i] = vs[clampi(g0 + i, o0, o1 - 1) * RW + w];
      T* dst = static_cast<T*>(p.v) + (head * D + w * EPW) * p.P + boff + g0;
      const bool whole = g0 >= o0 && g0 + E <= o1;
      if constexpr (EPW == 2) {
        if (whole) {
          V16 lo, hi;  // dims 2 w and 2 w + 1
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            lo[i] = (e[2 * i] & 0xffffu) | (e[2 * i + 1] << 16);
            hi[i] = (e[2 * i] >> 16) | (e[2 * i + 1] & 0xffff0000u);
          }
          *reinterpret_cast<V16*>(dst) = lo;
          *reinterpret_cast<V16*>(dst + p.P) = hi;
        } else {
#pragma unroll
          for (int i = 0; i < E; ++i)
            if (g0 + i >= o0 && g0 + i < o1) {
              dst[i] = (uint16_t)e[i];
              dst[p.P + i] = (uint16_t)(e[i] >> 16);
            }
        }
      } else {
        if (whole) {
          *reinterpret_cast<V16*>(dst) = V16{e[0], e[1], e[2], e[3]};
        } else {
#pragma unroll
          for (int i = 0; i < E; ++i)
            if (g0 + i >= o0 && g0 + i < o1) dst[i] = __uint_as_float(e[i]);
        }
      }
    }
    return;
  } else {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      mk = fmaxf(mk, __shfl_xor(mk, m));
      mv = fmaxf(mv, __shfl_xor(mv, m));
    }
    if (lane == 0) {
      amax[0][wave] = mk;
      amax[1][wave] = mv;
    }
    __syncthreads();
    mk = fmaxf(fmaxf(amax[0][0], amax[0][1]), fmaxf(amax[0][2], amax[0][3]));
    mv = fmaxf(fmaxf(amax[1][0], amax[1][1]), fmaxf(amax[1][2], amax[1][3]));
    const int ek = max(scale_exponent(mk), ek_old), ev = max(scale_exponent(mv), ev_old);
    uint8_t* kc = static_cast<uint8_t*>(p.k) + (head * p.P + boff) * D;
    uint8_t* vc = static_cast<uint8_t*>(p.v) + head * D * p.P + boff;
    if (tid == 0) p.k_exp[head * nb + blk] = (uint8_t)(ek + 127);
    if (tid == 64) p.v_exp[head * nb + blk] = (uint8_t)(ev + 127);
    {
      const bool grow = o0 > 0 && ek > ek_old;
      const float inv = pow2i(-ek), shift = pow2i(ek_old - ek);
      const int r0 = grow ? 0 : o0;
      for (int x = tid; x < (o1 - r0) * (D / 16); x += 256) {
        const int row = r0 + x / (D / 16), d0 = x % (D / 16) * 16;
        u32x4* dst = reinterpret_cast<u32x4*>(kc + (size_t)row * D + d0);
        u32x4 w;
        if (row >= o0) {
          const f32x4* src = reinterpret_cast<const f32x4*>(ks + row * KS + d0);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const f32x4 y = src[i];
            w[i] = codes4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
          }
        } else {
          const u32x4 was = *dst;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            w[i] = codes4(code_to_f32(was[i] & 255u) * shift, code_to_f32(was[i] >> 8 & 255u) * shift,
                          code_to_f32(was[i] >> 16 & 255u) * shift, code_to_f32(was[i] >> 24) * shift);
        }
        *dst = w;
      }
    }
    {
      const bool grow = o0 > 0 && ev > ev_old;
      const float inv = pow2i(-ev), shift = pow2i(ev_old - ev);
      const int r0 = grow ? 0 : o0;
      constexpr int EPW = 4 / sizeof(T);  // dims per dword
      // runs of 16 tokens of a dword of dims
      for (int x = tid; x < 4 * (RW - 1); x += 256) {
        const int g0 = x % 4 * 16, w = x / 4;
        if (g0 + 16 <= r0 || g0 >= o1) continue;
#pragma unroll
        for (int e = 0; e < EPW; ++e) {
          uint8_t* dst = vc + (size_t)(w * EPW + e) * p.P + g0;
          u32x4 code;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int t = g0 + 4 * i + j;
              const uint32_t raw = vs[clampi(t, o0, o1 - 1) * RW + w];
              const float nv = sizeof(T) == 4 ? __uint_as_float(raw) : (e ? bf16_hi(raw) : bf16_lo(raw));
              y[j] = nv * inv;
              if (grow && t < o0) y[j] = code_to_f32(dst[4 * i + j]) * shift;
            }
            code[i] = codes4(y[0], y[1], y[2], y[3]);
          }
          if (g0 >= r0 && g0 + 16 <= o1) {
            *reinterpret_cast<u32x4a8*>(dst) = u32x4a8{code[0], code[1], code[2], code[3]};
          } else {
#pragma unroll
            for (int t = 0; t < 16; ++t)
              if (g0 + t >= r0 && g0 + t < o1) dst[t] = (uint8_t)(code[t / 4] >> (8 * (t % 4)));
          }
        }
      }
    }
  }
}

template <typename T, int D>
void launch_for(bool eight, dim3 grid, const TokenWriteParams& p, hipStream_t s) {
  if (eight) token_write_kernel<T, D, true><<<grid, 256, 0, s>>>(p);
  else token_write_kernel<T, D, false><<<grid, 256, 0, s>>>(p);
}

}  // namespace

// Blocks that n tokens of a sequence can touch, wherever they begin: a boundary
// every 64 tokens of a page, and one more at a page's end if a short block is there.
int64_t token_write_units(int64_t n, int P) {
  return 2 + n / kTok + (P % kTok ? n / P + 2 : 0);
}

hipError_t launch_token_write(int dtype, int d, int B, bool eight, const TokenWriteParams& p, hipStream_t s) {
  const dim3 grid((uint32_t)(token_write_units(p.n, p.P) * p.H), B);
  if (dtype == HSA_DTYPE_BF16) {
    if (d == 128) launch_for<uint16_t, 128>(eight, grid, p, s);
    else launch_for<uint16_t, 64>(eight, grid, p, s);
  } else {
    if (d == 128) launch_for<float, 128>(eight, grid, p, s);
    else launch_for<float, 64>(eight, grid, p, s);
  }
  return hipGetLastError();
}

}  // namespace hsa
