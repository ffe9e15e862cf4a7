// Token append: the keys and values of a step, token-major as a projection
// writes them, go to any run of a sequence's tokens in the paged cache, keys rotated by their
// position on the way: into the pool in its own type, or into the 8-bit cache.
//
// A workgroup takes one block of up to 64 tokens of a page (the tokens that share
// a scale) of one head: its keys turn in registers, where they wait for the block's largest
// magnitude, its values are transposed through LDS into the d-major rows. A block that holds older tokens keeps its scale or
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

// N codes of x in units of 1 / inv.
template <int N>
__device__ __forceinline__ void store_codes(uint8_t* p, const float (&x)[N], float inv) {
  if constexpr (N == 1) {
    *p = (uint8_t)codes4(x[0] * inv, 0.f, 0.f, 0.f);
  } else {
    uint32_t* w = reinterpret_cast<uint32_t*>(p);
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
      w[i] = codes4(x[4 * i] * inv, x[4 * i + 1] * inv, x[4 * i + 2] * inv, x[4 * i + 3] * inv);
  }
}

template <typename T, int D, bool kEight, int kMode>
__global__ __launch_bounds__(256) void token_write_kernel(TokenWriteParams p) {
  using V16 = typename Vec16<T>::type;
  using Item = RopeItem<T, kMode>;
  constexpr int E = 16 / (int)sizeof(T);
  constexpr int CPR = D / E;                      // 16-byte chunks per token
  constexpr int NLD = kTok * CPR / 256;           // value chunks per thread
  constexpr int RW = D * (int)sizeof(T) / 4 + 1;  // dwords per value row: one more than d, so that rows fall on their own banks
  __shared__ uint32_t vs[kTok * RW];
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
  // keys: a thread has one item (RopeItem) of every 256 >> item_shift tokens; its turned
  // elements stay in registers until the block's scale is known
  float mk = 0.f, mv = 0.f;
  const RopeTable& r = p.table;
  const int step = 256 >> p.item_shift;
  const int j = tid & ((1 << p.item_shift) - 1), tk = tid >> p.item_shift;
  Item it;
  it.set(r, j);
  const bool mine = j < Item::count(r.rot, D);
  T* kdst = static_cast<T*>(p.k) + (head * p.P + boff) * D;
  constexpr int NK = kMode == kRopeSingle ? 1 : kTok * D / E / 256;
  float ku[NK][Item::N], kw[NK][Item::N];
  auto turned = [&](int t, const typename Item::El::Raw& ra, const typename Item::El::Raw& rb, float (&u)[Item::N],
                    float (&w)[Item::N]) {
    float cs[Item::NP], sn[Item::NP];
    it.angles(r, rope_positions(r, b, i0 + t, p.n), cs, sn);
    it.result(ra, rb, cs, sn, u, w);
  };
  auto largest = [&](const float (&u)[Item::N], const float (&w)[Item::N]) {
#pragma unroll
    for (int i = 0; i < Item::N; ++i) {
      mk = finite_max(mk, u[i]);
      if (kMode != kRopeInterleaved && it.turn) mk = finite_max(mk, w[i]);
    }
  };
  if constexpr (kMode != kRopeSingle) {
    typename Item::El::Raw ra[NK], rb[NK];
#pragma unroll
    for (int k = 0; k < NK; ++k)
      if (mine) it.load(ksrc + (int64_t)min(tk + k * step, ntok - 1) * p.k_token, ra[k], rb[k]);
    if (mine) {
      it.frequencies(r);
#pragma unroll
      for (int k = 0; k < NK; ++k) {
        const int t = tk + k * step;
        if (t < ntok) {
          turned(t, ra[k], rb[k], ku[k], kw[k]);
          if constexpr (kEight) largest(ku[k], kw[k]);
          else it.store(kdst + (size_t)(o0 + t) * D, ku[k], kw[k]);
        }
      }
    }
  } else if (mine) {
    it.frequencies(r);
    for (int t = tk; t < ntok; t += step) {
      typename Item::El::Raw ra, rb;
      it.load(ksrc + (int64_t)t * p.k_token, ra, rb);
      turned(t, ra, rb, ku[0], kw[0]);
      if constexpr (kEight) largest(ku[0], kw[0]);
      else it.store(kdst + (size_t)(o0 + t) * D, ku[0], kw[0]);
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
      const float inv = pow2i(-ek);
      auto put = [&](int t, const float (&u)[Item::N], const float (&w)[Item::N]) {
        uint8_t* row = kc + (size_t)(o0 + t) * D;
        store_codes<Item::N>(row + it.a, u, inv);
        if (kMode != kRopeInterleaved && it.turn) store_codes<Item::N>(row + it.b, w, inv);
      };
      if constexpr (kMode != kRopeSingle) {
#pragma unroll
        for (int k = 0; k < NK; ++k)
          if (mine && tk + k * step < ntok) put(tk + k * step, ku[k], kw[k]);
      } else if (mine) {
        for (int t = tk; t < ntok; t += step) {  // (turned again: one pair a thread is too many to keep)
          typename Item::El::Raw ra, rb;
          it.load(ksrc + (int64_t)t * p.k_token, ra, rb);
          turned(t, ra, rb, ku[0], kw[0]);
          put(t, ku[0], kw[0]);
        }
      }
      if (o0 > 0 && ek > ek_old) {  // the older rows, scaled down
        const float shift = pow2i(ek_old - ek);
        for (int x = tid; x < o0 * (D / 16); x += 256) {
          u32x4* dst = reinterpret_cast<u32x4*>(kc + 16 * x);
          u32x4 w = *dst;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            w[i] = codes4(code_to_f32(w[i] & 255u) * shift, code_to_f32(w[i] >> 8 & 255u) * shift,
                          code_to_f32(w[i] >> 16 & 255u) * shift, code_to_f32(w[i] >> 24) * shift);
          *dst = w;
        }
      }
    }
    {
      const bool grow = o0 > 0 && ev > ev_old;
      const float inv = pow2i(-ev), shift = pow2i(ev_old - ev);
      const int r0 = grow ? 0 : o0;
      constexpr int EPW = 4 / sizeof(T);  // dims per dword
      if (!grow && ntok <= 4) {
        // a few tokens (of a step that decodes): an element a thread
        for (int x = tid; x < ntok * D; x += 256) {
          const int t = o0 + x / D, e = x % D;
          const uint32_t raw = vs[t * RW + e / EPW];
          const float y = (sizeof(T) == 4 ? __uint_as_float(raw) : (e & 1 ? bf16_hi(raw) : bf16_lo(raw))) * inv;
          vc[(size_t)e * p.P + t] = (uint8_t)codes4(y, y, y, y);
        }
        return;
      }
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

template <typename T, int D, bool kEight, int kMode>
void launch_mode(dim3 grid, TokenWriteParams p, hipStream_t s) {
  const int n = RopeItem<T, kMode>::count(p.table.rot, D);
  while (1 << p.item_shift < n) ++p.item_shift;
  token_write_kernel<T, D, kEight, kMode><<<grid, 256, 0, s>>>(p);
}

template <typename T, int D, bool kEight>
void launch_as(dim3 grid, const TokenWriteParams& p, hipStream_t s) {
  switch (rope_mode<T>(p.table)) {
    case kRopeHalves: return launch_mode<T, D, kEight, kRopeHalves>(grid, p, s);
    case kRopeInterleaved: return launch_mode<T, D, kEight, kRopeInterleaved>(grid, p, s);
    default: return launch_mode<T, D, kEight, kRopeSingle>(grid, p, s);
  }
}

template <typename T, int D>
void launch_for(bool eight, dim3 grid, const TokenWriteParams& p, hipStream_t s) {
  if (eight) launch_as<T, D, true>(grid, p, s);
  else launch_as<T, D, false>(grid, p, s);
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
