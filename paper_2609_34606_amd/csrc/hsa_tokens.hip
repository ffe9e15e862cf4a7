// Token append: the keys and values of a step, token-major as a projection
// writes them, go to any run of a sequence's tokens in the paged cache, keys rotated by their
// position on the way: into the pool in its own type, or into the 8-bit cache.
//
// A workgroup takes one block of up to 64 tokens of a page (the tokens that share a scale): the
// keys of one head or two, which turn in registers and wait there for the block's largest
// magnitude, or the values of one, which are transposed through LDS into the d-major
// rows. A block that holds older tokens keeps its scale or grows it by a power of two; then, and
// only then, the older codes are read and written again (exact unless they become
// subnormal).
// Bound: HBM (the step's tokens read once, the codes written once): 4680 tokens, 12 heads x
// d128, out of a fused projection (43 MB) in 15.5 us, four such sequences in 49 us (3.5
// TB/s, a copy 5.1: a head's rows are 256 bytes of every token's 9216, a value row's new codes
// 64 bytes); for few tokens the launch's latency, 6.8 us for 32 single ones.
#include "hsa_fp8.h"
#include "hsa_rope.h"

namespace hsa {

// Blocks that n tokens of a sequence can touch, wherever they begin: a boundary
// every 64 tokens of a page, and one more at a page's end if a short block is there.
int64_t token_write_units(int64_t n, int P) {
  return 2 + n / kScaleTok + (P % kScaleTok ? n / P + 2 : 0);
}

namespace {


// N codes of x / 2^e (scale = 2^e).
template <int N>
__device__ __forceinline__ void store_codes(uint8_t* p, const float (&x)[N], float scale) {
  if constexpr (N == 1) {
    *p = (uint8_t)codes2(x[0], 0.f, scale);
  } else {
    uint32_t* w = reinterpret_cast<uint32_t*>(p);
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
      w[i] = codes4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3], scale);
  }
}

// Four codes scaled by a power of two.
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float shift) {
  return codes4(code_to_f32(w & 255u) * shift, code_to_f32(w >> 8 & 255u) * shift, code_to_f32(w >> 16 & 255u) * shift,
                code_to_f32(w >> 24) * shift, 1.f);
}

// Largest magnitude of a dword of T, as fp32 bits or above (NaN and infinities are
// 0x7f800000 and above): bf16 as two 16-bit magnitudes.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <typename T>
__device__ __forceinline__ uint32_t max_bits(uint32_t m, uint32_t w) {
  if constexpr (sizeof(T) == 2)
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m),
                                                                  __builtin_bit_cast(u16x2, w & 0x7fff7fffu)));
  return max(m, w & 0x7fffffffu);
}
template <typename T>
__device__ __forceinline__ uint32_t max_bits_f32(uint32_t m) {
  if constexpr (sizeof(T) == 2) return max(m << 16, m & 0xffff0000u);
  return m;
}

// Largest of a value over the workgroup's kW waves. buf: one slot a wave. What the workgroup has
// put into shared memory is there afterwards.
template <int kW>
__device__ __forceinline__ uint32_t max_all(uint32_t a, uint32_t* buf, int tid) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) a = max(a, (uint32_t)__shfl_xor((int)a, m));
  if ((tid & 63) == 0) buf[tid >> 6] = a;
  __syncthreads();
  uint32_t most = buf[0];
#pragma unroll
  for (int w = 1; w < kW; ++w) most = max(most, buf[w]);
  return most;
}

constexpr uint32_t kInf = 0x7f800000u;
__device__ __forceinline__ void finite_bits(uint32_t& m, float x) {
  const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
  m = u < kInf ? max(m, u) : m;
}

// One block of a sequence and the tokens of the step that fall into it.
struct TokenBlock {
  int b, page, blk, boff;  // batch entry, logical page, block of the page and its first token there
  int o0, o1, ntok;        // the step's tokens [o0, o1) of the block
  int i0;                  // the first of them within the step
  int nb;
};

// kTok: most tokens of a block; four threads each.
template <typename T, int D, bool kEight, int kMode, int kTok>
__device__ __forceinline__ void write_keys(const TokenWriteParams& p, const TokenBlock& t, int h_lo, int h_hi,
                                           uint32_t* amax) {
  using Item = RopeItem<T, kMode>;
  using Raw = typename Item::El::Raw;
  constexpr int E = 16 / (int)sizeof(T);
  constexpr int kThreads = 4 * kTok;
  constexpr int NK = kMode == kRopeSingle ? 1 : D / E / (kMode == kRopeHalves ? 8 : 4);  // items a thread
  const int tid = threadIdx.x, ntok = t.ntok;
  const T* ksrc = static_cast<const T*>(p.k_src) + (int64_t)t.b * p.k_batch + (int64_t)t.i0 * p.k_token;
  // A thread has one item (RopeItem) of every kThreads >> item_shift tokens.
  const RopeTable& r = p.table;
  const int step = kThreads >> p.item_shift, tk = tid >> p.item_shift, j = tid & ((1 << p.item_shift) - 1);
  Item it;
  it.set(r, j);
  const bool mine = j < Item::count(r.rot, D);
  Raw ra[NK], rb[NK];
  auto load = [&](int h) {
    if (kMode != kRopeSingle && mine) {
#pragma unroll
      for (int k = 0; k < NK; ++k)
        it.load(ksrc + (int64_t)min(tk + k * step, ntok - 1) * p.k_token + h * D, ra[k], rb[k]);
    }
  };
  load(h_lo);
  const size_t slot =
      clampi(ld_const(p.page_table + (size_t)t.b * p.max_pages + t.page), 0, p.num_slots - 1);
  it.frequencies(r);
  float cs[NK][Item::NP], sn[NK][Item::NP];
  auto angles = [&](int i, int k) { it.angles(r, rope_positions(r, t.b, t.i0 + i, p.n), cs[k], sn[k]); };
  if (kMode != kRopeSingle && mine && it.turn) {
#pragma unroll
    for (int k = 0; k < NK; ++k)
      if (tk + k * step < ntok) angles(tk + k * step, k);
  }
  for (int h = h_lo; h < h_hi; ++h) {
    const size_t head = slot * p.H + h;
    int e_old = kScaleMin;
    if (kEight && t.o0 > 0) e_old = (int)p.k_exp[head * t.nb + t.blk] - 127;
    float mk = 0.f;
    float ku[NK][Item::N], kw[NK][Item::N];
    T* kdst = kEight ? nullptr : static_cast<T*>(p.k) + (head * p.P + t.boff + t.o0) * D;
    // (NaN does not count: it keeps its code under any scale)
    auto largest = [&](int k) {
#pragma unroll
      for (int i = 0; i < Item::N; ++i) {
        mk = fmaxf(mk, fabsf(ku[k][i]));
        if (kMode != kRopeInterleaved && it.turn) mk = fmaxf(mk, fabsf(kw[k][i]));
      }
    };
    // single: the item's pair at token i (turned again where it is needed: one pair a
    // thread makes too many to keep)
    auto single = [&](int i) {
      it.load(ksrc + (int64_t)i * p.k_token + h * D, ra[0], rb[0]);
      if (it.turn) angles(i, 0);
      it.result(ra[0], rb[0], cs[0], sn[0], ku[0], kw[0]);
    };
    if (mine) {
      if constexpr (kMode != kRopeSingle) {
#pragma unroll
        for (int k = 0; k < NK; ++k)
          if (tk + k * step < ntok) {
            it.result(ra[k], rb[k], cs[k], sn[k], ku[k], kw[k]);
            if constexpr (kEight) largest(k);
            else it.store(kdst + (size_t)(tk + k * step) * D, ku[k], kw[k]);
          }
      } else {
        for (int i = tk; i < ntok; i += step) {
          single(i);
          if constexpr (kEight) largest(0);
          else it.store(kdst + (size_t)i * D, ku[0], kw[0]);
        }
      }
    }
    if (h + 1 < h_hi) load(h + 1);  // in flight during what follows
    if constexpr (kEight) {
      if (h > h_lo) __syncthreads();  // (the last head's maxima have been read)
      uint32_t bits = max_all<kThreads / 64>(__float_as_uint(mk), amax, tid);
      const bool wild = bits >= kInf;
      if (wild) {  // the largest finite magnitude
        __syncthreads();
        bits = 0;
        if (mine) {
          for (int i = tk, k = 0; i < ntok; i += step, ++k) {
            if constexpr (kMode == kRopeSingle) single(i);
#pragma unroll
            for (int kk = 0; kk < NK; ++kk)
              if (kMode == kRopeSingle || kk == k) {
#pragma unroll
                for (int x = 0; x < Item::N; ++x) {
                  finite_bits(bits, ku[kk][x]);
                  if (kMode != kRopeInterleaved && it.turn) finite_bits(bits, kw[kk][x]);
                }
              }
          }
        }
        bits = max_all<kThreads / 64>(bits, amax, tid);
      }
      const int e = max(scale_exponent(__uint_as_float(bits)), e_old);
      const float scale = wild ? 1.f : pow2i(e);
      if (tid == 0) p.k_exp[head * t.nb + t.blk] = (uint8_t)(e + 127);
      uint8_t* kc = static_cast<uint8_t*>(p.k) + (head * p.P + t.boff) * D;
      auto put = [&](int i, int k) {
        uint8_t* row = kc + (size_t)(t.o0 + i) * D;
        if (wild) {  // infinities become the largest code (in units of the scale: 448 * 2^120 is no fp32 number)
          const float unit = pow2i(-e);
#pragma unroll
          for (int x = 0; x < Item::N; ++x) {
            ku[k][x] = saturate(ku[k][x] * unit, kCodeMax);
            kw[k][x] = saturate(kw[k][x] * unit, kCodeMax);
          }
        }
        store_codes<Item::N>(row + it.a, ku[k], scale);
        if (kMode != kRopeInterleaved && it.turn) store_codes<Item::N>(row + it.b, kw[k], scale);
      };
      if (mine) {
        if constexpr (kMode != kRopeSingle) {
#pragma unroll
          for (int k = 0; k < NK; ++k)
            if (tk + k * step < ntok) put(tk + k * step, k);
        } else {
          for (int i = tk; i < ntok; i += step) {
            single(i);
            put(i, 0);
          }
        }
      }
      if (t.o0 > 0 && e > e_old) {  // the older rows, scaled down
        const float shift = pow2i(e_old - e);
        for (int x = tid; x < t.o0 * (D / 16); x += kThreads) {
          u32x4* dst = reinterpret_cast<u32x4*>(kc + 16 * x);
          u32x4 w = *dst;
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = rescale4(w[i], shift);
          *dst = w;
        }
      }
    }
  }
}

// vs: kTok rows of RW dwords, one more than a row's values, so that rows fall on their own banks.
template <typename T, int D, bool kEight, int kTok>
__device__ __forceinline__ void write_values(const TokenWriteParams& p, const TokenBlock& t, int h, uint32_t* vs,
                                             uint32_t* amax) {
  using V16 = typename Vec16<T>::type;
  constexpr int E = 16 / (int)sizeof(T);
  constexpr int CPR = D / E;                      // 16-byte chunks per token
  constexpr int kThreads = 4 * kTok;
  constexpr int NLD = CPR / 4;                    // chunks per thread
  constexpr int RW = D * (int)sizeof(T) / 4 + 1;  // dwords per LDS row
  constexpr int EPW = 4 / (int)sizeof(T);         // dims per dword
  const int tid = threadIdx.x, ntok = t.ntok, o0 = t.o0, o1 = t.o1;
  const T* src = static_cast<const T*>(p.v_src) + (int64_t)t.b * p.v_batch + (int64_t)t.i0 * p.v_token + h * D;
  V16 v[NLD];
#pragma unroll
  for (int l = 0; l < NLD; ++l)
    v[l] = *reinterpret_cast<const V16*>(src + (int64_t)min((tid + kThreads * l) / CPR, ntok - 1) * p.v_token +
                                         tid % CPR * E);
  const size_t slot =
      clampi(ld_const(p.page_table + (size_t)t.b * p.max_pages + t.page), 0, p.num_slots - 1);
  const size_t head = slot * p.H + h;
  int e_old = kScaleMin;
  if (kEight && o0 > 0) e_old = (int)p.v_exp[head * t.nb + t.blk] - 127;
  uint32_t mv = 0;
#pragma unroll
  for (int l = 0; l < NLD; ++l) {
    const int i = (tid + kThreads * l) / CPR;
    if (i >= ntok) continue;
    uint32_t* dst = vs + (o0 + i) * RW + tid % CPR * 4;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      dst[w] = v[l][w];
      if constexpr (kEight) mv = max_bits<T>(mv, v[l][w]);
    }
  }
  if constexpr (!kEight) {
    __syncthreads();
    // value rows: runs of E tokens (16 bytes of a row), a dword of dims each
    constexpr int TG = kTok / E;
#pragma unroll 2
    for (int x = tid; x < TG * (RW - 1); x += kThreads) {
      const int g0 = x % TG * E, w = x / TG;
      if (g0 + E <= o0 || g0 >= o1) continue;
      uint32_t e[E];
#pragma unroll
      for (int i = 0; i < E; ++i) e[i] = vs[clampi(g0 + i, o0, o1 - 1) * RW + w];
      T* dst = static_cast<T*>(p.v) + (head * D + w * EPW) * p.P + t.boff + g0;
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
  } else {
    uint32_t bits = max_all<kThreads / 64>(max_bits_f32<T>(mv), amax, tid);  // (its barrier: the rows are there)
    const bool wild = bits >= kInf;                            // infinities or NaN
    if (wild) {  // the largest finite magnitude
      __syncthreads();
      bits = 0;
      for (int x = tid; x < ntok * (RW - 1); x += kThreads) {
        const uint32_t w = vs[(o0 + x / (RW - 1)) * RW + x % (RW - 1)];
        if constexpr (sizeof(T) == 2) {
          finite_bits(bits, bf16_lo(w));
          finite_bits(bits, bf16_hi(w));
        } else {
          finite_bits(bits, __uint_as_float(w));
        }
      }
      bits = max_all<kThreads / 64>(bits, amax, tid);
    }
    const int e = max(scale_exponent(__uint_as_float(bits)), e_old);
    const float scale = wild ? 1.f : pow2i(e);
    if (tid == 0) p.v_exp[head * t.nb + t.blk] = (uint8_t)(e + 127);
    uint8_t* vc = static_cast<uint8_t*>(p.v) + head * D * p.P + t.boff;
    if (wild) {  // infinities become the largest code, as in write_keys (exact in bf16 too)
      const float unit = pow2i(-e);
      for (int x = tid; x < ntok * (RW - 1); x += kThreads) {
        uint32_t& w = vs[(o0 + x / (RW - 1)) * RW + x % (RW - 1)];
        if constexpr (sizeof(T) == 2)
          w = pack_bf16(saturate(bf16_lo(w) * unit, kCodeMax), saturate(bf16_hi(w) * unit, kCodeMax));
        else
          w = __float_as_uint(saturate(__uint_as_float(w) * unit, kCodeMax));
      }
      __syncthreads();
    }
    const bool grow = o0 > 0 && e > e_old;
    if (!grow && ntok <= 4) {
      // a few tokens (of a step that decodes): an element a thread
      for (int x = tid; x < ntok * D; x += kThreads) {
        const int i = o0 + x / D, c = x % D;
        const uint32_t raw = vs[i * RW + c / EPW];
        const float y = sizeof(T) == 4 ? __uint_as_float(raw) : (c & 1 ? bf16_hi(raw) : bf16_lo(raw));
        vc[(size_t)c * p.P + i] = (uint8_t)codes2(y, y, scale);
      }
      return;
    }
    // runs of 16 tokens (of small pages: 8) of a dword of dims
    constexpr int R = kTok >= 64 ? 16 : 8, kRuns = kTok / R;
    typedef uint32_t Run __attribute__((ext_vector_type(R / 4), aligned(8)));
    const float shift = pow2i(e_old - e);
    const int r0 = grow ? 0 : o0;
    for (int x = tid; x < kRuns * (RW - 1); x += kThreads) {
      const int g0 = x % kRuns * R, w = x / kRuns;
      uint8_t* dst = vc + (size_t)(w * EPW) * p.P + g0;
      if (g0 >= o0 && g0 + R <= o1) {
        const uint32_t* row = vs + g0 * RW + w;
        uint32_t c[R];
#pragma unroll
        for (int i = 0; i < R; ++i) c[i] = row[i * RW];
        Run lo, hi;  // dims EPW w and, in bf16, the next
#pragma unroll
        for (int i = 0; i < R / 4; ++i) {
          if constexpr (EPW == 2) {
            // pairs of tokens of one dim
            const uint32_t a0 = __builtin_amdgcn_perm(c[4 * i + 1], c[4 * i], 0x05040100u);
            const uint32_t a1 = __builtin_amdgcn_perm(c[4 * i + 3], c[4 * i + 2], 0x05040100u);
            const uint32_t b0 = __builtin_amdgcn_perm(c[4 * i + 1], c[4 * i], 0x07060302u);
            const uint32_t b1 = __builtin_amdgcn_perm(c[4 * i + 3], c[4 * i + 2], 0x07060302u);
            lo[i] = codes4_bf16(a0, a1, scale);
            hi[i] = codes4_bf16(b0, b1, scale);
          } else {
            lo[i] = codes4(__uint_as_float(c[4 * i]), __uint_as_float(c[4 * i + 1]), __uint_as_float(c[4 * i + 2]),
                           __uint_as_float(c[4 * i + 3]), scale);
          }
        }
        *reinterpret_cast<Run*>(dst) = lo;
        if constexpr (EPW == 2) *reinterpret_cast<Run*>(dst + p.P) = hi;
      } else if (g0 + R > r0 && g0 < o1) {
        // a run that the step begins or ends in, or of older tokens
        for (int i = max(g0, r0); i < min(g0 + R, o1); ++i) {
#pragma unroll
          for (int c = 0; c < EPW; ++c) {
            uint8_t* one = dst + (size_t)c * p.P + (i - g0);
            const uint32_t raw = vs[max(i, o0) * RW + w];
            const float y = EPW == 1 ? __uint_as_float(raw) : (c ? bf16_hi(raw) : bf16_lo(raw));
            *one = (uint8_t)(i < o0 ? codes2(code_to_f32(*one) * shift, 0.f, 1.f) : codes2(y, 0.f, scale));
          }
        }
      }
    }
  }
}

// A workgroup writes one block's keys of p.heads heads, or its values of one.
template <typename T, int D, bool kEight, int kMode, int kTok>
__global__ __launch_bounds__(4 * kTok) void token_write_kernel(TokenWriteParams p) {
  __shared__ uint32_t vs[kTok * (D * (int)sizeof(T) / 4 + 1)];
  __shared__ uint32_t amax[kTok / 16];
  const int groups = (p.H + p.heads - 1) / p.heads;
  const int unit = blockIdx.x / p.roles, role = blockIdx.x - unit * p.roles;
  if (role >= groups + p.H) return;
  TokenBlock t;
  t.b = blockIdx.y;
  // the step's tokens that fall into the table: [t0, t1) of the sequence
  const int64_t f = p.first ? p.first[t.b] : 0;
  const int64_t c = p.count ? min(p.count[t.b], p.n) : p.n;
  const int64_t t0 = f > 0 ? f : 0, cap = (int64_t)p.max_pages * p.P;
  const int64_t t1 = f + c < cap ? f + c : cap;
  if (t0 >= t1) return;
  // this unit's block, and the tokens of it that the step brings (tokens of the table are
  // below 2^31, see hsa_cache8_t)
  t.nb = (p.P + kScaleTok - 1) / kScaleTok;
  const int page0 = (int)t0 / p.P;
  const int g = ((int)t0 - page0 * p.P) / kScaleTok + unit;
  t.page = page0 + g / t.nb;
  t.blk = g % t.nb;
  t.boff = t.blk * kScaleTok;
  const int64_t base = (int64_t)t.page * p.P + t.boff;
  if (base >= t1) return;
  const int len = min(kScaleTok, p.P - t.boff);  // (at most kTok)
  t.o0 = t0 > base ? (int)(t0 - base) : 0;
  t.o1 = t1 - base < len ? (int)(t1 - base) : len;
  t.ntok = t.o1 - t.o0;
  if (t.ntok <= 0) return;
  t.i0 = (int)(base + t.o0 - f);
  if (role < groups) write_keys<T, D, kEight, kMode, kTok>(p, t, role * p.heads, min((role + 1) * p.heads, p.H), amax);
  else write_values<T, D, kEight, kTok>(p, t, role - groups, vs, amax);
}

template <typename T, int D, bool kEight, int kMode, int kTok>
void launch_mode(int B, TokenWriteParams p, hipStream_t s) {
  const int n = RopeItem<T, kMode>::count(p.table.rot, D);
  while (1 << p.item_shift < n) ++p.item_shift;
  // Two heads a workgroup share the angles of their tokens, once that leaves work for every
  // CU (8-bit append of 4680 tokens, 12 heads x d128: one 16.6 us, two 15.8, three 20.2, four
  // 16.1; four sequences at once 51.3, 49.2, 62.3, 51.6).
  const int64_t wgs = (int64_t)((p.n + kScaleTok - 1) / kScaleTok) * p.H * B;
  p.heads = kMode != kRopeSingle && wgs >= 768 ? 2 : 1;
  p.roles = (p.H + p.heads - 1) / p.heads + p.H;
  const dim3 grid((uint32_t)(token_write_units(p.n, p.P) * p.roles), B);
  token_write_kernel<T, D, kEight, kMode, kTok><<<grid, 4 * kTok, 0, s>>>(p);
}

// Pages of up to 16 tokens are blocks of a wave each, so that a CU holds more of them (8-bit append
// of 4680 tokens, 12 heads x d128, pages of 8: 16.7 us, by four waves 44.5; of 16: 15.1 and 22.6). A
// token's items have to fit its threads: single pairs of d = 128 do not.
template <typename T, int D, bool kEight, int kMode>
void launch_blocks(int B, const TokenWriteParams& p, hipStream_t s) {
  if (p.P <= 16 && RopeItem<T, kMode>::count(p.table.rot, D) <= 64) launch_mode<T, D, kEight, kMode, 16>(B, p, s);
  else launch_mode<T, D, kEight, kMode, kScaleTok>(B, p, s);
}

template <typename T, int D, bool kEight>
void launch_as(int B, const TokenWriteParams& p, hipStream_t s) {
  switch (rope_mode<T>(p.table, D)) {
    case kRopeHalves: return launch_blocks<T, D, kEight, kRopeHalves>(B, p, s);
    case kRopePart: return launch_blocks<T, D, kEight, kRopePart>(B, p, s);
    case kRopeInterleaved: return launch_blocks<T, D, kEight, kRopeInterleaved>(B, p, s);
    default: return launch_blocks<T, D, kEight, kRopeSingle>(B, p, s);
  }
}

template <typename T, int D>
void launch_for(int B, bool eight, const TokenWriteParams& p, hipStream_t s) {
  if (eight) launch_as<T, D, true>(B, p, s);
  else launch_as<T, D, false>(B, p, s);
}

}  // namespace

hipError_t launch_token_write(int dtype, int d, int B, bool eight, const TokenWriteParams& p, hipStream_t s) {
  if (dtype == HSA_DTYPE_BF16) {
    if (d == 128) launch_for<uint16_t, 128>(B, eight, p, s);
    else launch_for<uint16_t, 64>(B, eight, p, s);
  } else {
    if (d == 128) launch_for<float, 128>(B, eight, p, s);
    else launch_for<float, 64>(B, eight, p, s);
  }
  return hipGetLastError();
}

}  // namespace hsa
