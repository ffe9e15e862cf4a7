// Kept tokens: of the tokens that a step drafted behind a sequence, those of an accepted path move to the
// sequence's end, in the pool or in the 8-bit cache:
//
//   token first + i  <-  token first + index[i],  i < count, all read before any is written.
//
// A workgroup owns what it reads and writes (a batch entry's dims of one head, keys or values), so no
// other one can write a token that it still has to read. Bound: a launch's latency, and of long paths the 64-byte pieces
// of memory that single numbers of a value row lie in.
#include "hsa_fp8.h"
#include "hsa_kernels.h"

namespace hsa {
namespace {

constexpr int kThreads = 256;
// Dims of a workgroup of the pool: 128 bytes of a key row.
template <typename T>
constexpr int kSliceOf = 128 / (int)sizeof(T);

// Slot and place within its page of a sequence's token; false outside the table, and if its page has no slot (the place is
// one of the pool all the same).
struct TokenPlace {
  size_t slot;
  int off;
};
__device__ __forceinline__ bool place_of(const TokenKeepParams& p, int b, int64_t t, TokenPlace& at) {
  const bool in = t >= 0 && t < (int64_t)p.max_pages * p.P;
  const int token = in ? (int)t : 0, page = token / p.P;
  at.off = token - page * p.P;
  const int slot = p.page_table[(size_t)b * p.max_pages + page];
  at.slot = clampi(slot, 0, p.num_slots - 1);
  return in & (slot >= 0) & (slot < p.num_slots);
}

// The pool: a slice of the dims of one head's keys or values. T: an element's bits. (32 sequences' paths of up to 8
// tokens, 8 heads, d = 128: 4.7 us, nearly all of it latency.)
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void keep_pool_kernel(TokenKeepParams p) {
  constexpr int kSlice = kSliceOf<T>;
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  T* buf = reinterpret_cast<T*>(smem);  // [n][kSlice] keys, [kSlice][n] values
  __shared__ TokenPlace from[HSA_MAX_TREE], to[HSA_MAX_TREE];
  __shared__ bool ok[HSA_MAX_TREE];
  constexpr int kSlices = D / kSlice;
  const int tid = threadIdx.x, b = blockIdx.y;
  const int slice = blockIdx.x % kSlices, role = blockIdx.x / kSlices, h = role >> 1;
  const bool values = role & 1;
  const int n = p.count ? clampi(p.count[b], 0, p.n) : p.n;
  if (tid < n) {
    const int64_t first = p.first ? p.first[b] : 0;
    const bool in = place_of(p, b, first + p.index[(size_t)b * p.n + tid], from[tid]);
    ok[tid] = place_of(p, b, first + tid, to[tid]) && in;
  }
  __syncthreads();
  if (!values) {
    constexpr int E = 16 / (int)sizeof(T), C = kSlice / E;  // 16-byte pieces of a row
    T* pool = static_cast<T*>(p.k) + slice * kSlice;
    for (int x = tid; x < n * C; x += kThreads) {
      const int i = x / C, c = x % C;
      if (ok[i])
        *reinterpret_cast<u32x4*>(buf + i * kSlice + c * E) =
            ld_global16(pool + ((from[i].slot * p.H + h) * p.P + from[i].off) * D + c * E);
    }
    __syncthreads();
    for (int x = tid; x < n * C; x += kThreads) {
      const int i = x / C, c = x % C;
      if (ok[i])
        *reinterpret_cast<u32x4*>(pool + ((to[i].slot * p.H + h) * p.P + to[i].off) * D + c * E) =
            *reinterpret_cast<const u32x4*>(buf + i * kSlice + c * E);
    }
  } else {
    T* pool = static_cast<T*>(p.v);
    for (int x = tid; x < n * kSlice; x += kThreads) {
      const int c = x / n, i = x - c * n;
      if (ok[i]) buf[x] = pool[((from[i].slot * p.H + h) * D + slice * kSlice + c) * p.P + from[i].off];
    }
    __syncthreads();
    for (int x = tid; x < n * kSlice; x += kThreads) {
      const int c = x / n, i = x - c * n;
      if (ok[i]) pool[((to[i].slot * p.H + h) * D + slice * kSlice + c) * p.P + to[i].off] = buf[x];
    }
  }
}

// Four codes in units of another scale.
__device__ __forceinline__ uint32_t recode4(uint32_t w, float shift) {
  return codes4(saturate(code_to_f32(w & 255u) * shift, kCodeMax), saturate(code_to_f32(w >> 8 & 255u) * shift, kCodeMax),
                saturate(code_to_f32(w >> 16 & 255u) * shift, kCodeMax), saturate(code_to_f32(w >> 24) * shift, kCodeMax), 1.f);
}
__device__ __forceinline__ uint8_t recode(uint32_t code, float shift) {
  return (uint8_t)codes2(saturate(code_to_f32(code) * shift, kCodeMax), 0.f, 1.f);
}
// Magnitudes of four codes, NaN as 0.
__device__ __forceinline__ uint32_t magnitudes(uint32_t w) {
  w &= 0x7f7f7f7fu;
  return w & ~((((w + 0x01010101u) & 0x80808080u) >> 7) * 255u);
}
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {  // of two 16-bit numbers each
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

constexpr int kNoneKept = -1024;  // in the place of a block's exponent
constexpr int kKeepBlocks = HSA_MAX_TREE / 8 + 2;  // scale blocks that a run of tokens touches (pages of 8)

// The 8-bit cache: the keys or values of one head. The kept tokens' numbers are appended as
// hsa_cache8_write appends them: a block that begins with them takes the smallest scale that holds
// them, one with tokens that stay (older ones, and those whose source is no token) the larger of its own and
// that, and one of which none is kept stays as it is. Codes wait in shared memory, keys as [token][dim] in 16-byte
// pieces, values as [dim][token], until every one is there; then they go out, in runs of four where a
// value row has them (64 sequences' paths of up to 100 tokens, 8 heads, d = 128: 17.7 us, 25.8 with the ends of the
// runs in the same loop, where every wave waits for its few lanes that have one; the loads alone take 10).
template <int D>
__global__ __launch_bounds__(kThreads) void keep_codes_kernel(TokenKeepParams p) {
  extern __shared__ __attribute__((aligned(16))) uint8_t buf[];
  __shared__ TokenPlace from[HSA_MAX_TREE];
  __shared__ int exps[HSA_MAX_TREE];      // of the token's block, without the bias
  __shared__ uint32_t most[HSA_MAX_TREE]; // its largest magnitude
  __shared__ bool ok[HSA_MAX_TREE];
  __shared__ uint32_t ok_words[HSA_MAX_TREE / 32 + 1];  // the same as bits
  __shared__ float shifts[HSA_MAX_TREE];  // from its scale to its new block's
  __shared__ int block_e[kKeepBlocks], block_old[kKeepBlocks];
  const int tid = threadIdx.x, lane = tid & 63, b = blockIdx.y, h = blockIdx.x >> 1;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool values = blockIdx.x & 1;
  const int n = p.count ? clampi(p.count[b], 0, p.n) : p.n;
  const int64_t first = p.first ? p.first[b] : 0;
  const int nb = (p.P + kScaleTok - 1) / kScaleTok;
  uint8_t* pool = static_cast<uint8_t*>(values ? p.v : p.k);
  uint8_t* pool_exp = values ? p.v_exp : p.k_exp;
  bool mine = false;
  if (tid <= HSA_MAX_TREE / 32) ok_words[tid] = 0;
  if (tid < n) {
    TokenPlace at, to;
    const bool there = place_of(p, b, first + tid, to);
    mine = place_of(p, b, first + p.index[(size_t)b * p.n + tid], at) & there;
    from[tid] = at;
    ok[tid] = mine;
    exps[tid] = (int)pool_exp[(at.slot * p.H + h) * nb + at.off / kScaleTok] - 127;
    most[tid] = 0;
  }
  __syncthreads();
  const uint64_t all_ok = __ballot(mine);
  if (lane < 2) ok_words[2 * wave + lane] = (uint32_t)(all_ok >> (32 * lane));
  constexpr int C = D / 16;
  if (!values) {
    for (int x = tid; x < n * C; x += kThreads) {
      const int i = x / C, c = x % C;
      if (!ok[i]) continue;
      const u32x4 w = ld_global16(pool + ((from[i].slot * p.H + h) * p.P + from[i].off) * D + 16 * c);
      *reinterpret_cast<u32x4*>(buf + i * D + 16 * c) = w;
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t y = magnitudes(w[j]);
        m = max2(m, max2(y & 0x00ff00ffu, y >> 8 & 0x00ff00ffu));
      }
      atomicMax(most + i, max(m & 0xffffu, m >> 16));
    }
  } else {
    for (int i = lane; i < n; i += 64) {  // a token a lane, every fourth dim a wave
      if (!ok[i]) continue;
      const uint8_t* src = pool + ((from[i].slot * p.H + h) * D + wave) * p.P + from[i].off;
      uint32_t m = 0;
#pragma unroll 8
      for (int c = 0; c < D / 4; ++c) {
        const uint32_t w = src[(size_t)(4 * c) * p.P];
        buf[(wave + 4 * c) * n + i] = (uint8_t)w;
        m = max(m, magnitudes(w));
      }
      atomicMax(most + i, m);
    }
  }
  // destination blocks: those of tokens [t0, t1) of the table
  const int64_t t0 = first > 0 ? first : 0, cap = (int64_t)p.max_pages * p.P;
  const int64_t t1 = first + n < cap ? first + n : cap;
  if (t0 >= t1) return;  // (every thread)
  const int page0 = (int)t0 / p.P, g0 = ((int)t0 - page0 * p.P) / kScaleTok;
  const int page1 = (int)(t1 - 1) / p.P, g1 = ((int)(t1 - 1) - page1 * p.P) / kScaleTok;
  const int blocks = (page1 - page0) * nb + g1 - g0 + 1;
  __syncthreads();
  struct Block {
    size_t head;
    int boff, o0, o1, i0;  // first token in its page; kept tokens [o0, o1) of it, the first of them i0
  };
  auto block_of = [&](int u, int& blk) {
    Block x;
    const int page = page0 + (g0 + u) / nb;
    blk = (g0 + u) % nb;
    x.boff = blk * kScaleTok;
    const int64_t base = (int64_t)page * p.P + x.boff;
    const int len = min(kScaleTok, p.P - x.boff);
    x.o0 = t0 > base ? (int)(t0 - base) : 0;
    x.o1 = t1 - base < len ? (int)(t1 - base) : len;
    x.i0 = (int)(base + x.o0 - first);
    x.head = (size_t)clampi(p.page_table[(size_t)b * p.max_pages + page], 0, p.num_slots - 1) * p.H + h;
    return x;
  };
  // a wave takes a block's scale: a lane a token
  for (int u = wave; u < blocks; u += kThreads / 64) {
    int blk;
    const Block x = block_of(u, blk);
    int e = kScaleMin;
    const bool one = lane < x.o1 - x.o0 && ok[x.i0 + lane];
    if (one) {
      const int i = x.i0 + lane;
      if (most[i]) e = clampi(scale_exponent(code_to_f32(most[i])) + exps[i], kScaleMin, kScaleMax);
    }
    const int kept = __popcll(__ballot(one));
    if (kept == 0) {
      if (lane == 0) block_e[u] = kNoneKept;
      continue;
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) e = max(e, __shfl_xor(e, m));
    uint8_t* at = pool_exp + x.head * nb + blk;
    const int old = (int)*at - 127;
    if (kept < x.o1) e = max(e, old);  // (some of its tokens up to the last one stay)
    if (lane == 0) {
      block_e[u] = e;
      block_old[u] = old;
      *at = (uint8_t)(e + 127);
    }
  }
  __syncthreads();
  if (mine) {
    const int page = (int)(first + tid) / p.P;
    shifts[tid] = pow2i(exps[tid] - block_e[(page - page0) * nb + ((int)(first + tid) - page * p.P) / kScaleTok - g0]);
  }
  __syncthreads();
  for (int u = 0; u < blocks; ++u) {
    int blk;
    const Block x = block_of(u, blk);
    const int e = block_e[u];
    if (e == kNoneKept) continue;
    const float shift = pow2i(block_old[u] - e);
    const bool grows = e > block_old[u];  // then, and only then, codes that stay are written again
    const int r0 = x.o0 > 0 && grows ? 0 : x.o0;
    if (!values) {
      uint8_t* dst = pool + (x.head * p.P + x.boff) * D;
      for (int y = tid; y < (x.o1 - r0) * C; y += kThreads) {
        const int o = r0 + y / C, c = y % C;
        u32x4* at = reinterpret_cast<u32x4*>(dst + o * D + 16 * c);
        const int i = x.i0 + o - x.o0;
        const bool stays = o < x.o0 || !ok[i];
        if (stays && !grows) continue;
        u32x4 w = stays ? *at : *reinterpret_cast<const u32x4*>(buf + i * D + 16 * c);
        const float by = stays ? shift : shifts[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = recode4(w[j], by);
        *at = w;
      }
    } else {
      uint8_t* dst = pool + x.head * D * p.P + x.boff;
      // four tokens of a value row, one by one
      auto some = [&](int c, int o) __attribute__((always_inline)) {
        uint8_t* at = dst + (size_t)c * p.P + o;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int i = x.i0 + o + j - x.o0;
          if (o + j >= x.o0 && o + j < x.o1) {
            if (ok[i]) at[j] = recode(buf[c * n + i], shifts[i]);
            else if (grows) at[j] = recode(at[j], shift);
          } else if (o + j >= r0 && o + j < x.o0) {
            at[j] = recode(at[j], shift);
          }
        }
      };
      // whole runs of four (4-byte aligned: rows of 8 tokens, blocks of 64), then those at the ends and older ones
      const int whole0 = (x.o0 + 3) / 4, whole = max(x.o1 / 4 - whole0, 0), q0 = r0 / 4;
      for (int y = tid; y < whole * D; y += kThreads) {
        const int c = y / whole, o = 4 * (whole0 + y - c * whole), i = x.i0 + o - x.o0;
        const uint64_t bits = (uint64_t)ok_words[(i >> 5) + 1] << 32 | ok_words[i >> 5];
        if ((bits >> (i & 31) & 15u) != 15u) {
          some(c, o);
          continue;
        }
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = saturate(code_to_f32(buf[c * n + i + j]) * shifts[i + j], kCodeMax);
        *reinterpret_cast<uint32_t*>(dst + (size_t)c * p.P + o) = codes4(v[0], v[1], v[2], v[3], 1.f);
      }
      const int before = min(whole0, (x.o1 + 3) / 4) - q0, after = (x.o1 + 3) / 4 - max(whole0 + whole, q0 + before);
      for (int y = tid; y < (before + after) * D; y += kThreads) {
        const int c = y / (before + after), q = y - c * (before + after);
        some(c, 4 * (q < before ? q0 + q : (x.o1 + 3) / 4 - after + q - before));
      }
    }
  }
}

}  // namespace

hipError_t launch_token_keep(int dtype, int d, int B, bool eight, const TokenKeepParams& p, hipStream_t s) {
  if (eight) {
    if (d == 128) keep_codes_kernel<128><<<dim3(2 * p.H, B), kThreads, p.n * 128, s>>>(p);
    else keep_codes_kernel<64><<<dim3(2 * p.H, B), kThreads, p.n * 64, s>>>(p);
    return hipGetLastError();
  }
  const bool half = dtype == HSA_DTYPE_BF16;
  const dim3 grid(2 * p.H * (d / (half ? kSliceOf<uint16_t> : kSliceOf<uint32_t>)), B);
  const size_t lds = (size_t)p.n * 128;
  if (half) {
    if (d == 128) keep_pool_kernel<uint16_t, 128><<<grid, kThreads, lds, s>>>(p);
    else keep_pool_kernel<uint16_t, 64><<<grid, kThreads, lds, s>>>(p);
  } else {
    if (d == 128) keep_pool_kernel<uint32_t, 128><<<grid, kThreads, lds, s>>>(p);
    else keep_pool_kernel<uint32_t, 64><<<grid, kThreads, lds, s>>>(p);
  }
  return hipGetLastError();
}

}  // namespace hsa
