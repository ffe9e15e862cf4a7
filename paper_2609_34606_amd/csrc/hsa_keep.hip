// Kept tokens: of the tokens that a step drafted behind a sequence, those of an accepted path move to the
// sequence's end, in the pool or in the 8-bit cache:
//
//   token first + i  <-  token first + index[i],  i < count, all read before any is written.
//
// A workgroup owns what it reads and writes (a batch entry's dims of one head, keys or values), so no
// other one can write a token that it still has to read. Bound: a launch's latency.
#include "hsa_fp8.h"
#include "hsa_kernels.h"

namespace hsa {
namespace {

constexpr int kThreads = 256;
// Dims of a workgroup of the pool: 128 bytes of a key row.
template <typename T>
constexpr int kSliceOf = 128 / (int)sizeof(T);

// Slot and place within its page of a sequence's token; false outside the table.
struct TokenPlace {
  size_t slot;
  int off;
};
__device__ __forceinline__ bool place_of(const TokenKeepParams& p, int b, int64_t t, TokenPlace& at) {
  if (t < 0 || t >= (int64_t)p.max_pages * p.P) return false;
  const int page = (int)t / p.P;
  at.off = (int)t - page * p.P;
  at.slot = clampi(p.page_table[(size_t)b * p.max_pages + page], 0, p.num_slots - 1);
  return true;
}

// The pool: a slice of the dims of one head's keys or values. T: an element's bits.
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

// A code in units of another scale, 2^shift of its own.
__device__ __forceinline__ uint8_t recode(uint32_t code, float shift) {
  return (uint8_t)codes2(saturate(code_to_f32(code) * shift, kCodeMax), 0.f, 1.f);
}

// The 8-bit cache: the keys or values of one head. The kept tokens' numbers are appended as
// hsa_cache8_write appends them: a block that begins with them takes the smallest scale that holds
// them, one with older tokens keeps the larger of its own and that. A wave takes a block.
template <int D>
__global__ __launch_bounds__(kThreads) void keep_codes_kernel(TokenKeepParams p) {
  __shared__ __attribute__((aligned(16))) uint8_t buf[HSA_MAX_TREE * D];  // [token][dim]
  __shared__ TokenPlace from[HSA_MAX_TREE];
  __shared__ int16_t exps[HSA_MAX_TREE];     // of the token's block, without the bias
  __shared__ int needs[HSA_MAX_TREE];        // the smallest exponent that holds it
  __shared__ bool ok[HSA_MAX_TREE];
  const int tid = threadIdx.x, lane = tid & 63, b = blockIdx.y, h = blockIdx.x >> 1;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool values = blockIdx.x & 1;
  const int n = p.count ? clampi(p.count[b], 0, p.n) : p.n;
  const int64_t first = p.first ? p.first[b] : 0;
  const int nb = (p.P + kScaleTok - 1) / kScaleTok;
  uint8_t* pool = static_cast<uint8_t*>(values ? p.v : p.k);
  uint8_t* pool_exp = values ? p.v_exp : p.k_exp;
  if (tid < n) {
    TokenPlace to;
    const bool in = place_of(p, b, first + p.index[(size_t)b * p.n + tid], from[tid]);
    ok[tid] = place_of(p, b, first + tid, to) && in;
    exps[tid] = in ? (int16_t)(pool_exp[(from[tid].slot * p.H + h) * nb + from[tid].off / kScaleTok] - 127) : 0;
  }
  __syncthreads();
  if (!values) {
    for (int x = tid; x < n * (D / 16); x += kThreads) {
      const int i = x / (D / 16), c = x % (D / 16);
      if (ok[i])
        *reinterpret_cast<u32x4*>(buf + i * D + 16 * c) =
            ld_global16(pool + ((from[i].slot * p.H + h) * p.P + from[i].off) * D + 16 * c);
    }
  } else {
    for (int x = tid; x < n * D; x += kThreads) {
      const int c = x / n, i = x - c * n;
      if (ok[i]) buf[i * D + c] = pool[((from[i].slot * p.H + h) * D + c) * p.P + from[i].off];
    }
  }
  __syncthreads();
  if (tid < n) {
    uint32_t most = 0;  // largest magnitude, NaN apart
    for (int c = 0; c < D; ++c) {
      const uint32_t m = buf[tid * D + c] & 0x7fu;
      most = m != 0x7fu ? max(most, m) : most;
    }
    needs[tid] = ok[tid] && most ? clampi(scale_exponent(code_to_f32(most)) + exps[tid], kScaleMin, kScaleMax) : kScaleMin;
  }
  __syncthreads();
  // destination blocks: those of tokens [t0, t1) of the table
  const int64_t t0 = first > 0 ? first : 0, cap = (int64_t)p.max_pages * p.P;
  const int64_t t1 = first + n < cap ? first + n : cap;
  if (t0 >= t1) return;
  const int page0 = (int)t0 / p.P, g0 = ((int)t0 - page0 * p.P) / kScaleTok;
  const int page1 = (int)(t1 - 1) / p.P, g1 = ((int)(t1 - 1) - page1 * p.P) / kScaleTok;
  const int blocks = (page1 - page0) * nb + g1 - g0 + 1;
  for (int u = wave; u < blocks; u += kThreads / 64) {
    const int page = page0 + (g0 + u) / nb, blk = (g0 + u) % nb, boff = blk * kScaleTok;
    const int64_t base = (int64_t)page * p.P + boff;
    const int len = min(kScaleTok, p.P - boff);
    const int o0 = t0 > base ? (int)(t0 - base) : 0, o1 = t1 - base < len ? (int)(t1 - base) : len;
    const int i0 = (int)(base + o0 - first), ntok = o1 - o0;
    const size_t slot = clampi(p.page_table[(size_t)b * p.max_pages + page], 0, p.num_slots - 1);
    const size_t head = slot * p.H + h;
    int e = lane < ntok ? needs[i0 + lane] : kScaleMin;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) e = max(e, __shfl_xor(e, m));
    const int e_old = (int)pool_exp[head * nb + blk] - 127;
    if (o0 > 0) e = max(e, e_old);
    if (lane == 0) pool_exp[head * nb + blk] = (uint8_t)(e + 127);
    const bool grow = o0 > 0 && e > e_old;
    const float shift = pow2i(e_old - e);
    const int r0 = grow ? 0 : o0;  // older codes are written again only if the scale grows
    const int rows = o1 - r0;
    for (int x = lane; x < rows * D; x += 64) {
      const int o = r0 + (values ? x % rows : x / D), c = values ? x / rows : x % D;
      uint8_t* dst = pool + (values ? (head * D + c) * p.P + boff + o : (head * p.P + boff + o) * D + c);
      if (o < o0) {
        *dst = recode(*dst, shift);
      } else {
        const int i = i0 + o - o0;
        if (ok[i]) *dst = recode(buf[i * D + c], pow2i(exps[i] - e));
      }
    }
  }
}

}  // namespace

hipError_t launch_token_keep(int dtype, int d, int B, bool eight, const TokenKeepParams& p, hipStream_t s) {
  if (eight) {
    if (d == 128) keep_codes_kernel<128><<<dim3(2 * p.H, B), kThreads, 0, s>>>(p);
    else keep_codes_kernel<64><<<dim3(2 * p.H, B), kThreads, 0, s>>>(p);
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
