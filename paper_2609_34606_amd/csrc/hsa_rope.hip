// Rotary positions (queries, or keys outside a cache): pair i of a head is
// turned by the angle position * frequency_i.
//
// Every element is read and written once, so the launch is bound by memory (by
// its own latency for few tokens). The angle's cosine and sine cost about 35 instructions
// a pair; a thread computes those of one item (rope_mode) of a token once and
// applies them to kHeads heads, whose loads are in flight together. Neighbouring
// lanes take neighbouring 16-byte pieces of a head. 4680 tokens, 12 heads x d128 in bf16, out
// of a fused projection: 7.2 us, 4.0 TB/s (a 1 GiB copy 5.1); one token 2.5 us.
#include <math.h>

#include "hsa_rope.h"

namespace hsa {
namespace {

template <typename T, int kMode, int kHeads>
__global__ __launch_bounds__(256) void rope_kernel(RopeParams p) {
  using Item = RopeItem<T, kMode>;
  const RopeTable& r = p.table;
  const uint32_t id = blockIdx.x * 256u + threadIdx.x;
  const uint32_t row = id / p.n_items;                 // (token, head group)
  const uint32_t tok = row / p.n_groups;
  if (tok >= (uint32_t)p.n) return;
  const int t = (int)tok, h0 = (int)(row - tok * p.n_groups) * kHeads, b = blockIdx.y;
  Item it;
  it.set(r, (int)(id - row * p.n_items));
  const T* x = static_cast<const T*>(p.x) + (int64_t)b * p.x_batch + (int64_t)t * p.x_token;
  T* o = static_cast<T*>(p.o) + (int64_t)b * p.o_batch + (int64_t)t * p.o_token;
  typename Item::El::Raw ra[kHeads], rb[kHeads];
#pragma unroll
  for (int k = 0; k < kHeads; ++k) it.load(x + min(h0 + k, p.heads - 1) * p.d, ra[k], rb[k]);
  it.frequencies(r);
  float c[Item::NP], s[Item::NP];
  it.angles(r, rope_positions(r, b, t, p.n), c, s);
#pragma unroll
  for (int k = 0; k < kHeads; ++k) {
    if (h0 + k < p.heads) {
      float u[Item::N], v[Item::N];
      it.result(ra[k], rb[k], c, s, u, v);
      it.store(o + (h0 + k) * p.d, u, v);
    }
  }
}

template <typename T, int kMode>
hipError_t launch(RopeParams p, int B, hipStream_t s) {
  p.n_items = RopeItem<T, kMode>::count(p.table.rot, p.d);
  // Two heads a thread share its angles, once that leaves a wave a SIMD (12 heads x d128,
  // 4680 tokens, interleaved: one head 9.0 us, two 7.3, four 7.4; 300 tokens: 3.5, 3.6, 3.8).
  const int k = p.heads >= 2 && (int64_t)B * p.n * p.n_items * ((p.heads + 1) / 2) >= 65536 ? 2 : 1;
  p.n_groups = (p.heads + k - 1) / k;
  const int64_t threads = (int64_t)p.n * p.n_groups * p.n_items;
  const dim3 grid((uint32_t)((threads + 255) / 256), B);
  if (k == 2) rope_kernel<T, kMode, 2><<<grid, 256, 0, s>>>(p);
  else rope_kernel<T, kMode, 1><<<grid, 256, 0, s>>>(p);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_as(const RopeParams& p, int B, hipStream_t s) {
  switch (rope_mode<T>(p.table, p.d)) {
    case kRopeHalves:
    case kRopePart: return launch<T, kRopePart>(p, B, s);
    case kRopeInterleaved: return launch<T, kRopeInterleaved>(p, B, s);
    default: return launch<T, kRopeSingle>(p, B, s);
  }
}

}  // namespace

hipError_t launch_rope(int dtype, int B, const RopeParams& p, hipStream_t s) {
  return dtype == HSA_DTYPE_BF16 ? launch_as<uint16_t>(p, B, s) : launch_as<float>(p, B, s);
}

bool rope_table(const hsa_rope_t* r, int d, bool inverse, const int32_t* pos, const int32_t* first, RopeTable& t) {
  constexpr double kTau = 6.28318530717958647692;
  // Quarter turns a position: 2^31 positions then stay below 2^50, where fp64 still holds the
  // fraction of a quarter that cos_sin_quarters takes off.
  constexpr double kMostQuarters = 524288.0;
  if (r->rot_dim < 2 || r->rot_dim > d || r->rot_dim % 2) return false;
  if (r->layout != HSA_ROPE_HALF && r->layout != HSA_ROPE_INTERLEAVED) return false;
  if (r->axes < 1 || r->axes > 3 || (r->axes > 1 && !pos)) return false;
  int dims[3] = {r->rot_dim, 0, 0}, sum = 0;
  if (r->axes > 1)
    for (int a = 0; a < r->axes; ++a) {
      dims[a] = r->axis_dim[a];
      if (dims[a] < 2 || dims[a] % 2 || dims[a] > r->rot_dim) return false;
      sum += dims[a];
    }
  if (r->axes > 1 && sum != r->rot_dim) return false;
  if (!(r->theta > 0.0) || isinf(r->theta) || !isfinite((float)r->amplitude)) return false;
  if (r->scaling != HSA_ROPE_UNSCALED && (!(r->factor > 0.0) || isinf(r->factor))) return false;
  if (r->scaling == HSA_ROPE_PARTS) {
    if (!(r->low >= 0.0) || !(r->high > r->low) || isinf(r->high) || r->orig_len < 1) return false;
  } else if (r->scaling != HSA_ROPE_UNSCALED && r->scaling != HSA_ROPE_LINEAR) {
    return false;
  }
  int i = 0;
  for (int a = 0; a < r->axes; ++a) {
    // The powers by repeated products in 80 bits, 64 of them significant: 63 products lose at
    // most six, and the rounding to fp64 is as exact as pow()'s, in a tenth of its time.
    const long double ratio = powl(r->theta, -2.0L / dims[a]);
    long double power = 1.0L;
    for (int k = 0; k < dims[a] / 2; ++k, ++i, power *= ratio) {
      double f = (double)power;
      if (r->scaling == HSA_ROPE_LINEAR) {
        f /= r->factor;
      } else if (r->scaling == HSA_ROPE_PARTS) {
        const double turns = r->orig_len * f / kTau;
        double w = (turns - r->low) / (r->high - r->low);
        w = w < 0.0 ? 0.0 : (w > 1.0 ? 1.0 : w);
        f = w * f + (1.0 - w) * f / r->factor;
      }
      t.quarters[i] = 4.0 * (inverse ? -f : f) / kTau;
      if (!(fabs(t.quarters[i]) <= kMostQuarters)) return false;
      t.axis[i] = (int8_t)a;
    }
  }
  t.rot = r->rot_dim;
  t.layout = r->layout;
  t.axes = r->axes;
  t.amplitude = r->amplitude == 0.0 ? 1.f : (float)r->amplitude;
  t.pos = pos;
  t.first = first;
  return true;
}

}  // namespace hsa
