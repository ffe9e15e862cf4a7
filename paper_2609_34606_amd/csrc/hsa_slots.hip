// Page tables on the device: which slots of a pool are free, which are shared, and the copies of pages
// that follow from it. refs[s] counts the table's entries that hold slot s; 0: free. Everything is whole
// numbers, and the order of choices is fixed (rows in order, pages in order, the lowest free slot
// first), so the same tables give the same tables.
#include "hsa_device.h"
#include "hsa_kernels.h"

namespace hsa {
namespace {

constexpr int kPlan = 1024;  // threads of a planning workgroup

// What a workgroup's atomics left in memory (its plain loads may have older copies).
__device__ __forceinline__ int ld_fresh(const int32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Exclusive sum over the workgroup, in thread order; total: the sum of all. Every thread must call it.
__device__ __forceinline__ int scan_all(int x, int* buf, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int sum = x;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int y = __shfl_up(sum, m);
    if (lane >= m) sum += y;
  }
  if (lane == 63) buf[wave] = sum;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kPlan / 64; ++w) {
    const int y = buf[w];
    before += w < wave ? y : 0;
    total += y;
  }
  __syncthreads();
  return before + sum - x;
}

typedef int32_t i32x4a4 __attribute__((ext_vector_type(4), aligned(4)));

// The first `most` slots s with test(refs[s]), ascending, in out; returns how many there are (up to
// `most`). Each thread takes kEach consecutive slots a round.
template <typename Test>
__device__ __forceinline__ int list_slots(const int32_t* refs, int lo, int hi, int most, int32_t* out, int* buf, Test test) {
  constexpr int kEach = 16;
  int found = 0;
  for (int s0 = lo; s0 < hi && found < most; s0 += kPlan * kEach) {
    const int mine = s0 + (int)threadIdx.x * kEach;
    uint32_t on = 0;
    if (mine + kEach <= hi) {
      i32x4a4 r[kEach / 4];
#pragma unroll
      for (int i = 0; i < kEach / 4; ++i) r[i] = *reinterpret_cast<const i32x4a4*>(refs + mine + 4 * i);
#pragma unroll
      for (int i = 0; i < kEach; ++i) on |= (test(r[i >> 2][i & 3]) ? 1u : 0u) << i;
    } else {
      for (int i = 0; mine + i < hi; ++i) on |= (test(refs[mine + i]) ? 1u : 0u) << i;
    }
    int total;
    int at = found + scan_all(__popc(on), buf, total);
    for (; on; on &= on - 1, ++at)
      if (at < most) out[at] = mine + __builtin_ctz(on);
    found += total;
  }
  return min(found, most);
}

// ---------------------------------------------------------------- take
// Pages of a row that hold its tokens [first, end).
struct RowPages {
  int lo, n, inside;  // inside: tokens of the first page before `first`
};
__device__ __forceinline__ RowPages row_pages(const SlotsParams& p, int b) {
  RowPages r;
  const int first = p.first ? max(p.first[b], 0) : 0, end = p.end[b];
  r.lo = first / p.P;
  r.inside = first - r.lo * p.P;
  const int hi = min((int)(((int64_t)end + p.P - 1) / p.P), p.max_pages);
  r.n = end > first ? max(hi - r.lo, 0) : 0;
  return r;
}

// An entry gets a slot of its own in the place of `was`. lead: it is the row's first wanted one.
__device__ __forceinline__ void take_slot(const SlotsParams& p, int b, int page, int was, int now, bool lead) {
  p.page_table[(size_t)b * p.max_pages + page] = now;
  p.refs[now] = 1;
  if (was < 0) return;
  atomicSub(p.refs + was, 1);
  const RowPages r = row_pages(p, b);
  if (p.moves && lead && r.inside > 0) {
    p.moves[3 * b] = was;
    p.moves[3 * b + 1] = now;
    p.moves[3 * b + 2] = r.inside;
  }
}

// Small tables: one workgroup. The wanted entries of all rows are numbered in order, kEach a thread, 1024 apart, and
// stay in registers; what is shared is counted before anything changes. ws: wanting entries and the last of them for each
// slot, the free slots. Bound: a launch, and a few loads and sums of the workgroup that wait for each other (64
// rows of 16 pages, a page each that most rows share: 8.4 us). In us, this way and the other, rows times pages all
// wanted: 64 x 16 8.6 and 15.7, 256 x 16 17.6 and 16.7, 16 x 256 16.2 and 16.3, 4096 x 1 21.8 and 26.9.
constexpr int kSmallTable = 4 * kPlan;
__global__ __launch_bounds__(kPlan) void slots_take_kernel(SlotsParams p) {
  constexpr int kEach = kSmallTable / kPlan, kWaves = kPlan / 64;
  __shared__ int starts[kSmallTable + 1];  // number of a row's first wanted entry
  __shared__ int pages[kSmallTable];       // its page, less that number
  __shared__ int buf[kWaves];
  __shared__ int counts[kEach * kWaves];   // entries in need, of each wave and step; sums before it
  __shared__ int any_shared;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int32_t* wants = p.ws;
  int32_t* last = wants + p.num_slots;
  int32_t* free_slots = last + p.num_slots;
  if (tid == 0) any_shared = 0;
  int n = 0;  // wanted entries
  for (int b0 = 0; b0 < p.B; b0 += kPlan) {
    int total;
    const int b = b0 + tid;
    const RowPages r = b < p.B ? row_pages(p, b) : RowPages{0, 0, 0};
    const int at = n + scan_all(r.n, buf, total);
    if (b < p.B) {
      starts[b] = at;
      pages[b] = r.lo - at;
    }
    n += total;
  }
  if (tid == 0) starts[p.B] = n;
  __syncthreads();
  // the entries 1024 j + tid: rows, slots (INT32_MAX: no entry), and how many entries hold them (0: none, or
  // past the pool)
  int row[kEach], slot[kEach], refs[kEach];
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const int x = kPlan * j + tid;
    slot[j] = INT32_MAX;
    row[j] = 0;
    if (x < n) {
      int lo = 0, hi = p.B;  // the last row that starts at or before x
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid] <= x) lo = mid;
        else hi = mid;
      }
      row[j] = lo;
      slot[j] = p.page_table[(size_t)lo * p.max_pages + x + pages[lo]];
    }
  }
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    refs[j] = slot[j] >= 0 && slot[j] < p.num_slots ? p.refs[slot[j]] : 0;
    if (refs[j] > 1) {
      wants[slot[j]] = 0;
      last[slot[j]] = -1;
      any_shared = 1;
    }
  }
  __syncthreads();
  if (any_shared) {
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      if (refs[j] > 1) {
        atomicAdd(wants + slot[j], 1);
        atomicMax(last + slot[j], kPlan * j + tid);
      }
    __syncthreads();
  }
  // An entry needs a slot if it has none, or shares one: but the last of the entries that hold it, if
  // all of them want it, keeps it.
  uint32_t need = 0;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    bool is = slot[j] < 0;
    if (refs[j] > 1) is = !(ld_fresh(wants + slot[j]) == refs[j] && ld_fresh(last + slot[j]) == kPlan * j + tid);
    need |= (is ? 1u : 0u) << j;
    const uint64_t all = __ballot(is);
    if (lane == 0) counts[j * kWaves + wave] = __popcll(all);
  }
  __syncthreads();
  int needs;
  const int before = scan_all(tid < kEach * kWaves ? counts[tid] : 0, buf, needs);
  if (tid < kEach * kWaves) counts[tid] = before;
  const int n_free = list_slots(p.refs, 0, p.num_slots, needs, free_slots, buf, [](int r) { return r == 0; });
  if (p.moves)
    for (int x = tid; x < 3 * p.B; x += kPlan) p.moves[x] = -1;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const bool is = need >> j & 1u;
    const uint64_t all = __ballot(is);
    const int rank = counts[j * kWaves + wave] + __popcll(all & ((1ull << lane) - 1));
    if (is && rank < n_free) {
      const int x = kPlan * j + tid;
      take_slot(p, row[j], x + pages[row[j]], slot[j], free_slots[rank], x == starts[row[j]]);
    }
  }
  if (p.missing && tid == 0) *p.missing = needs - n_free;
}

// Larger tables, in four launches: a row of the table or 4096 slots a workgroup. ws: as above, an entry's rank
// among those of its row that get a slot, a row's number of them, free slots of each 4096. Bound: four launches' latency
// (128 rows of 512 pages, 32768 slots: 21 us together with the release before; one workgroup took 58).
constexpr int kRow = 256, kPerChunk = 4096;
struct TakeWs {
  int32_t *wants, *last, *free_slots, *ranks, *row_needs, *chunk_free;
  int chunks;
};
__host__ __device__ __forceinline__ TakeWs take_ws(const SlotsParams& p) {
  TakeWs w;
  w.wants = p.ws;
  w.last = w.wants + p.num_slots;
  w.free_slots = w.last + p.num_slots;
  w.ranks = w.free_slots + p.num_slots;
  w.row_needs = w.ranks + (size_t)p.B * p.max_pages;
  w.chunk_free = w.row_needs + p.B;
  w.chunks = (p.num_slots + kPerChunk - 1) / kPerChunk;
  return w;
}
// Sum over the workgroup of kRow threads. Every thread must call it.
__device__ __forceinline__ int sum_row(int x, int* buf) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) x += __shfl_xor(x, m);
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = x;
  __syncthreads();
  const int total = buf[0] + buf[1] + buf[2] + buf[3];
  __syncthreads();
  return total;
}
// Numbers of set flags in the threads before this one; total: of all.
__device__ __forceinline__ int rank_row(bool is, int* buf, int& total) {
  const uint64_t all = __ballot(is);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (lane == 0) buf[wave] = __popcll(all);
  __syncthreads();
  int before = __popcll(all & ((1ull << lane) - 1));
  total = 0;
#pragma unroll
  for (int w = 0; w < kRow / 64; ++w) {
    before += w < wave ? buf[w] : 0;
    total += buf[w];
  }
  __syncthreads();
  return before;
}

__global__ __launch_bounds__(kRow) void take_clear_kernel(SlotsParams p) {
  __shared__ int buf[kRow / 64];
  const TakeWs w = take_ws(p);
  const int s0 = blockIdx.x * kPerChunk, hi = min(s0 + kPerChunk, p.num_slots);
  int free = 0;
  for (int s = s0 + threadIdx.x; s < hi; s += kRow) {
    w.wants[s] = 0;
    w.last[s] = -1;
    free += p.refs[s] == 0;
  }
  free = sum_row(free, buf);
  if (threadIdx.x == 0) w.chunk_free[blockIdx.x] = free;
}
__global__ __launch_bounds__(kRow) void take_count_kernel(SlotsParams p) {
  const TakeWs w = take_ws(p);
  const int b = blockIdx.x;
  const RowPages r = row_pages(p, b);
  for (int i = threadIdx.x; i < r.n; i += kRow) {
    const int at = b * p.max_pages + r.lo + i, slot = p.page_table[at];  // (a table has at most 2^30 entries)
    if (slot >= 0 && slot < p.num_slots && p.refs[slot] > 1) {
      atomicAdd(w.wants + slot, 1);
      atomicMax(w.last + slot, at);
    }
  }
}
__global__ __launch_bounds__(kRow) void take_decide_kernel(SlotsParams p) {
  __shared__ int buf[kRow / 64];
  const TakeWs w = take_ws(p);
  const int tid = threadIdx.x;
  if ((int)blockIdx.x < p.B) {
    const int b = blockIdx.x;
    const RowPages r = row_pages(p, b);
    int needs = 0;
    for (int i0 = 0; i0 < r.n; i0 += kRow) {
      const int at = b * p.max_pages + r.lo + i0 + tid;
      bool is = false;
      if (i0 + tid < r.n) {
        const int slot = p.page_table[at], refs = slot >= 0 && slot < p.num_slots ? p.refs[slot] : 0;
        is = slot < 0 || (refs > 1 && !(w.wants[slot] == refs && w.last[slot] == at));
      }
      int total;
      const int rank = rank_row(is, buf, total);
      if (i0 + tid < r.n) w.ranks[at] = is ? needs + rank : -1;
      needs += total;
    }
    if (tid == 0) w.row_needs[b] = needs;
    return;
  }
  // the free slots of a chunk, behind those of the chunks before it
  const int c = blockIdx.x - p.B;
  int before = 0;
  for (int x = tid; x < c; x += kRow) before += w.chunk_free[x];
  before = sum_row(before, buf);
  const int hi = min((c + 1) * kPerChunk, p.num_slots);
  for (int s0 = c * kPerChunk; s0 < hi; s0 += kRow) {
    int total;
    const bool is = s0 + tid < hi && p.refs[s0 + tid] == 0;
    const int rank = rank_row(is, buf, total);
    if (is) w.free_slots[before + rank] = s0 + tid;
    before += total;
  }
}
__global__ __launch_bounds__(kRow) void take_apply_kernel(SlotsParams p) {
  __shared__ int buf[kRow / 64];
  const TakeWs w = take_ws(p);
  const int b = blockIdx.x, tid = threadIdx.x;
  const RowPages r = row_pages(p, b);
  int before = 0, n_free = 0;
  for (int x = tid; x < b; x += kRow) before += w.row_needs[x];
  for (int x = tid; x < w.chunks; x += kRow) n_free += w.chunk_free[x];
  before = sum_row(before, buf);
  n_free = sum_row(n_free, buf);
  if (p.moves && tid < 3) p.moves[3 * b + tid] = -1;
  __syncthreads();
  for (int i = tid; i < r.n; i += kRow) {
    const int at = b * p.max_pages + r.lo + i, rank = w.ranks[at];
    if (rank >= 0 && before + rank < n_free)
      take_slot(p, b, r.lo + i, p.page_table[at], w.free_slots[before + rank], i == 0);
  }
  if (p.missing && b == p.B - 1 && tid == 0) *p.missing = max(before + w.row_needs[b] - n_free, 0);
}

// ---------------------------------------------------------------- fork, free
__device__ __forceinline__ int parent_of(const SlotsParams& p, int b) {
  const int x = p.parent[b];
  return x >= 0 && x < p.B ? x : b;
}

// The new rows go to ws first: a row may be the parent of one and the child of another. Bound: two launches
// (64 rows of 16 pages 2.3 us each).
__global__ __launch_bounds__(256) void slots_fork_kernel(SlotsParams p) {
  const int b = blockIdx.y, page = blockIdx.x * 256 + threadIdx.x;
  const int from = parent_of(p, b);
  if (page >= p.max_pages || from == b) return;
  const int was = p.page_table[(size_t)b * p.max_pages + page], now = p.page_table[(size_t)from * p.max_pages + page];
  p.ws[(size_t)b * p.max_pages + page] = now;
  if (was == now) return;
  if (was >= 0 && was < p.num_slots) atomicSub(p.refs + was, 1);
  if (now >= 0 && now < p.num_slots) atomicAdd(p.refs + now, 1);
}
__global__ __launch_bounds__(256) void slots_forked_kernel(SlotsParams p) {
  const int b = blockIdx.y, page = blockIdx.x * 256 + threadIdx.x;
  if (page >= p.max_pages || parent_of(p, b) == b) return;
  p.page_table[(size_t)b * p.max_pages + page] = p.ws[(size_t)b * p.max_pages + page];
}

// Bound: a launch (128 rows of 512 pages: 2.7 us).
__global__ __launch_bounds__(256) void slots_free_kernel(SlotsParams p) {
  const int b = blockIdx.y, page = blockIdx.x * 256 + threadIdx.x;
  const int keep = p.end[b];
  if (page >= p.max_pages || keep < 0 || (int64_t)page * p.P < keep) return;
  int32_t* at = p.page_table + (size_t)b * p.max_pages + page;
  const int slot = *at;
  if (slot >= 0 && slot < p.num_slots) atomicSub(p.refs + slot, 1);
  *at = -1;
}

// ---------------------------------------------------------------- compact
// One workgroup: the slots in use behind the n-th (n: slots in use), in order, go to the free ones before
// it, in order. ws: where each slot goes, its count then, the holes, the slots that move. Bound: the workgroup's reads of
// the counts, one after another (1500 slots: 8.1 us, and 4.7 for the tables).
__global__ __launch_bounds__(kPlan) void slots_compact_kernel(SlotsParams p) {
  __shared__ int buf[kPlan / 64];
  const int tid = threadIdx.x;
  int32_t* to = p.ws;
  int32_t* refs = to + p.num_slots;
  int32_t* holes = refs + p.num_slots;
  int32_t* movers = holes + p.num_slots;
  int mine = 0, live;
  for (int s = tid; s < p.num_slots; s += kPlan) {
    const int r = p.refs[s];
    to[s] = s;
    refs[s] = r;
    mine += r > 0;
  }
  scan_all(mine, buf, live);
  const int n = list_slots(p.refs, 0, live, p.n_moves, holes, buf, [](int r) { return r <= 0; });
  list_slots(p.refs, live, p.num_slots, p.n_moves, movers, buf, [](int r) { return r > 0; });
  __syncthreads();
  for (int i = tid; i < p.n_moves; i += kPlan) {
    const bool is = i < n;
    const int src = is ? movers[i] : -1, dst = is ? holes[i] : -1;
    p.moves[3 * i] = src;
    p.moves[3 * i + 1] = dst;
    p.moves[3 * i + 2] = is ? p.P : -1;
    if (is) {
      to[src] = dst;
      refs[dst] = p.refs[src];
      refs[src] = 0;
    }
  }
}
__global__ __launch_bounds__(256) void slots_compacted_kernel(SlotsParams p) {
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x, entries = (int64_t)p.B * p.max_pages;
  if (x < entries) {
    const int slot = p.page_table[x];
    p.table_out[x] = slot >= 0 && slot < p.num_slots ? p.ws[slot] : slot;
  }
  if (x < p.num_slots) p.refs_out[x] = p.ws[p.num_slots + x];
}

// ---------------------------------------------------------------- copies
constexpr int kCopyBytes = 32768;  // of a workgroup

// Pages slot to slot: moves[i] = {from, to, tokens}. A whole page is one run of bytes for its keys and one for
// its values; of a part, the rows of its first tokens (up to eight more than asked for, whole granules).
// Bound: HBM (371 pages of 256 tokens of 8 heads of the 8-bit cache, 389 MB read and written: 67 to 81 us, 5.8 to 4.8
// TB/s; parts of 64 pages of bf16, 33 MB, 10 to 11 us).
__global__ __launch_bounds__(256) void page_copy_kernel(PageCopyParams p, int parts) {
  const int move = blockIdx.x / parts, part = blockIdx.x - move * parts, tid = threadIdx.x;
  const int src = p.moves[3 * move], dst = p.moves[3 * move + 1];
  const int tokens = (clampi(p.moves[3 * move + 2], 0, p.P) + 7) & ~7;  // (P is a multiple of 8)
  if (src < 0 || dst < 0 || src >= p.num_slots || dst >= p.num_slots || src == dst || tokens == 0) return;
  const size_t slot = (size_t)p.H * p.P * p.d * p.size;  // bytes
  const uint8_t* ks = static_cast<const uint8_t*>(p.k) + src * slot;
  const uint8_t* vs = static_cast<const uint8_t*>(p.v) + src * slot;
  uint8_t* kd = static_cast<uint8_t*>(p.k) + dst * slot;
  uint8_t* vd = static_cast<uint8_t*>(p.v) + dst * slot;
  const int half = parts / 2;
  const bool values = part >= half;
  const int at = values ? part - half : part;
  const int64_t lo = (int64_t)at * kCopyBytes;
  if (tokens == p.P) {
    const int64_t hi = lo + kCopyBytes < (int64_t)slot ? lo + kCopyBytes : (int64_t)slot;
    const uint8_t* s = values ? vs : ks;
    uint8_t* d = values ? vd : kd;
    for (int64_t x = lo + 16 * tid; x < hi; x += 16 * 256) *reinterpret_cast<u32x4*>(d + x) = ld_global16(s + x);
  } else if (!values) {
    const int64_t row = (int64_t)tokens * p.d * p.size, all = row * p.H, page = (int64_t)p.P * p.d * p.size;
    const int64_t hi = lo + kCopyBytes < all ? lo + kCopyBytes : all;
    for (int64_t x = lo + 16 * tid; x < hi; x += 16 * 256) {
      const int64_t o = x / row * page + x % row;
      *reinterpret_cast<u32x4*>(kd + o) = ld_global16(ks + o);
    }
  } else {
    // eight tokens of a value row: 8, 16 or 32 bytes
    const int64_t row = (int64_t)tokens * p.size, all = row * p.d * p.H, page = (int64_t)p.P * p.size;
    const int64_t hi = lo + kCopyBytes < all ? lo + kCopyBytes : all;
    for (int64_t x = lo + 8 * tid; x < hi; x += 8 * 256) {
      const int64_t o = x / row * page + x % row;
      *reinterpret_cast<u32x2*>(vd + o) = *reinterpret_cast<const u32x2*>(vs + o);
    }
  }
  if (part == 0 && p.k_exp) {
    const int nb = (p.P + HSA_CACHE8_BLOCK - 1) / HSA_CACHE8_BLOCK, n = (tokens + HSA_CACHE8_BLOCK - 1) / HSA_CACHE8_BLOCK;
    for (int x = tid; x < p.H * n; x += 256) {
      const size_t o = (size_t)(x / n) * nb + x % n, a = (size_t)src * p.H * nb + o, c = (size_t)dst * p.H * nb + o;
      p.k_exp[c] = p.k_exp[a];
      p.v_exp[c] = p.v_exp[a];
    }
  }
}

}  // namespace

size_t slots_take_ints(const SlotsParams& p) {
  const TakeWs w = take_ws(p);
  return 3 * (size_t)p.num_slots + (size_t)p.B * p.max_pages + p.B + w.chunks;
}
size_t slots_fork_ints(const SlotsParams& p) { return (size_t)p.B * p.max_pages; }
size_t slots_compact_ints(const SlotsParams& p) { return 4 * (size_t)p.num_slots; }

hipError_t launch_slots_take(const SlotsParams& p, hipStream_t s) {
  if ((int64_t)p.B * p.max_pages <= kSmallTable) {
    slots_take_kernel<<<1, kPlan, 0, s>>>(p);
  } else {
    const int chunks = take_ws(p).chunks;
    take_clear_kernel<<<chunks, kRow, 0, s>>>(p);
    take_count_kernel<<<p.B, kRow, 0, s>>>(p);
    take_decide_kernel<<<p.B + chunks, kRow, 0, s>>>(p);
    take_apply_kernel<<<p.B, kRow, 0, s>>>(p);
  }
  return hipGetLastError();
}

hipError_t launch_slots_fork(const SlotsParams& p, hipStream_t s) {
  const dim3 grid((p.max_pages + 255) / 256, p.B);
  slots_fork_kernel<<<grid, 256, 0, s>>>(p);
  slots_forked_kernel<<<grid, 256, 0, s>>>(p);
  return hipGetLastError();
}

hipError_t launch_slots_free(const SlotsParams& p, hipStream_t s) {
  slots_free_kernel<<<dim3((p.max_pages + 255) / 256, p.B), 256, 0, s>>>(p);
  return hipGetLastError();
}

hipError_t launch_slots_compact(const SlotsParams& p, hipStream_t s) {
  slots_compact_kernel<<<1, kPlan, 0, s>>>(p);
  const int64_t entries = (int64_t)p.B * p.max_pages, n = entries > p.num_slots ? entries : p.num_slots;
  slots_compacted_kernel<<<(uint32_t)((n + 255) / 256), 256, 0, s>>>(p);
  return hipGetLastError();
}

int64_t page_copy_parts(const PageCopyParams& p) {
  const int64_t slot = (int64_t)p.H * p.P * p.d * p.size;
  return 2 * ((slot + kCopyBytes - 1) / kCopyBytes);
}

hipError_t launch_page_copy(const PageCopyParams& p, hipStream_t s) {
  const int64_t parts = page_copy_parts(p);
  page_copy_kernel<<<(uint32_t)(parts * p.n), 256, 0, s>>>(p, (int)parts);
  return hipGetLastError();
}

}  // namespace hsa
