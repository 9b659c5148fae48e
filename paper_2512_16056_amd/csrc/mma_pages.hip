// Pages of the cache for gfx950 (MI355X): sequences that go on from others (fork) and held pages moved together
// (compact). Both first decide which page goes where, over counts and tables of some ten thousand words, and then
// copy pages in every layer. The decisions depend on each other in order (the k-th request for a page gets the k-th
// free one), so one workgroup makes them, with few barriers; the copies are bound by HBM.
#include "mma_ops.h"

namespace mma {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kWide = 1024;                 // threads of a workgroup that decides
constexpr uint32_t kWaves = kWide / kOpsWave;
constexpr uint32_t kCopy = 16384;                // bytes that a workgroup copies at once

// Words that other workgroups or waves change within the kernel: past the L1 cache.
__device__ __forceinline__ int32_t look(const int32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void put(int32_t* p, int32_t v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Exclusive sum of a value over the workgroup's threads; *total of all of them.
__device__ __forceinline__ uint32_t before_mine(uint32_t v, uint32_t* waves, uint32_t* total) {
  const uint32_t lane = threadIdx.x % kOpsWave, wave = threadIdx.x / kOpsWave;
  uint32_t up = v;
#pragma unroll
  for (int x = 1; x < kOpsWave; x *= 2) {
    const uint32_t y = __shfl_up(up, x, kOpsWave);
    if (lane >= static_cast<uint32_t>(x)) up += y;
  }
  __syncthreads();
  if (lane == kOpsWave - 1) waves[wave] = up;
  __syncthreads();
  uint32_t sum = 0, mine = 0;
  for (uint32_t w = 0; w < kWaves; ++w) {
    if (w == wave) mine = sum;
    sum += waves[w];
  }
  *total = sum;
  return mine + up - v;
}

// ---------------------------------------------------------------- fork
// What sequence `parent` hands on: its entries, of which `full` blocks are whole.
struct Child {
  uint32_t entries, full;
  int32_t parent;  // -1: none
};

__device__ __forceinline__ Child child_of(const ForkArgs& a, uint32_t i) {
  Child c{0, 0, a.parents[i]};
  if (c.parent < 0 || static_cast<uint32_t>(c.parent) >= a.num_seqs) {
    c.parent = -1;
    return c;
  }
  const int32_t n = a.lens[c.parent];
  c.entries = n < 0 ? 0 : static_cast<uint32_t>(n) < a.max_len ? n : a.max_len;
  c.full = c.entries / a.tokens;
  return c;
}

// Places of a child: its entries' and those for the tokens to come.
__device__ __forceinline__ uint32_t places_of(const ForkArgs& a, const Child& c, uint32_t i) {
  const int32_t g = a.grow ? a.grow[i] : 0;
  const uint64_t n = (static_cast<uint64_t>(c.entries) + (g < 0 ? 0 : g) + a.tokens - 1) / a.tokens;
  return n < a.out_stride ? static_cast<uint32_t>(n) : a.out_stride;
}

__global__ __launch_bounds__(256) void fork_counts_kernel(ForkArgs a) {
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  if (i < a.num_blocks) a.refs_out[i] = a.refs[i];
}

// One row a workgroup: a sequence's, whose places' counts change by its children, or a child's, which takes over its
// parent's whole blocks and has no others yet.
__global__ __launch_bounds__(256) void fork_rows_kernel(ForkArgs a) {
  __shared__ uint32_t children;
  if (blockIdx.x < a.num_seqs) {
    const uint32_t seq = blockIdx.x;
    if (!threadIdx.x) children = 0;
    __syncthreads();
    uint32_t n = 0;
    for (uint32_t i = threadIdx.x; i < a.num_children; i += 256) n += a.parents[i] == static_cast<int32_t>(seq) ? 1 : 0;
    if (n) atomicAdd(&children, n);
    __syncthreads();
    const int32_t len = a.lens[seq];
    const uint32_t entries = len < 0 ? 0 : static_cast<uint32_t>(len) < a.max_len ? len : a.max_len, full = entries / a.tokens;
    const int32_t* row = a.table + static_cast<uint64_t>(seq) * a.table_stride;
    for (uint32_t j = threadIdx.x; j < a.table_stride; j += 256) {
      const int32_t id = row[j], by = static_cast<int32_t>(j < full ? children : 0) - 1;
      if (by && static_cast<uint32_t>(id) < a.num_blocks) atomicAdd(a.refs_out + id, by);
    }
  } else {
    const uint32_t i = blockIdx.x - a.num_seqs;
    const Child c = child_of(a, i);
    if (!threadIdx.x) a.lens_out[i] = static_cast<int32_t>(c.entries);
    const int32_t* from = a.table + static_cast<uint64_t>(c.parent < 0 ? 0 : c.parent) * a.table_stride;
    int32_t* to = a.table_out + static_cast<uint64_t>(i) * a.out_stride;
    for (uint32_t j = threadIdx.x; j < a.out_stride; j += 256) {
      int32_t id = -1;
      if (c.parent >= 0 && j < c.full) {
        id = from[j];
        if (static_cast<uint32_t>(id) >= a.num_blocks) id = -1;
      }
      to[j] = id;
    }
  }
}

// The open blocks and the new ones. A block that is open for some children and held by nothing else goes to the first of
// them: each puts the lowest number in the block's own count, below every count that there is.
__global__ __launch_bounds__(kWide) void fork_give_kernel(ForkArgs a) {
  __shared__ uint32_t waves[kWaves], free_before[kWaves];
  const uint32_t t = threadIdx.x, lane = t % kOpsWave, wave = t / kOpsWave;
  const auto open_block = [&](uint32_t i, const Child& c) -> int32_t {  // or -1
    if (c.entries == c.full * a.tokens) return -1;
    const int32_t id = a.table[static_cast<uint64_t>(c.parent) * a.table_stride + c.full];
    return static_cast<uint32_t>(id) < a.num_blocks ? id : -1;
  };
  for (uint32_t i = t; i < a.num_children; i += kWide) {
    const int32_t id = open_block(i, child_of(a, i));
    a.from[i] = id >= 0 && look(a.refs_out + id) == 0 ? id : -1;  // for now: what it may keep
  }
  __syncthreads();
  for (uint32_t i = t; i < a.num_children; i += kWide)
    if (a.from[i] >= 0) atomicMin(a.refs_out + a.from[i], INT32_MIN + static_cast<int32_t>(i));
  __syncthreads();
  uint32_t need = 0;  // of all children before this round's
  for (uint32_t first = 0; first < a.num_children; first += kWide) {
    const uint32_t i = first + t;
    uint32_t wants = 0;
    if (i < a.num_children) {
      const Child c = child_of(a, i);
      const int32_t id = open_block(i, c);
      const bool keeps = a.from[i] >= 0 && look(a.refs_out + id) == INT32_MIN + static_cast<int32_t>(i);
      if (keeps) a.table_out[static_cast<uint64_t>(i) * a.out_stride + c.full] = id;
      const bool copies = id >= 0 && !keeps;
      a.to[i] = keeps ? id : -1;
      a.from[i] = copies ? id : -1;
      const uint32_t here = (c.entries + a.tokens - 1) / a.tokens, until = places_of(a, c, i);
      wants = (copies ? 1 : 0) + (until > here ? until - here : 0);
    }
    uint32_t sum;
    const uint32_t mine = before_mine(wants, waves, &sum);
    if (i < a.num_children) a.wants[i] = need + mine;
    need += sum;
  }
  __syncthreads();
  for (uint32_t i = t; i < a.num_children; i += kWide)  // kept ones count once
    if (a.to[i] >= 0) {
      put(a.refs_out + a.to[i], 1);
      a.to[i] = -1;
    }
  __syncthreads();
  // Free blocks, a wave a run of them: first how many, then each to the request of its number.
  const uint32_t run = ((a.num_blocks + kWide - 1) / kWide) * kOpsWave, begin = wave * run;
  uint32_t n = 0;
  for (uint32_t j = 0; j < run; j += kOpsWave) {
    const uint32_t id = begin + j + lane;
    n += __popcll(__ballot(id < a.num_blocks && look(a.refs_out + id) == 0));
  }
  if (!lane) free_before[wave] = n;
  __syncthreads();
  uint32_t number = 0, all = 0;
  for (uint32_t w = 0; w < kWaves; ++w) {
    if (w < wave) number += free_before[w];
    all += free_before[w];
  }
  for (uint32_t j = 0; j < run && number < need; j += kOpsWave) {
    const uint32_t id = begin + j + lane;
    const bool free = id < a.num_blocks && look(a.refs_out + id) == 0;
    const uint64_t them = __ballot(free);
    const uint32_t k = number + __popcll(them & ((1ull << lane) - 1));
    number += __popcll(them);
    if (!free || k >= need) continue;
    uint32_t lo = 0, hi = a.num_children;  // the last child whose requests start at or before k
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) / 2;
      if (a.wants[mid] <= k) lo = mid;
      else hi = mid;
    }
    const Child c = child_of(a, lo);
    const uint32_t nth = k - a.wants[lo], here = (c.entries + a.tokens - 1) / a.tokens;
    const bool copies = a.from[lo] >= 0;
    const uint32_t place = copies && !nth ? c.full : here + nth - (copies ? 1 : 0);
    a.table_out[static_cast<uint64_t>(lo) * a.out_stride + place] = static_cast<int32_t>(id);
    if (copies && !nth) a.to[lo] = static_cast<int32_t>(id);
    put(a.refs_out + id, 1);
  }
  if (!t) *a.free_out = static_cast<int32_t>(all) - static_cast<int32_t>(need);
}

// ---------------------------------------------------------------- compact
// Counts of pages, new ids and the list of moves. n pages are held: the k-th of those from n on goes to the k-th hole below n.
__global__ __launch_bounds__(kWide) void compact_list_kernel(CompactArgs a) {
  __shared__ uint32_t held_before[kWaves];
  const uint32_t t = threadIdx.x, lane = t % kOpsWave, wave = t / kOpsWave;
  const uint32_t run = ((a.num_blocks + kWide - 1) / kWide) * kOpsWave, begin = wave * run;
  uint32_t n = 0;
  for (uint32_t j = 0; j < run; j += kOpsWave) {
    const uint32_t id = begin + j + lane;
    n += __popcll(__ballot(id < a.num_blocks && a.refs[id] != 0));
  }
  if (!lane) held_before[wave] = n;
  __syncthreads();
  uint32_t number = 0, held = 0;
  for (uint32_t w = 0; w < kWaves; ++w) {
    if (w < wave) number += held_before[w];
    held += held_before[w];
  }
  // Held ones below `held`: needed by the waves that number the moves; the wave whose run has that place counts them.
  __shared__ uint32_t low_held;
  const uint32_t start = number;
  uint32_t at = number;
  for (uint32_t j = 0; j < run; j += kOpsWave) {
    const uint32_t id = begin + j + lane;
    const uint64_t them = __ballot(id < a.num_blocks && a.refs[id] != 0);
    if (held - (begin + j) < kOpsWave && !lane) low_held = at + __popcll(them & ((1ull << (held - begin - j)) - 1));
    at += __popcll(them);
  }
  if (held >= run * kWaves && !t) low_held = held;
  __syncthreads();
  at = start;
  for (uint32_t j = 0; j < run; j += kOpsWave) {
    const uint32_t id = begin + j + lane;
    const bool is = id < a.num_blocks && a.refs[id] != 0;
    const uint64_t them = __ballot(is);
    const uint32_t rank = at + __popcll(them & ((1ull << lane) - 1));  // held ones before it
    at += __popcll(them);
    if (id >= a.num_blocks) continue;
    if (id < held && !is) a.to[id - rank] = static_cast<int32_t>(id);
    if (id >= held && is) a.from[rank - low_held] = static_cast<int32_t>(id);
  }
  __syncthreads();
  const uint32_t moves = held - low_held;
  for (uint32_t id = t; id < a.num_blocks; id += kWide) {
    const int32_t r = a.refs[id];
    if (id < held ? r != 0 : r == 0) {
      a.moved[id] = r ? static_cast<int32_t>(id) : -1;
      a.refs_out[id] = r;
    }
  }
  __syncthreads();
  for (uint32_t k = t; k < moves; k += kWide) {  // a page and the hole that it fills by one thread: refs_out may be refs
    const int32_t from = a.from[k], to = a.to[k], r = a.refs[from];
    a.moved[from] = to;
    a.moved[to] = -1;
    a.refs_out[to] = r;
    a.refs_out[from] = 0;
  }
  if (!t) {
    *a.held_out = static_cast<int32_t>(held);
    *a.moves = moves;
  }
}

__global__ __launch_bounds__(256) void compact_table_kernel(CompactArgs a) {
  const uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= a.places) return;
  const int32_t id = a.table[i];
  int32_t to = -1;
  if (static_cast<uint32_t>(id) < a.num_blocks) to = a.moved[id];
  a.table_out[i] = to >= 0 ? to : id;
}

// ---------------------------------------------------------------- copies
// Pages from[k] to to[k] (where both are there) in every layer, K and V: 16 KiB at a time. Nothing is read that another
// copy of the call writes.
__global__ __launch_bounds__(256) void move_pages_kernel(MoveArgs a) {
  const uint32_t moves = a.moves ? *a.moves : a.most;
  const uint32_t chunks = static_cast<uint32_t>((a.piece + kCopy - 1) / kCopy), per = chunks * 2 * a.layers;
  const uint64_t items = static_cast<uint64_t>(moves) * per;
  for (uint64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const uint32_t k = static_cast<uint32_t>(item / per), rest = static_cast<uint32_t>(item % per);
    const int32_t from = a.from[k], to = a.to[k];
    if (from < 0 || to < 0) continue;
    const uint32_t layer = rest / (2 * chunks), which = rest / chunks % 2;
    const uint64_t at = static_cast<uint64_t>(rest % chunks) * kCopy;
    uint8_t* const base = reinterpret_cast<uint8_t*>(a.layer[layer]) + (which ? a.v_offset : 0) + at;
    const uint8_t* const p = base + static_cast<uint64_t>(from) * a.piece;
    uint8_t* const q = base + static_cast<uint64_t>(to) * a.piece;
    const uint64_t n = a.piece - at;
    u32x4 w[4];
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
      const uint32_t b = (i * 256 + threadIdx.x) * 16;
      if (b < n) w[i] = *reinterpret_cast<const u32x4*>(p + b);
    }
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
      const uint32_t b = (i * 256 + threadIdx.x) * 16;
      if (b < n) *reinterpret_cast<u32x4*>(q + b) = w[i];
    }
  }
}

}  // namespace

hipError_t launch_fork(const ForkArgs& a, hipStream_t stream) {
  hipError_t e;
  if (a.refs_out != a.refs && (e = launch(fork_counts_kernel, (a.num_blocks + 255) / 256, 256, stream, a)) != hipSuccess) return e;
  if (a.num_seqs + a.num_children && (e = launch(fork_rows_kernel, a.num_seqs + a.num_children, 256, stream, a)) != hipSuccess) return e;
  return launch(fork_give_kernel, 1, kWide, stream, a);
}

hipError_t launch_compact(const CompactArgs& a, hipStream_t stream) {
  const hipError_t e = launch(compact_list_kernel, 1, kWide, stream, a);
  if (e != hipSuccess || !a.places) return e;
  return launch(compact_table_kernel, static_cast<uint32_t>((a.places + 255) / 256), 256, stream, a);
}

hipError_t launch_moves(const MoveArgs& a, hipStream_t stream) {
  const uint64_t items = static_cast<uint64_t>(a.most) * ((a.piece + kCopy - 1) / kCopy) * 2 * a.layers;
  return launch(move_pages_kernel, static_cast<uint32_t>(items < 4096 ? items : 4096), 256, stream, a);
}

}  // namespace mma
