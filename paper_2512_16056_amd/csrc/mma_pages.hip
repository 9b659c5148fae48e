// Pages of the cache for gfx950 (MI355X): sequences that go on from others (fork) and held pages moved together
// (compact). Both first decide which page goes where, over counts and tables of some ten thousand words, and then
// copy pages in every layer. The decisions depend on each other in order (the k-th request for a page gets the k-th
// free one), so one workgroup makes them, with few barriers; the copies are bound by HBM.
#include "mma_ops.h"

#include <algorithm>

namespace mma {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kWide = 1024;                 // threads of a workgroup that decides
constexpr uint32_t kWaves = kWide / kOpsWave;
constexpr uint32_t kCopy = 16384;                // bytes that a workgroup copies at once
constexpr uint32_t kForkBlocks = 32768;          // of a pool whose counts are in LDS
constexpr uint64_t kForkPlaces = 16384;          // of tables that one workgroup goes through (500 places: 5.6 us, in three
                                                 // launches 19; 36000: 27 and 18.5)
constexpr uint32_t kMasks = 2048;                // groups of 64 blocks whose bits are in LDS
constexpr uint32_t kMoves = 4096;                // moves of a compaction that are

// Words that other workgroups or waves change within the kernel: past the L1 cache.
__device__ __forceinline__ int32_t look(const int32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void put(int32_t* p, int32_t v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// A barrier for what is in LDS: stores to memory on their way are not waited for, as __syncthreads would (about 1 us each).
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
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
  lds_barrier();
  if (lane == kOpsWave - 1) waves[wave] = up;
  lds_barrier();
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

// What a workgroup of kWide threads has in LDS: the counts of a pool of up to kForkBlocks blocks, and up to kWide children, a
// thread each.
struct Small {
  int32_t refs[kForkBlocks];
  uint32_t entries[kWide], wants[kWide], copied[kWide];
  int32_t to[kWide];
  uint32_t waves[kWaves], free_before[kWaves];
};

__device__ __forceinline__ void load_counts(Small& s, const int32_t* refs, uint32_t n) {
  typedef uint32_t u32x4_anywhere __attribute__((ext_vector_type(4), aligned(4)));
  const uint32_t t = threadIdx.x;
  constexpr uint32_t kAtOnce = 4;
#pragma unroll 1
  for (uint32_t first = 0; first < n; first += kAtOnce * 4 * kWide) {
    u32x4 v[kAtOnce];
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) {  // all on their way before the first is waited for
      const uint32_t i = first + (k * kWide + t) * 4;
      v[k] = u32x4{0, 0, 0, 0};
      if (i + 4 <= n) v[k] = *reinterpret_cast<const u32x4_anywhere*>(refs + i);
    }
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) {
      const uint32_t i = first + (k * kWide + t) * 4;
      if (i + 4 <= n) *reinterpret_cast<u32x4*>(s.refs + i) = v[k];
    }
  }
  const uint32_t rest = n & ~3u;
  if (t < n - rest) s.refs[rest + t] = refs[rest + t];
}

// A thread's child: what its parent hands on, and its open block or -1.
__device__ __forceinline__ int32_t load_child(const ForkArgs& a, Small& s, Child* c, uint32_t* until) {
  const uint32_t t = threadIdx.x;
  *c = Child{0, 0, -1};
  *until = 0;
  int32_t open = -1;
  if (t < a.num_children) {
    *c = child_of(a, t);
    *until = places_of(a, *c, t);
    if (c->entries != c->full * a.tokens) {
      open = a.table[static_cast<uint64_t>(c->parent) * a.table_stride + c->full];
      if (static_cast<uint32_t>(open) >= a.num_blocks) open = -1;
    }
  }
  s.entries[t] = c->entries;
  return open;
}

// As fork_give_kernel, in LDS.
__device__ __forceinline__ void give_small(const ForkArgs& a, Small& s, const Child& c, int32_t open, uint32_t until) {
  const uint32_t t = threadIdx.x, lane = t % kOpsWave, wave = t / kOpsWave;
  int32_t* const refs = s.refs;
  const bool may = open >= 0 && refs[open] == 0;
  lds_barrier();
  if (may) atomicMin(&refs[open], INT32_MIN + static_cast<int32_t>(t));
  lds_barrier();
  const bool keeps = may && refs[open] == INT32_MIN + static_cast<int32_t>(t), copies = open >= 0 && !keeps;
  lds_barrier();
  if (keeps) refs[open] = 1;
  const uint32_t here = (c.entries + a.tokens - 1) / a.tokens;
  uint32_t need;
  s.wants[t] = before_mine((copies ? 1 : 0) + (until > here ? until - here : 0), s.waves, &need);
  s.copied[t] = copies ? c.full : ~0u;  // the place
  s.to[t] = -1;
  lds_barrier();
  const uint32_t run = ((a.num_blocks + kWide - 1) / kWide) * kOpsWave, begin = wave * run;
  uint32_t n = 0;
  for (uint32_t j = 0; j < run; j += kOpsWave) {
    const uint32_t id = begin + j + lane;
    n += __popcll(__ballot(id < a.num_blocks && refs[id] == 0));
  }
  if (!lane) s.free_before[wave] = n;
  lds_barrier();
  uint32_t number = 0, all = 0;
  for (uint32_t w = 0; w < kWaves; ++w) {
    if (w < wave) number += s.free_before[w];
    all += s.free_before[w];
  }
  for (uint32_t j = 0; j < run && number < need; j += kOpsWave) {
    const uint32_t id = begin + j + lane;
    const bool free = id < a.num_blocks && refs[id] == 0;
    const uint64_t them = __ballot(free);
    const uint32_t k = number + __popcll(them & ((1ull << lane) - 1));
    number += __popcll(them);
    if (!free || k >= need) continue;
    uint32_t lo = 0, hi = a.num_children;  // the last child whose requests start at or before k
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) / 2;
      if (s.wants[mid] <= k) lo = mid;
      else hi = mid;
    }
    const uint32_t nth = k - s.wants[lo], copied = s.copied[lo];
    const uint32_t place = copied == ~0u ? (s.entries[lo] + a.tokens - 1) / a.tokens + nth : copied + nth;
    a.table_out[static_cast<uint64_t>(lo) * a.out_stride + place] = static_cast<int32_t>(id);
    if (copied != ~0u && !nth) s.to[lo] = static_cast<int32_t>(id);
    refs[id] = 1;
  }
  if (!t) *a.free_out = static_cast<int32_t>(all) - static_cast<int32_t>(need);
  lds_barrier();
  if (t < a.num_children) {
    if (keeps) a.table_out[static_cast<uint64_t>(t) * a.out_stride + c.full] = open;
    a.from[t] = copies ? open : -1;
    a.to[t] = s.to[t];
  }
  for (uint32_t i = t; i < a.num_blocks; i += kWide) a.refs_out[i] = refs[i];
}

// After fork_rows_kernel. 192 children: 9.2 us, most of it loads and stores of the counts and rounds over them; the whole fork
// takes 25.7 us, with the counts in memory (fork_give_kernel) 29.6.
__global__ __launch_bounds__(kWide) void fork_give_small_kernel(ForkArgs a) {
  __shared__ __attribute__((aligned(16))) Small s;
  Child c;
  uint32_t until;
  load_counts(s, a.refs_out, a.num_blocks);
  const int32_t open = load_child(a, s, &c, &until);
  __syncthreads();
  give_small(a, s, c, open, until);
}

// All in one launch, for tables of up to kForkPlaces places: what bounds it is a chain of some ten loads and barriers.
__global__ __launch_bounds__(kWide) void fork_small_kernel(ForkArgs a) {
  __shared__ __attribute__((aligned(16))) Small s;
  __shared__ uint32_t children[kWide], full[kWide];
  __shared__ int32_t parent[kWide];
  const uint32_t t = threadIdx.x;
  load_counts(s, a.refs, a.num_blocks);
  children[t] = 0;
  if (t < a.num_seqs) {
    const int32_t n = a.lens[t];
    full[t] = (n < 0 ? 0 : static_cast<uint32_t>(n) < a.max_len ? n : a.max_len) / a.tokens;
  }
  Child c;
  uint32_t until;
  const int32_t open = load_child(a, s, &c, &until);
  parent[t] = c.parent;
  if (t < a.num_children) a.lens_out[t] = static_cast<int32_t>(c.entries);
  __syncthreads();
  if (c.parent >= 0) atomicAdd(&children[c.parent], 1u);
  __syncthreads();
  // The children's rows (whole blocks of the parent, none behind them yet), then the sequences' counts, eight places a thread
  // on their way.
  const uint32_t outs = a.num_children * a.out_stride, ins = a.num_seqs * a.table_stride;
  constexpr uint32_t kAtOnce = 8;
  for (uint32_t first = t; first < outs; first += kAtOnce * kWide) {
    int32_t id[kAtOnce];
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) {
      const uint32_t i = first + k * kWide;
      id[k] = -1;
      if (i >= outs) continue;
      const uint32_t child = i / a.out_stride, j = i - child * a.out_stride;
      if (j < s.entries[child] / a.tokens) id[k] = a.table[static_cast<uint64_t>(parent[child]) * a.table_stride + j];
    }
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) {
      const uint32_t i = first + k * kWide;
      if (i < outs) a.table_out[i] = static_cast<uint32_t>(id[k]) < a.num_blocks ? id[k] : -1;
    }
  }
  for (uint32_t first = t; first < ins; first += kAtOnce * kWide) {
    int32_t id[kAtOnce], by[kAtOnce];
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) {
      const uint32_t i = first + k * kWide;
      by[k] = 0;
      if (i >= ins) continue;
      const uint32_t seq = i / a.table_stride, j = i - seq * a.table_stride;
      by[k] = static_cast<int32_t>(j < full[seq] ? children[seq] : 0) - 1;
      id[k] = a.table[i];
    }
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k)
      if (by[k] && static_cast<uint32_t>(id[k]) < a.num_blocks) atomicAdd(&s.refs[id[k]], by[k]);
  }
  __syncthreads();
  give_small(a, s, c, open, until);
}

// ---------------------------------------------------------------- compact
// Counts of pages, new ids and the list of moves (4096 blocks: 5.6 us; 64: 2.7). n pages are held: the k-th of those from n on goes to the k-th hole below n.
// Which are held is kept in LDS, a bit each, where it fits (pools of up to 131072 blocks).
__global__ __launch_bounds__(kWide) void compact_list_kernel(CompactArgs a) {
  __shared__ uint64_t masks[kMasks];
  __shared__ int32_t froms[kMoves], tos[kMoves];  // the first moves
  __shared__ uint32_t held_before[kWaves], low_held;
  const uint32_t t = threadIdx.x, lane = t % kOpsWave, wave = t / kOpsWave;
  const uint32_t run = ((a.num_blocks + kWide - 1) / kWide) * kOpsWave, begin = wave * run;  // a wave's blocks
  const bool fits = run / kOpsWave * kWaves <= kMasks;
  uint32_t n = 0;
  for (uint32_t j = 0; j < run; j += 4 * kOpsWave) {
    int32_t r[4];
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) {
      const uint32_t id = begin + j + k * kOpsWave + lane;
      r[k] = j + k * kOpsWave < run && id < a.num_blocks ? a.refs[id] : 0;
    }
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) {
      const uint64_t them = __ballot(r[k] != 0);
      if (fits && !lane && j + k * kOpsWave < run) masks[(begin + j) / kOpsWave + k] = them;
      n += __popcll(them);
    }
  }
  if (!lane) held_before[wave] = n;
  __syncthreads();
  uint32_t number = 0, held = 0;
  for (uint32_t w = 0; w < kWaves; ++w) {
    if (w < wave) number += held_before[w];
    held += held_before[w];
  }
  const auto group = [&](uint32_t j) -> uint64_t {
    if (fits) return masks[(begin + j) / kOpsWave];
    const uint32_t id = begin + j + lane;
    return __ballot(id < a.num_blocks && a.refs[id] != 0);
  };
  // Held ones below `held`: needed by the waves that number the moves; the wave whose run has that place counts them.
  if (held >= begin && held < begin + run) {
    uint32_t at = number;
    for (uint32_t j = 0; j < run; j += kOpsWave) {
      const uint64_t them = group(j);
      if (held - (begin + j) < kOpsWave && !lane) low_held = at + __popcll(them & ((1ull << (held - begin - j)) - 1));
      at += __popcll(them);
    }
  }
  if (held >= run * kWaves && !t) low_held = held;
  __syncthreads();
  uint32_t at = number;
  for (uint32_t j = 0; j < run; j += kOpsWave) {
    const uint32_t id = begin + j + lane;
    const uint64_t them = group(j);
    const bool is = them >> lane & 1;
    const uint32_t rank = at + __popcll(them & ((1ull << lane) - 1));  // held ones before it
    at += __popcll(them);
    if (id >= a.num_blocks) continue;
    if (id < held && !is) {
      a.to[id - rank] = static_cast<int32_t>(id);
      if (id - rank < kMoves) tos[id - rank] = static_cast<int32_t>(id);
    }
    if (id >= held && is) {
      a.from[rank - low_held] = static_cast<int32_t>(id);
      if (rank - low_held < kMoves) froms[rank - low_held] = static_cast<int32_t>(id);
    }
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
    const int32_t from = k < kMoves ? froms[k] : a.from[k], to = k < kMoves ? tos[k] : a.to[k], r = a.refs[from];
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

// ---------------------------------------------------------------- copies
// Pages from[k] to to[k] (where both are there) in every layer, K and V: 16 KiB at a time, past the caches (983 pages of 64 KiB
// in 4 layers, 515 MB read and written: 97 us, 5.3 TB/s). Nothing is read that another copy of the call writes. Of a compaction
// also the table's places.
__global__ __launch_bounds__(256) void move_pages_kernel(MoveArgs a) {
  for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x; i < a.places; i += gridDim.x * 256ull) {
    const int32_t id = a.table[i];
    int32_t to = -1;
    if (static_cast<uint32_t>(id) < a.num_blocks) to = a.moved[id];
    a.table_out[i] = to >= 0 ? to : id;
  }
  const uint32_t moves = a.moves ? *a.moves : a.most;
  const uint32_t chunks = static_cast<uint32_t>((a.piece + kCopy - 1) / kCopy), per = chunks * 2 * a.layers;
  const uint64_t items = static_cast<uint64_t>(moves) * per;
  // A workgroup's items follow each other's distance; the next one's loads are on their way before this one's stores.
  struct Item {
    const uint8_t* p;
    uint8_t* q;
    uint32_t n;  // bytes, 0: none
  };
  const auto item_of = [&](uint64_t item) {
    Item r{nullptr, nullptr, 0};
    if (item >= items) return r;
    const uint32_t k = static_cast<uint32_t>(item / per), rest = static_cast<uint32_t>(item % per);
    const int32_t from = a.from[k], to = a.to[k];
    if (from < 0 || to < 0) return r;
    const uint32_t layer = rest / (2 * chunks), which = rest / chunks % 2;
    const uint64_t at = static_cast<uint64_t>(rest % chunks) * kCopy;
    uint8_t* const base = reinterpret_cast<uint8_t*>(a.layer[layer]) + (which ? a.v_offset : 0) + at;
    r.p = base + static_cast<uint64_t>(from) * a.piece;
    r.q = base + static_cast<uint64_t>(to) * a.piece;
    r.n = a.piece - at < kCopy ? static_cast<uint32_t>(a.piece - at) : kCopy;
    return r;
  };
  constexpr uint32_t kLoads = kCopy / 4096;
  u32x4 w[kLoads];
  const auto load = [&](const Item& x) {
#pragma unroll
    for (uint32_t i = 0; i < kLoads; ++i) {
      const uint32_t b = (i * 256 + threadIdx.x) * 16;
      if (b < x.n) w[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(x.p + b));
    }
  };
  Item now = item_of(blockIdx.x);
  load(now);
  for (uint64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const Item next = item_of(item + gridDim.x);
    u32x4 out[kLoads];
#pragma unroll
    for (uint32_t i = 0; i < kLoads; ++i) out[i] = w[i];
    load(next);
#pragma unroll
    for (uint32_t i = 0; i < kLoads; ++i) {
      const uint32_t b = (i * 256 + threadIdx.x) * 16;
      if (b < now.n) __builtin_nontemporal_store(out[i], reinterpret_cast<u32x4*>(now.q + b));
    }
    now = next;
  }
}

}  // namespace

hipError_t launch_fork(const ForkArgs& a, hipStream_t stream) {
  hipError_t e;
  const uint64_t places = static_cast<uint64_t>(a.num_seqs) * a.table_stride + static_cast<uint64_t>(a.num_children) * a.out_stride;
  const bool small = a.num_blocks <= kForkBlocks && a.num_children <= kWide;
  if (small && a.num_seqs <= kWide && places <= kForkPlaces) return launch(fork_small_kernel, 1, kWide, stream, a);
  if (a.refs_out != a.refs && (e = launch(fork_counts_kernel, (a.num_blocks + 255) / 256, 256, stream, a)) != hipSuccess) return e;
  if (a.num_seqs + a.num_children && (e = launch(fork_rows_kernel, a.num_seqs + a.num_children, 256, stream, a)) != hipSuccess) return e;
  return small ? launch(fork_give_small_kernel, 1, kWide, stream, a) : launch(fork_give_kernel, 1, kWide, stream, a);
}

hipError_t launch_compact(const CompactArgs& a, hipStream_t stream) { return launch(compact_list_kernel, 1, kWide, stream, a); }

hipError_t launch_moves(const MoveArgs& a, hipStream_t stream) {
  const uint64_t items = std::max(static_cast<uint64_t>(a.most) * ((a.piece + kCopy - 1) / kCopy) * 2 * a.layers, (a.places + 255) / 256);
  if (!items) return hipSuccess;
  return launch(move_pages_kernel, static_cast<uint32_t>(std::min<uint64_t>(items, 4096)), 256, stream, a);
}

}  // namespace mma
