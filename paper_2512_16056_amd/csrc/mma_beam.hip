// Beam search's selection for gfx950 (MI355X): of each request the best continuations over its beams and
// the vocabulary.
//
// v = s + (x - lse), lse = log of the sum of exp x over the row. Within a row v is ordered as x is, so a row's best are
// found from its logits alone while its sum is formed; only across beams the sums enter. So a workgroup of
// beam_chunk_kernel reads 8192 logits of a row once, into registers, and leaves their maximum, their sum of exp and the
// `keep` best; beam_merge_kernel joins what a request's workgroups left. Rows in more parts than a merge takes are joined
// row by row between the two (beam_row_kernel).
//
// Sums and v are in 64 bits: two candidates of different beams may lie as close as the rounding of a 32-bit sum, and
// which of them is chosen is a whole number. The vector units do 64-bit multiply-adds at half the rate of 32-bit ones, so
// it costs little: 2^f on [-1/2, 1/2] is a polynomial of degree 8 (relative error 1.1e-12, interpolated at Chebyshev's
// points), about 13 64-bit operations a logit.
#include "mma_ops.h"

namespace mma {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kThreads = 512;
constexpr uint32_t kPer = kBeamChunk / kThreads;  // logits of a thread
constexpr uint32_t kList = 1024;                  // candidates that a workgroup ranks
constexpr uint32_t kMerge = 1024;                 // threads of a merge
constexpr uint32_t kMergePer = kBeamMerge / kMerge;

__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }

// Whole numbers in the order of floats; -0 has to be 0 already.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x);
  return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t b) {
  return __builtin_bit_cast(float, b ^ (b >> 31 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ uint64_t ordered(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  return b ^ (b >> 63 ? ~0ull : 1ull << 63);
}
__device__ __forceinline__ double unordered(uint64_t b) {
  return __builtin_bit_cast(double, b ^ (b >> 63 ? 1ull << 63 : ~0ull));
}

// A candidate of a row: its logit, then the lower token first. 0: none.
__device__ __forceinline__ uint64_t key_of(float x, uint32_t token) {
  return static_cast<uint64_t>(ordered(x)) << 32 | (0xffffffffu - token);
}

// e^d of -700 <= d <= 0.
__device__ __forceinline__ double exp_of(double d) {
  constexpr double kMagic = 6755399441055744.0;  // 1.5 2^52: added, it leaves the nearest whole number in the low bits
  const double t = fma(d, 1.4426950408889634, kMagic);
  const double f = fma(d, 1.4426950408889634, kMagic - t);
  double p = 1.325497460306718e-06;
  p = fma(p, f, 1.531007807039615e-05);
  p = fma(p, f, 0.00015403457039410448);
  p = fma(p, f, 0.0013333450573018062);
  p = fma(p, f, 0.009618129157656703);
  p = fma(p, f, 0.055504109412010456);
  p = fma(p, f, 0.24022650695821055);
  p = fma(p, f, 0.6931471805459343);
  p = fma(p, f, 0.9999999999999997);
  const uint64_t b = __builtin_bit_cast(uint64_t, p);  // times 2^n: into the exponent
  const uint32_t high = static_cast<uint32_t>(b >> 32) + (static_cast<uint32_t>(__builtin_bit_cast(uint64_t, t)) << 20);
  return __builtin_bit_cast(double, static_cast<uint64_t>(high) << 32 | static_cast<uint32_t>(b));
}

__device__ __forceinline__ float max_of_wave(float v) {
#pragma unroll
  for (int x = 1; x < kOpsWave; x *= 2) v = fmaxf(v, __shfl_xor(v, x, kOpsWave));
  return v;
}
__device__ __forceinline__ double sum_of_wave(double v) {
#pragma unroll
  for (int x = 1; x < kOpsWave; x *= 2) v += __shfl_xor(v, x, kOpsWave);
  return v;
}

// How many threads of the workgroup, over their N values each, hold what `is` says; the same for every thread.
template <int N, class F>
__device__ __forceinline__ uint32_t count_of(uint32_t* waves, F is) {
  uint32_t n = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) n += __popcll(__ballot(is(i)));
  __syncthreads();
  if (threadIdx.x % kOpsWave == 0) waves[threadIdx.x / kOpsWave] = n;
  __syncthreads();
  n = 0;
  for (uint32_t w = 0; w < blockDim.x / kOpsWave; ++w) n += waves[w];
  return n;
}

// A number that at least `keep` of 256 in LDS reach, and a quarter more at most where they differ: by one wave, bit by bit
// from the top. (Each of 256 threads ranking its own number against the others took 17 us, waiting on LDS.)
__device__ __forceinline__ uint32_t bound_of(const uint32_t* numbers, uint32_t keep) {
  const u32x4 x = *reinterpret_cast<const u32x4*>(numbers + threadIdx.x % kOpsWave * 4);
  const uint32_t enough = keep + keep / 4;
  uint32_t bound = 0;
  for (uint32_t bit = 1u << 31; bit; bit >>= 1) {
    const uint32_t next = bound | bit;
    const uint32_t n = __popcll(__ballot(x[0] >= next)) + __popcll(__ballot(x[1] >= next)) + __popcll(__ballot(x[2] >= next)) +
                       __popcll(__ballot(x[3] >= next));
    if (n >= keep) bound = next;
    if (n >= keep && n <= enough) break;
  }
  return bound;
}

// Places in a list for the lanes whose bits `is` has, after those of `*at`, which moves on by as many.
__device__ __forceinline__ uint32_t place_of(uint64_t is, uint32_t* at) {
  const uint32_t mine = *at + __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(is >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(is), 0));
  *at += __popcll(is);
  return mine;
}

// Candidates of a list in LDS: larger values first, equal ones by place (PLACES; else there are no equal ones).
struct List {
  uint64_t value[kList + 8];
  uint32_t rank[kList];
  uint32_t n;
};

// Ranks of the list's n candidates, counted by all of THREADS threads: of few candidates several threads have one, each
// against its share of the others. The list is filled up with zeros to a multiple of 8.
template <int THREADS, bool PLACES>
__device__ __forceinline__ void rank_list(List& l, const uint32_t* places, uint32_t n) {
  const uint32_t t = threadIdx.x, filled = (n + 7) & ~7u;
  if (t < 8 && n + t < filled) l.value[n + t] = 0;
  for (uint32_t i = t; i < n; i += THREADS) l.rank[i] = 0;
  __syncthreads();
  const uint32_t waves = (n + kOpsWave - 1) / kOpsWave;  // that the candidates fill
  const uint32_t parts = waves ? (THREADS / kOpsWave + waves - 1) / waves : 0, len = parts ? ((filled / 8 + parts - 1) / parts) * 8 : 0;
  for (uint32_t w = t / kOpsWave; w < waves * parts; w += THREADS / kOpsWave) {
    const uint32_t i = w % waves * kOpsWave + t % kOpsWave, begin = w / waves * len;
    const uint32_t end = begin + len < filled ? begin + len : filled;
    const uint64_t mine = i < n ? l.value[i] : ~0ull;
    const uint32_t place = PLACES && i < n ? places[i] : 0;
    uint32_t rank = 0;
    for (uint32_t j = begin; j < end; j += 8) {
#pragma unroll
      for (uint32_t x = 0; x < 8; ++x) {
        const uint64_t other = l.value[j + x];
        rank += other > mine ? 1 : 0;
        if constexpr (PLACES) rank += static_cast<uint32_t>(other == mine) & static_cast<uint32_t>(places[j + x] < place);  // those past n are 0, mine is not
      }
    }
    if (i < n && rank) atomicAdd(&l.rank[i], rank);
  }
  __syncthreads();
}

// A beam whose candidates come from its logits.
__device__ __forceinline__ bool grows(const BeamArgs& a, uint32_t row) {
  return finite(a.scores[row]) && !(a.done && a.done[row]);
}

template <class T>
__device__ __forceinline__ float to_float(const u32x4& w, uint32_t j) {
  const uint32_t word = w[j / (4 / sizeof(T))];  // a bit cast of the vector's element itself would take its first one
  if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, word);
  else return static_cast<float>(__builtin_bit_cast(T, static_cast<uint16_t>(word >> (j % 2 * 16))));
}

// 8192 logits of a row. Rows start at any multiple of an element: reads go from the 16 bytes that the row's start lies in.
// The `keep` best: as many of the threads' maxima reach a bound, so the keep-th best logit does. What reaches it (few
// more than keep) goes to a list and is ranked there. Where more reach it than the list holds, as of many equal
// logits, the bound is found bit by bit over all logits instead. One wave looks for the bound while the others form
// their sums.
template <class T>
__global__ __launch_bounds__(kThreads, 4) void beam_chunk_kernel(BeamArgs a) {
  constexpr uint32_t VEC = 16 / sizeof(T), NC = kPer / VEC;
  __shared__ List l;
  __shared__ __attribute__((aligned(16))) uint32_t maxima[kThreads / 2];
  __shared__ float tops[kThreads / kOpsWave];
  __shared__ double sums[kThreads / kOpsWave];
  __shared__ uint32_t waves[kThreads / kOpsWave], bound;
  const uint32_t row = blockIdx.x / a.splits, split = blockIdx.x % a.splits, t = threadIdx.x;
  const uint64_t start = reinterpret_cast<uint64_t>(a.logits) + row * a.row_bytes;
  const uint32_t ahead = static_cast<uint32_t>(start % 16) / sizeof(T);  // elements between there and the row's start
  const uint64_t first = static_cast<uint64_t>(split) * kBeamChunk, end = static_cast<uint64_t>(a.vocab) + ahead;
  const T* const from = reinterpret_cast<const T*>(start & ~15ull) + first;
  const uint32_t here = end <= first ? 0 : end - first < kBeamChunk ? static_cast<uint32_t>(end - first) : kBeamChunk;  // 0: a part
  // that only rows with another start have
  if (!grows(a, row)) return;  // the merge does not read its part
  float x[kPer], top = -INFINITY;
  bool bad = false;
  if ((first || !ahead) && here == kBeamChunk) {
    u32x4 w[NC];
#pragma unroll
    for (uint32_t i = 0; i < NC; ++i) w[i] = *reinterpret_cast<const u32x4*>(from + (i * kThreads + t) * VEC);
#pragma unroll
    for (uint32_t i = 0; i < kPer; ++i) x[i] = to_float<T>(w[i / VEC], i % VEC) + 0.0f;
  } else {
    const uint32_t low = first ? 0 : ahead;
    u32x4 w[NC];
#pragma unroll
    for (uint32_t i = 0; i < NC; ++i) {
      const uint32_t v = (i * kThreads + t) * VEC;
      w[i] = v < here ? *reinterpret_cast<const u32x4*>(from + v) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (uint32_t i = 0; i < kPer; ++i) {
      const uint32_t v = (i / VEC * kThreads + t) * VEC + i % VEC;
      const float y = to_float<T>(w[i / VEC], i % VEC) + 0.0f;
      x[i] = v >= low && v < here ? y : -INFINITY;
    }
  }
#pragma unroll
  for (uint32_t i = 0; i < kPer; ++i) {
    bad = bad || !(x[i] < INFINITY);
    top = fmaxf(top, x[i]);
  }
  const auto token_of = [&](uint32_t i) {
    return static_cast<uint32_t>(first - ahead) + (i / VEC * kThreads + t) * VEC + i % VEC;
  };
  float high = fmaxf(top, __shfl_xor(top, 1, kOpsWave));
  if (t % 2 == 0) maxima[t / 2] = ordered(high);
  high = max_of_wave(high);
  if (t % kOpsWave == 0) tops[t / kOpsWave] = high;
  if (!t) l.n = 0;
  __syncthreads();
  float all = tops[0];
#pragma unroll
  for (uint32_t i = 1; i < kThreads / kOpsWave; ++i) all = fmaxf(all, tops[i]);
  if (t / kOpsWave == split % (kThreads / kOpsWave)) {
    const uint32_t b = bound_of(maxima, a.keep);
    if (t % kOpsWave == 0) bound = b;
  }

  // The sum, from the chunk's maximum. Logits far below it count for e^-600, nothing.
  double sum[2] = {0, 0};
  if (all > -INFINITY) {
    const float floor = all - 600.0f;
    const double from_top = all;
#pragma unroll
    for (uint32_t i = 0; i < kPer; ++i) sum[i % 2] += exp_of(static_cast<double>(fmaxf(x[i], floor)) - from_top);
  }
  if (bad) sum[0] = NAN;
  sum[0] = sum_of_wave(sum[0] + sum[1]);
  if (t % kOpsWave == 0) sums[t / kOpsWave] = sum[0];
  __syncthreads();

  // The candidates: no -infinity among them.
  const float least = bound > ordered(-3.4028234664e38f) ? unordered(bound) : -3.4028234664e38f;
  if (__any(top >= least)) {
    uint32_t mine = 0, at = 0;
#pragma unroll
    for (uint32_t i = 0; i < kPer; ++i) mine += __popcll(__ballot(x[i] >= least));
    if (t % kOpsWave == 0) at = atomicAdd(&l.n, mine);
    at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
    for (uint32_t i = 0; i < kPer; ++i) {
      const uint64_t is = __ballot(x[i] >= least);
      if (!is) continue;
      const uint32_t to = place_of(is, &at);
      if (x[i] >= least && to < kList) l.value[to] = key_of(x[i], token_of(i));
    }
  }
  __syncthreads();
  const uint64_t part = static_cast<uint64_t>(row) * a.splits + split;
  if (!t) {
    a.part_max[part] = all;
    double add = sums[0];
#pragma unroll
    for (uint32_t i = 1; i < kThreads / kOpsWave; ++i) add += sums[i];
    a.part_sum[part] = add;
  }
  uint32_t n = l.n;
  if (n > kList) {  // the largest key that at least `keep` candidates reach, which are then exactly so many
    uint64_t key = 0;
#pragma unroll 1
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t next = key | 1ull << bit;
      if (count_of<kPer>(waves, [&](int i) { return x[i] > -INFINITY && key_of(x[i], token_of(i)) >= next; }) >= a.keep) key = next;
    }
    __syncthreads();
    if (!t) l.n = 0;
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < kPer; ++i)
      if (x[i] > -INFINITY && key_of(x[i], token_of(i)) >= key) l.value[atomicAdd(&l.n, 1u)] = key_of(x[i], token_of(i));
    __syncthreads();
    n = l.n;
  }
  rank_list<kThreads, false>(l, nullptr, n);
  uint64_t* const out = a.lists + part * a.keep;
  for (uint32_t i = t; i < n; i += kThreads)
    if (l.rank[i] < a.keep) out[l.rank[i]] = l.value[i];
  for (uint32_t i = n + t; i < a.keep; i += kThreads) out[i] = 0;
}

// The `keep` best of `total` values, `per` of each of 1024 threads side by side (0: none), ties to the lower place thread *
// per + i. Found as in beam_chunk_kernel, with the maxima of four threads each: values come in descending lists, and
// these are the lists' first ones. (With values 1024 apart a thread has one rank of many lists, the bound was so low that the
// list overflowed: 32 beams of 8 parts of 64, 42 us.) give(rank, value, place); returns how many there are.
template <class F>
__device__ __forceinline__ uint32_t best_of(const uint64_t (&v)[kMergePer], uint32_t total, uint32_t per, uint32_t keep, F give) {
  __shared__ List l;
  __shared__ __attribute__((aligned(16))) uint32_t maxima[256];
  __shared__ uint32_t places[kList + 8], waves[kMerge / kOpsWave], bound;
  const uint32_t t = threadIdx.x;
  if (!t) l.n = 0;
  if (total > 256) {  // else all go to the list
    uint64_t top = 0;
#pragma unroll
    for (uint32_t i = 0; i < kMergePer; ++i) top = v[i] > top ? v[i] : top;
    uint32_t high = static_cast<uint32_t>(top >> 32);
#pragma unroll
    for (int x = 1; x < 4; x *= 2) {
      const uint32_t y = __shfl_xor(high, x, kOpsWave);
      high = y > high ? y : high;
    }
    if (t % 4 == 0) maxima[t / 4] = high;
    __syncthreads();
    if (t < kOpsWave) {
      const uint32_t b = bound_of(maxima, keep);
      if (!t) bound = b;
    }
  }
  __syncthreads();
  uint64_t least = total > 256 ? static_cast<uint64_t>(bound) << 32 : 1;
  if (!least) least = 1;
  uint32_t mine = 0, at = 0;
#pragma unroll
  for (uint32_t i = 0; i < kMergePer; ++i) mine += __popcll(__ballot(v[i] >= least));
  if (mine && t % kOpsWave == 0) at = atomicAdd(&l.n, mine);
  at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
  for (uint32_t i = 0; i < kMergePer; ++i) {
    const uint64_t is = __ballot(v[i] >= least);
    if (!is) continue;
    const uint32_t to = place_of(is, &at);
    if (v[i] >= least && to < kList) l.value[to] = v[i], places[to] = t * per + i;
  }
  __syncthreads();
  uint32_t n = l.n;
  if (n > kList) {
    uint64_t key = 0;
#pragma unroll 1
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t next = key | 1ull << bit;
      if (count_of<kMergePer>(waves, [&](int i) { return v[i] >= next; }) >= keep) key = next;
    }
    // All above it, and of those that equal it the lowest places, up to `until`.
    const uint32_t more = keep - count_of<kMergePer>(waves, [&](int i) { return v[i] > key; });
    uint32_t until = 0;
#pragma unroll 1
    for (uint32_t bit = kBeamMerge; bit; bit /= 2) {
      const uint32_t next = until + bit;
      if (next <= kBeamMerge && count_of<kMergePer>(waves, [&](int i) { return v[i] == key && t * per + i < next; }) < more) until = next;
    }
    __syncthreads();
    if (!t) l.n = 0;
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < kMergePer; ++i)
      if (v[i] > key || (v[i] == key && t * per + i <= until)) {
        const uint32_t at = atomicAdd(&l.n, 1u);
        if (at < kList) l.value[at] = v[i], places[at] = t * per + i;
      }
    __syncthreads();
    n = l.n;
  }
  rank_list<kMerge, true>(l, places, n);
  for (uint32_t i = t; i < n; i += kMerge)
    if (l.rank[i] < keep) give(l.rank[i], l.value[i], places[i]);
  return n < keep ? n : keep;
}

// The best of a row's parts.
__global__ __launch_bounds__(kMerge) void beam_row_kernel(BeamArgs a) {
  const uint32_t row = blockIdx.x, n = a.splits * a.keep, t = threadIdx.x;
  if (!grows(a, row)) return;
  const uint64_t* from = a.lists + static_cast<uint64_t>(row) * n;
  uint64_t v[kMergePer];
  const uint32_t each = (n + kMerge - 1) / kMerge;
#pragma unroll
  for (uint32_t i = 0; i < kMergePer; ++i) {
    v[i] = 0;
    if (i < each && t * each + i < n) v[i] = from[t * each + i];
  }
  uint64_t* const out = a.rows + static_cast<uint64_t>(row) * a.keep;
  const uint32_t found = best_of(v, n, each, a.keep, [&](uint32_t rank, uint64_t key, uint32_t) { out[rank] = key; });
  for (uint32_t i = found + t; i < a.keep; i += kMerge) out[i] = 0;
}

// A request: of each beam log-sum-exp of its parts, then the best over all.
__global__ __launch_bounds__(kMerge) void beam_merge_kernel(BeamArgs a) {
  __shared__ double scores[kBeamMost], lses[kBeamMost];
  __shared__ uint8_t state[kBeamMost];  // 0: no candidates, 1: from its logits, 2: done
  const uint32_t item = blockIdx.x, t = threadIdx.x;
  constexpr uint32_t kLanes = kMerge / kBeamMost;  // of a beam
  const uint64_t* const lists = a.rows ? a.rows : a.lists;
  const uint32_t per = a.rows ? a.keep : a.splits * a.keep, n = a.beams * per;  // candidates of a beam, of all
  const uint64_t* const from = lists + static_cast<uint64_t>(item) * n;
  uint64_t v[kMergePer];
  const uint32_t each = (n + kMerge - 1) / kMerge;
#pragma unroll
  for (uint32_t i = 0; i < kMergePer; ++i) {  // the keys first; lists of beams that have none hold anything
    v[i] = 0;
    if (i < each && t * each + i < n) v[i] = from[t * each + i];
  }
  if (t / kLanes < a.beams) {
    const uint32_t beam = t / kLanes, lane = t % kLanes, row = item * a.beams + beam;
    const float* m = a.part_max + static_cast<uint64_t>(row) * a.splits;
    const double* s = a.part_sum + static_cast<uint64_t>(row) * a.splits;
    // Asked for at once: of a beam without candidates they are anything.
    const float score = a.scores[row];
    const uint8_t over = a.done ? a.done[row] : 0;
    const float m0 = lane < a.splits ? m[lane] : -INFINITY;
    const double s0 = lane < a.splits ? s[lane] : 0.0;
    uint8_t is = !finite(score) ? 0 : over ? 2 : 1;
    double lse = 0;
    if (is == 1) {
      float top = m0;
      for (uint32_t i = lane + kLanes; i < a.splits; i += kLanes) top = fmaxf(top, m[i]);
#pragma unroll
      for (uint32_t x = 1; x < kLanes; x *= 2) top = fmaxf(top, __shfl_xor(top, x, kLanes));
      const auto part = [&](float max, double sum) {
        return sum * (max > -INFINITY ? exp_of(static_cast<double>(fmaxf(max, top - 600.0f)) - top) : 0.0);
      };
      double sum = part(m0, s0);
      for (uint32_t i = lane + kLanes; i < a.splits; i += kLanes) sum += part(m[i], s[i]);
#pragma unroll
      for (uint32_t x = 1; x < kLanes; x *= 2) sum += __shfl_xor(sum, x, kLanes);
      if (!(sum > 0)) is = 0;  // no logit above -infinity, or one that is no number or +infinity
      lse = top + log(sum);
    }
    if (!lane) {
      scores[beam] = score;
      lses[beam] = lse;
      state[beam] = is;
    }
  }
  __syncthreads();
  {
    uint32_t beam = t * each / per, in = t * each - beam * per, is = 0;  // of the thread's first value, then of the next
    double score = 0, lse = 0;
    bool fresh = true;
#pragma unroll
    for (uint32_t i = 0; i < kMergePer; ++i) {
      if (i >= each || t * each + i >= n) break;
      if (fresh) is = state[beam], score = scores[beam], lse = lses[beam];
      const uint64_t key = v[i];
      v[i] = 0;
      if (is == 1 && key) v[i] = ordered(score + (unordered(static_cast<uint32_t>(key >> 32)) - lse) + 0.0);
      if (is == 2 && !in) v[i] = ordered(score + 0.0);
      fresh = ++in == per;
      if (fresh) in = 0, ++beam;
    }
  }
  const uint64_t to = static_cast<uint64_t>(item) * a.keep;
  const uint32_t found = best_of(v, n, each, a.keep, [&](uint32_t rank, uint64_t value, uint32_t at) {
    const uint32_t beam = at / per;
    a.tokens[to + rank] = state[beam] == 2 ? a.done_token : static_cast<int32_t>(0xffffffffu - static_cast<uint32_t>(from[at]));
    a.parents[to + rank] = static_cast<int32_t>(item * a.beams + beam);
    a.scores_out[to + rank] = static_cast<float>(unordered(value));
  });
  for (uint32_t i = found + t; i < a.keep; i += kMerge) {
    a.tokens[to + i] = a.parents[to + i] = -1;
    a.scores_out[to + i] = -INFINITY;
  }
}

}  // namespace

hipError_t launch_beam(const BeamArgs& a, uint32_t type, hipStream_t stream) {
  const uint32_t rows = a.batch * a.beams, grid = rows * a.splits;
  hipError_t e = type == MMA_TYPE_F32   ? launch(beam_chunk_kernel<float>, grid, kThreads, stream, a)
                 : type == MMA_TYPE_F16 ? launch(beam_chunk_kernel<_Float16>, grid, kThreads, stream, a)
                                        : launch(beam_chunk_kernel<__bf16>, grid, kThreads, stream, a);
  if (e != hipSuccess) return e;
  if (a.rows && (e = launch(beam_row_kernel, rows, kMerge, stream, a)) != hipSuccess) return e;
  return launch(beam_merge_kernel, a.batch, kMerge, stream, a);
}

}  // namespace mma
