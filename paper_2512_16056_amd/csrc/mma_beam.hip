// Beam search's selection for gfx950 (MI355X): of each request the best continuations over its beams and
// the vocabulary.
//
// v = s + (x - lse), lse = log of the sum of exp x over the row. Within a row v is ordered as x is, so a row's best are
// found from its logits alone while its sum is formed; only across beams the sums enter. So a workgroup of
// beam_part_kernel reads a run of a row's logits once, 4096 at a time, and leaves their sum of exp and the `keep` best;
// beam_merge_kernel joins what a request's workgroups left. Rows in more parts than a merge takes are joined row by row
// between the two (beam_row_kernel).
//
// Sums and v are in 64 bits: two candidates of different beams may lie as close as the rounding of a 32-bit sum, and
// which of them is chosen is a whole number. 2^f on [-1/2, 1/2] is a polynomial of degree 7 (relative error 5.5e-11,
// interpolated at Chebyshev's points). A 64-bit multiply-add takes a SIMD no longer than a 32-bit one, 4 cycles for 64
// lanes, and a logit some 15 such instructions.
#include "mma_ops.h"

namespace mma {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_anywhere __attribute__((ext_vector_type(4), aligned(2)));

constexpr uint32_t kThreads = 256;
constexpr uint32_t kPer = kBeamChunk / kThreads;  // logits of a thread at a time
constexpr uint32_t kList = 1024;                  // candidates of a part
constexpr uint32_t kMerge = 1024;                 // threads of a merge
constexpr uint32_t kMergePer = kBeamMerge / kMerge;
constexpr uint32_t kMergeList = 2816;             // candidates of a merge
constexpr int kOrderBits = 52;                    // of what equal values of a merge go by
constexpr float kLeast = -3.4028234664e38f;       // the least finite number

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
  return static_cast<uint64_t>(ordered(x + 0.0f)) << 32 | (0xffffffffu - token);  // -0 as 0
}

constexpr double kE2 = 1.4426950408889634;     // log2(e)
constexpr double kMagic = 6755399441055744.0;  // 1.5 2^52: added, it leaves the nearest whole number in the low bits

// e^d 2^-R, where `magic` is kMagic - R, for a whole number R: d up to 2^49 in size, the result from 2^-1000 to 2^1000.
__device__ __forceinline__ double exp_of(double d, double magic = kMagic) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const double t = fma(d, kE2, magic);
  const double f = fma(d, kE2, magic - t);
  double p = 1.5303699001378845e-05;
  p = fma(p, f, 0.00015469729140704658);
  p = fma(p, f, 0.0013333478480888061);
  p = fma(p, f, 0.009618025613598036);
  p = fma(p, f, 0.055504109063177154);
  p = fma(p, f, 0.24022651213495422);
  p = fma(p, f, 0.6931471805568341);
  p = fma(p, f, 0.9999999999595622);
  u32x2 b = __builtin_bit_cast(u32x2, p);  // times 2^n: into the exponent
  b[1] += static_cast<uint32_t>(__builtin_bit_cast(uint64_t, t)) << 20;
  return __builtin_bit_cast(double, b);
}

// e^(x - top) for an x up to `top`, no less than e^-600. The difference is of 64 bits: from 2^33 on 32 bits round 600 less to 1024
// less, or to `top` itself. 1 of `top`, where the polynomial is 4e-11 less: a row's only candidate then has lse = its logit.
__device__ __forceinline__ double power_below(float x, float top) {
  const double p = exp_of(fmax(static_cast<double>(x) - top, -600.0));
  return x == top ? 1.0 : p;
}

// Powers, as of exp_of, of four numbers, no less than `floor`, added to `sums`: side by side, so that a wave by itself keeps the unit busy.
__device__ __forceinline__ void exp_of_4(const float* x, float floor, double magic, double (&sums)[4]) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  constexpr double kTerms[7] = {0.00015469729140704658, 0.0013333478480888061, 0.009618025613598036, 0.055504109063177154,
                                0.24022651213495422, 0.6931471805568341, 0.9999999999595622};
  double d[4], t[4], p[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) d[i] = __builtin_amdgcn_fmed3f(x[i], floor, INFINITY);  // the larger one, in one instruction
#pragma unroll
  for (int i = 0; i < 4; ++i) t[i] = fma(d[i], kE2, magic);
#pragma unroll
  for (int i = 0; i < 4; ++i) d[i] = fma(d[i], kE2, magic - t[i]);
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = 1.5303699001378845e-05;
#pragma unroll
  for (int j = 0; j < 7; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = fma(p[i], d[i], kTerms[j]);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    u32x2 b = __builtin_bit_cast(u32x2, p[i]);
    b[1] += static_cast<uint32_t>(__builtin_bit_cast(uint64_t, t[i])) << 20;
    sums[i] += __builtin_bit_cast(double, b);
  }
}

// A lane's value from another place of its row of 16 lanes.
template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t x) {
  return __builtin_amdgcn_mov_dpp(x, CTRL, 0xf, 0xf, true);
}
// Joined over the wave's lanes, without LDS: neighbours, pairs, halves of a row and rows mirrored, then rows exchanged.
template <class F>
__device__ __forceinline__ uint32_t over_wave(uint32_t x, F join) {
  x = join(x, moved<0xb1>(x));
  x = join(x, moved<0x4e>(x));
  x = join(x, moved<0x141>(x));
  x = join(x, moved<0x140>(x));
  auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = join(static_cast<uint32_t>(a[0]), static_cast<uint32_t>(a[1]));
  a = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return join(static_cast<uint32_t>(a[0]), static_cast<uint32_t>(a[1]));
}
__device__ __forceinline__ uint32_t max_of_wave(uint32_t x) {
  return over_wave(x, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
template <int CTRL>
__device__ __forceinline__ double plus_moved(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint64_t m = static_cast<uint64_t>(moved<CTRL>(static_cast<uint32_t>(b >> 32))) << 32 | moved<CTRL>(static_cast<uint32_t>(b));
  return v + __builtin_bit_cast(double, m);
}
__device__ __forceinline__ double sum_of_row(double v) {  // over 16 lanes
  return plus_moved<0x140>(plus_moved<0x141>(plus_moved<0x4e>(plus_moved<0xb1>(v))));
}
__device__ __forceinline__ double sum_of_wave(double v) {
  v = sum_of_row(v);
  v += __shfl_xor(v, 16, kOpsWave);
  return v + __shfl_xor(v, 32, kOpsWave);
}

// The sum of what each wave has, for every thread.
__device__ __forceinline__ uint32_t sum_of_waves(uint32_t* waves, uint32_t n) {
  __syncthreads();
  if (threadIdx.x % kOpsWave == 0) waves[threadIdx.x / kOpsWave] = n;
  __syncthreads();
  n = 0;
  for (uint32_t w = 0; w < blockDim.x / kOpsWave; ++w) n += waves[w];
  return n;
}

// How many threads of the workgroup, over their N values each, hold what `is` says; the same for every thread.
template <int N, class F>
__device__ __forceinline__ uint32_t count_of(uint32_t* waves, F is) {
  uint32_t n = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) n += __popcll(__ballot(is(i)));
  return sum_of_waves(waves, n);
}

// A number that at least `keep` of N in LDS reach, and a quarter more at most where they differ: by one wave, from the
// largest with as few of its low bits gone as it takes, then bit by bit. (Each of 256 threads ranking its own number
// against the others took 17 us, waiting on LDS; all 32 bits one by one 2.3 us.)
template <int N>
__device__ __forceinline__ uint32_t bound_of(const uint32_t* numbers, uint32_t keep) {
  u32x4 x[N / 256];
#pragma unroll
  for (int i = 0; i < N / 256; ++i) x[i] = *reinterpret_cast<const u32x4*>(numbers + (i * kOpsWave + threadIdx.x % kOpsWave) * 4);
  const auto reach = [&](uint32_t v) {
    uint64_t who[N / 64];
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < N / 64; ++i) who[i] = __ballot(x[i / 4][i % 4] >= v);
#pragma unroll
    for (int i = 0; i < N / 64; ++i) n += __popcll(who[i]);
    return n;
  };
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < N / 256; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) top = x[i][j] > top ? x[i][j] : top;
  top = __builtin_amdgcn_readfirstlane(max_of_wave(top));
  uint32_t gone = 0;
#pragma unroll 1
  for (uint32_t half = 16; half; half /= 2)
    if (reach(top >> (gone + half - 1) << (gone + half - 1)) < keep) gone += half;
  uint32_t bound = top >> gone << gone, n = reach(bound);
  if (n < keep) bound = 0, gone = 32, n = N;
#pragma unroll 1
  for (uint32_t bit = gone > 1 ? 1u << (gone - 2) : 0; bit && n > keep + keep / 4; bit >>= 1) {
    const uint32_t next = reach(bound | bit);
    if (next >= keep) bound |= bit, n = next;
  }
  return bound;
}

// Candidates of a list in LDS: larger values first, equal ones by place (PLACES; else there are no equal ones).
template <int N>
struct List {
  uint64_t value[N + 8];
  uint32_t rank[N];
};

// Ranks of the list's n candidates. Up to 64 are one wave's; of more, all of THREADS threads count, several of them for one
// candidate where there are few, each against its share of the others. The list is filled up with zeros to a multiple of 8.
template <int THREADS, bool PLACES, int N>
__device__ __forceinline__ void rank_list(List<N>& l, const uint32_t* places, uint32_t n) {
  const uint32_t t = threadIdx.x, filled = (n + 7) & ~7u;
  if (n <= kOpsWave) {
    if (t < n) {
      const uint64_t mine = l.value[t];
      const uint32_t low = static_cast<uint32_t>(mine), high = static_cast<uint32_t>(mine >> 32), place = PLACES ? places[t] : 0;
      uint32_t rank = 0;
      for (uint32_t j = 0; j < n; ++j) {
        const uint64_t other = static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(high, j))) << 32 |
                               static_cast<uint32_t>(__builtin_amdgcn_readlane(low, j));
        rank += other > mine ? 1 : 0;
        if constexpr (PLACES) rank += static_cast<uint32_t>(other == mine) & static_cast<uint32_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(place, j)) < place);
      }
      l.rank[t] = rank;
    }
    __syncthreads();
    return;
  }
  if (t < 8 && n + t < filled) l.value[n + t] = 0;
  for (uint32_t i = t; i < n; i += THREADS) l.rank[i] = 0;
  __syncthreads();
  const uint32_t waves = (n + kOpsWave - 1) / kOpsWave;  // that the candidates fill
  const uint32_t parts = (THREADS / kOpsWave + waves - 1) / waves, len = ((filled / 8 + parts - 1) / parts) * 8;
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

// Leaves of a list of n (more than keep, at most N) those that reach a bound which hardly more than `keep` do, by the upper
// halves of their values; the others' order does not matter. Returns how many.
template <int THREADS, int N>
__device__ __forceinline__ uint32_t thin(List<N>& l, uint32_t* places, uint32_t* numbers, uint32_t* waves, uint32_t n, uint32_t keep) {
  const uint32_t t = threadIdx.x;
  constexpr uint32_t kMine = (N + THREADS - 1) / THREADS;
  static_assert(N % 256 == 0, "");
  uint64_t v[kMine];
  uint32_t place[kMine];
  for (uint32_t i = t; i < N; i += THREADS) numbers[i] = i < n ? static_cast<uint32_t>(l.value[i] >> 32) : 0;
#pragma unroll
  for (uint32_t i = 0; i < kMine; ++i) {
    v[i] = i * THREADS + t < n ? l.value[i * THREADS + t] : 0;
    place[i] = places && i * THREADS + t < n ? places[i * THREADS + t] : 0;
  }
  __syncthreads();
  if (t < kOpsWave) {
    const uint32_t b = n <= 256    ? bound_of<256>(numbers, keep)
                       : n <= 512  ? bound_of<512>(numbers, keep)
                       : n <= 1024 ? bound_of<1024>(numbers, keep)
                                   : bound_of<N>(numbers, keep);
    if (!t) waves[0] = b, waves[1] = 0;
  }
  __syncthreads();
  const uint32_t b = waves[0];
#pragma unroll
  for (uint32_t i = 0; i < kMine; ++i)
    if (v[i] && v[i] >> 32 >= b) {
      const uint32_t to = atomicAdd(&waves[1], 1u);
      l.value[to] = v[i];
      if (places) places[to] = place[i];
    }
  __syncthreads();
  return waves[1];
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

// A run of a row's logits, 4096 at a time, the next ones on their way. Rows start at any multiple of an element, and a thread's
// logits go by their tokens all the same, not by 16 aligned bytes: equal rows so have equal sums, to the last bit, and
// beams that are alike tie.
//
// The sum of exp is a thread's own, from its largest logit of the first time, until the end. Of each time a thread leaves
// the upper half of its largest logit in LDS, and nothing else: no wave waits for another. After up to 32 times the
// `keep` best are found from these: as many of the threads' largest reach a bound, so the keep-th best logit does; the few
// times of threads that have reached it are read again, and what reaches it goes to a list, which is thinned where it is
// long and ranked at the end. Where the list overflows, as of equal logits, it is found anew, 4096 logits after 4096 (careful).
//
// 192 rows of 128001 in 32 bits (98 MB): 28.6 us, 3.4 TB/s, where reading them would take 16.4. What bounds it is vector
// instructions, some 330 a wave for 1024 logits, 224 of them the powers: 4.6 cycles each, 17 us were every SIMD busy to the
// end; as older waves go first, the last workgroups of a CU have its SIMDs to themselves and are slower than that. With every
// wave collecting candidates as logits passed it was 39 us, with a wait of the workgroup at every 8192 logits 47.
template <class T>
__global__ __launch_bounds__(kThreads, 4) void beam_part_kernel(BeamArgs a) {
  constexpr uint32_t VEC = 16 / sizeof(T), NC = kPer / VEC, kWaves = kThreads / kOpsWave, kSegment = kThreads * VEC, kRound = 32;
  __shared__ List<kList> l;
  __shared__ __attribute__((aligned(16))) uint32_t numbers[kList];
  __shared__ uint16_t highs[kRound][kThreads];
  __shared__ uint16_t hits[kList];  // times of threads whose largest reaches the bound: time of the round * 256 + thread
  __shared__ float tops[kWaves];
  __shared__ double sums[kWaves];
  __shared__ uint32_t waves[kWaves], bound, listed, hit;
  const uint32_t row = blockIdx.x / a.splits, split = blockIdx.x % a.splits, t = threadIdx.x, lane = t % kOpsWave, wave = t / kOpsWave;
  const uint32_t first = split * a.run * kBeamChunk, all = a.vocab - first;  // of the part's first logit; logits from there on
  const uint32_t many = all < a.run * kBeamChunk ? all : a.run * kBeamChunk, times = (many + kBeamChunk - 1) / kBeamChunk;
  const uint16_t* const from = reinterpret_cast<const uint16_t*>(a.logits + row * a.row_bytes) + first * static_cast<uint64_t>(sizeof(T) / 2);
  if (!grows(a, row)) return;  // the merge does not read its part
  u32x4 w[NC];
  float x[kPer];
  const auto place_at = [&](uint32_t time, uint32_t i) { return time * kBeamChunk + i / VEC * kSegment + t * VEC + i % VEC; };
  // 16 bytes of the run from logit `at` on, those that are in it.
  const auto vector_at = [&](uint32_t at) -> u32x4 {
    const uint16_t* const p = from + static_cast<uint64_t>(at) * (sizeof(T) / 2);
    if (at + VEC <= many) return *reinterpret_cast<const u32x4_anywhere*>(p);
    const uint32_t n = at < many ? (many - at) * static_cast<uint32_t>(sizeof(T) / 2) : 0;  // halves of words
    u32x4 v;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) v[j] = (2 * j < n ? p[2 * j] : 0u) | (2 * j + 1 < n ? static_cast<uint32_t>(p[2 * j + 1]) << 16 : 0u);
    return v;
  };
  const auto load = [&](uint32_t time) {
    if ((time + 1) * kBeamChunk <= many) {
      const uint8_t* const p = reinterpret_cast<const uint8_t*>(from) + static_cast<uint64_t>(time) * kBeamChunk * sizeof(T) + t * 16;
#pragma unroll
      for (uint32_t i = 0; i < NC; ++i) w[i] = *reinterpret_cast<const u32x4_anywhere*>(p + i * kThreads * 16);
    } else {
#pragma unroll
      for (uint32_t i = 0; i < NC; ++i) w[i] = vector_at(place_at(time, i * VEC));
    }
  };
  const auto arrive = [&](uint32_t time) {  // and ask for the next ones
#pragma unroll
    for (uint32_t i = 0; i < kPer; ++i) x[i] = to_float<T>(w[i / VEC], i % VEC);
    if ((time + 1) * kBeamChunk > many) {
#pragma unroll
      for (uint32_t i = 0; i < kPer; ++i) x[i] = place_at(time, i) < many ? x[i] : -INFINITY;
    }
    if (time + 1 < times) load(time + 1);
    float top = x[0];
#pragma unroll
    for (uint32_t i = 1; i < kPer; ++i) top = fmaxf(top, x[i]);
    return top;
  };
  const auto key_at = [&](uint32_t time, uint32_t i) { return key_of(x[i], first + place_at(time, i)); };
  float ref = -INFINITY, floor = 0, least = kLeast;
  // The sum of e^x 2^-R, R the whole number next to log2 e^ref; or of e^(x - ref), where `ref` is so large that the product
  // with log2 e would lose the difference.
  double sum = 0, magic = kMagic;
  const auto near = [&] { return fabsf(ref) < 0x1p20f; };
  bool bad = false;
  if (!t) listed = 0;
  load(0);
  float best = -INFINITY;  // the thread's largest of the round
  for (uint32_t time = 0; time < times; ++time) {
    const float top = arrive(time);
    highs[time % kRound][t] = static_cast<uint16_t>(ordered(top != top ? -INFINITY : top + 0.0f) >> 16);
    best = fmaxf(best, top);
    bad = bad || top == INFINITY;
    // A new `ref` where none was or the old one is far below: no power passes 64 bits' range, and logits far below it count for
    // e^-596, nothing.
    if ((top > ref + 300.0f || ref == -INFINITY) && top > -INFINITY && top < INFINITY) {
      if (near()) sum /= exp_of(ref, magic);
      sum = ref > top - 600.0f ? sum * exp_of(static_cast<double>(ref) - top) : 0.0;
      ref = top;
      magic = kMagic - rint(ref * kE2);
      floor = ref - 596.0f;
      if (near()) sum *= exp_of(ref, magic);
    }
    if (near()) {
      double more[4] = {0, 0, 0, 0};
#pragma unroll
      for (uint32_t i = 0; i < kPer; i += 4) exp_of_4(x + i, floor, magic, more);
      sum += (more[0] + more[1]) + (more[2] + more[3]);
    } else if (ref > -INFINITY) {
#pragma unroll
      for (uint32_t i = 0; i < kPer; ++i) sum += exp_of(fmax(static_cast<double>(x[i]) - ref, -600.0));
    }
#pragma unroll
    for (uint32_t i = 0; i < kPer; i += 2) bad = bad || __builtin_isunordered(x[i], x[i + 1]);
    if (time + 1 < times && (time + 1) % kRound) continue;

    // The round's candidates: no -infinity among them.
    const uint32_t rounds = time / kRound * kRound, of_round = time + 1 - rounds;
    numbers[t] = ordered(best + 0.0f);
    if (!t) hit = 0;
    __syncthreads();
    if (wave == split % kWaves) {
      const uint32_t b = bound_of<256>(numbers, a.keep);
      if (!lane) bound = b;
    }
    __syncthreads();
    if (bound > ordered(least)) least = unordered(bound);
    if (best >= least) {
      const uint32_t high = ordered(least) >> 16;
      for (uint32_t i = 0; i < of_round; ++i)
        if (highs[i][t] >= high) {
          const uint32_t to = atomicAdd(&hit, 1u);
          if (to < kList) hits[to] = static_cast<uint16_t>(i * kThreads + t);
        }
    }
    best = -INFINITY;
    __syncthreads();
    const uint32_t reached = hit;
    if (reached > kList) {
      if (!t) listed = kList + 1;  // careful
    } else {
      for (uint32_t i = t; i < reached * NC; i += kThreads) {  // a thread 16 bytes of a hit
        const uint32_t h = hits[i / NC], at = (rounds + h / kThreads) * kBeamChunk + i % NC * kSegment + h % kThreads * VEC;
        const u32x4 v = vector_at(at);
#pragma unroll
        for (uint32_t j = 0; j < VEC; ++j) {
          const float y = to_float<T>(v, j);
          if (y >= least && at + j < many) {
            const uint32_t to = atomicAdd(&listed, 1u);
            if (to < kList) l.value[to] = key_of(y, first + at + j);
          }
        }
      }
    }
    __syncthreads();
    const uint32_t n = listed;
    if (time + 1 < times) {  // room for the next round, and a better bound
      if (n > 2 * a.keep && n <= kList) {
        const uint32_t left = thin<kThreads>(l, nullptr, numbers, waves, n, a.keep);
        const uint32_t b = waves[0];
        if (b > ordered(least)) least = unordered(b);
        __syncthreads();
        if (!t) listed = left;
      }
      __syncthreads();
    }
  }
  // The threads' sums, from the largest of what they are taken from.
  float high = unordered(max_of_wave(ordered(ref)));
  if (!lane) tops[wave] = high;
  __syncthreads();
  high = tops[0];
#pragma unroll
  for (uint32_t i = 1; i < kWaves; ++i) high = fmaxf(high, tops[i]);
  if (near()) sum /= exp_of(ref, magic);
  if (ref > -INFINITY) sum *= power_below(ref, high);
  if (bad) sum = NAN;
  sum = sum_of_wave(sum);
  if (!lane) sums[wave] = sum;
  uint32_t n = listed;
  __syncthreads();
  const uint64_t part = static_cast<uint64_t>(row) * a.splits + split;
  if (!t) {
    double add = sums[0];
#pragma unroll
    for (uint32_t i = 1; i < kWaves; ++i) add += sums[i];
    a.part_max[part] = high;
    a.part_sum[part] = add;
  }
  if (n > kList) {  // careful: each time the list of the best so far and what beats its last one
    n = 0;
    least = kLeast;
    load(0);
#pragma unroll 1
    for (uint32_t time = 0; time < times; ++time) {
      arrive(time);
      if (!t) listed = n;
      __syncthreads();
#pragma unroll
      for (uint32_t i = 0; i < kPer; ++i)
        if (x[i] >= least) {
          const uint32_t to = atomicAdd(&listed, 1u);
          if (to < kList) l.value[to] = key_at(time, i);
        }
      __syncthreads();
      uint32_t have = listed;
      __syncthreads();
      if (have > kList) {  // of these logits the largest key that at least `keep` reach, which are then exactly so many
        uint64_t key = 0;
#pragma unroll 1
        for (int bit = 63; bit >= 0; --bit) {
          const uint64_t next = key | 1ull << bit;
          if (count_of<kPer>(waves, [&](int i) { return x[i] >= kLeast && key_at(time, i) >= next; }) >= a.keep) key = next;
        }
        if (!t) listed = n;
        __syncthreads();
#pragma unroll
        for (uint32_t i = 0; i < kPer; ++i)
          if (x[i] >= kLeast && key_at(time, i) >= key) l.value[atomicAdd(&listed, 1u)] = key_at(time, i);
        __syncthreads();
        have = listed;
      }
      if (have <= n) continue;  // nothing new
      rank_list<kThreads, false>(l, nullptr, have);
      uint64_t mine[kList / kThreads];
      uint32_t rank[kList / kThreads];
#pragma unroll
      for (uint32_t i = 0; i < kList / kThreads; ++i) {
        rank[i] = kList;
        if (i * kThreads + t < have) mine[i] = l.value[i * kThreads + t], rank[i] = l.rank[i * kThreads + t];
      }
      __syncthreads();
#pragma unroll
      for (uint32_t i = 0; i < kList / kThreads; ++i)
        if (rank[i] < a.keep) l.value[rank[i]] = mine[i];
      n = have < a.keep ? have : a.keep;
      __syncthreads();
      // Equal ones of lower tokens may follow: they beat the last one too.
      if (n == a.keep) least = unordered(static_cast<uint32_t>(l.value[n - 1] >> 32));
    }
  } else if (n > kOpsWave && n > a.keep + a.keep / 2) {
    n = thin<kThreads>(l, nullptr, numbers, waves, n, a.keep);
  }
  rank_list<kThreads, false>(l, nullptr, n);
  uint64_t* const out = a.lists + part * a.keep;
  for (uint32_t i = t; i < n; i += kThreads)
    if (l.rank[i] < a.keep) out[l.rank[i]] = l.value[i];
  for (uint32_t i = n + t; i < a.keep; i += kThreads) out[i] = 0;
}

// A thread's share of n keys in descending lists of `keep`, side by side; `lists` of them are a beam's.
struct Keys {
  uint64_t v[kMergePer];
  uint32_t at, has;  // the place of the first one, and how many
  uint32_t threads;  // that have some
  uint32_t starts;   // bit i: the i-th is the first of a list, or of the thread's
  uint32_t beam, more;  // of the first one; bit i: the i-th is of the next
  __device__ __forceinline__ Keys(const uint64_t* from, uint32_t n, uint32_t keep, uint32_t lists) {
    const uint32_t per = (n + kMerge - 1) / kMerge;
    at = threadIdx.x * per;
    threads = (n + per - 1) / per;
    has = at >= n ? 0 : n - at < per ? n - at : per;
#pragma unroll
    for (uint32_t i = 0; i < kMergePer; ++i) {
      v[i] = 0;
      if (i < has) v[i] = from[at + i];
    }
    uint32_t list = at / keep, in = at - list * keep;
    beam = list / lists;
    list -= beam * lists;
    starts = 1;
    more = 0;
    for (uint32_t i = 1; i < per; ++i) {
      if (++in < keep) continue;
      in = 0;
      starts |= 1u << i;
      if (++list < lists) continue;
      list = 0;
      more |= 1u << i;
    }
  }
  __device__ __forceinline__ uint32_t beam_of(uint32_t i) const { return beam + __popc(more & ((2u << i) - 1)); }
};

// The `keep` best of the threads' keys; value(i) is what counts of a thread's i-th (0: none), descending within a list. Ties go
// to the lower place, which is the lower beam, the larger logit and the lower token, as long as equal values of a beam have equal
// logits. Where rounding may have made other logits' values equal (TIES; near_zero(i), and give says so of what it is given), they
// go by order(place), lower ones first, and are given once more. Found as in beam_part_kernel: as many of the threads' largest,
// which are their lists' first ones, reach a bound; of a list only what comes before the first value below it is looked at; and
// where a few lists hold most of the best, so that much more does reach it, what was found is thinned once more before it is
// ranked (32 beams of 4 parts of 64, scores apart by 6: 78 us without). give(rank, value, place); returns how many there are.
template <bool TIES, class V, class Z, class O, class F>
__device__ __forceinline__ uint32_t best_of(const Keys& k, uint32_t keep, V value, Z near_zero, O order, F give) {
  __shared__ List<kMergeList> l;
  __shared__ __attribute__((aligned(16))) uint32_t numbers[kMergeList];
  __shared__ uint32_t places[kMergeList + 8], waves[kMerge / kOpsWave], bound, listed, merged;
  const uint32_t t = threadIdx.x;
  if (!t) listed = merged = 0;
  uint64_t top = 0;
#pragma unroll
  for (uint32_t i = 0; i < kMergePer; ++i)
    if (i < k.has && k.starts >> i & 1) {
      const uint64_t v = value(i);
      top = v > top ? v : top;
    }
  numbers[t] = static_cast<uint32_t>(top >> 32);
  __syncthreads();
  if (t < kOpsWave) {
    const uint32_t b = k.threads <= 256 ? bound_of<256>(numbers, keep) : k.threads <= 512 ? bound_of<512>(numbers, keep) : bound_of<kMerge>(numbers, keep);
    if (!t) bound = b;
  }
  __syncthreads();
  const uint64_t least = bound ? static_cast<uint64_t>(bound) << 32 : 1;
  bool before = true;  // whether the value before in the list reached the bound
#pragma unroll
  for (uint32_t i = 0; i < kMergePer; ++i) {
    const bool look = i < k.has && (before || (k.starts >> i & 1));
    if (!__any(look)) continue;
    const uint64_t v = look ? value(i) : 0;
    before = v >= least;
    if (before) {
      const uint32_t to = atomicAdd(&listed, 1u);
      if (to < kMergeList) l.value[to] = v, places[to] = k.at + i;
    }
  }
  __syncthreads();
  uint32_t n = listed;
  if (n > kMergeList) {  // of many equal ones: the bound bit by bit over all
    uint64_t is[kMergePer];
#pragma unroll
    for (uint32_t i = 0; i < kMergePer; ++i) is[i] = i < k.has ? value(i) : 0;
    uint64_t key = 0;
#pragma unroll 1
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t next = key | 1ull << bit;
      if (count_of<kMergePer>(waves, [&](int i) { return is[i] >= next; }) >= keep) key = next;
    }
    // All above it, and of those that equal it the lowest places, or by order, up to `until`.
    const uint32_t more = keep - count_of<kMergePer>(waves, [&](int i) { return is[i] > key; });
    uint32_t equal = 0, close = 0;
#pragma unroll
    for (uint32_t i = 0; i < kMergePer; ++i) {
      equal |= (is[i] == key ? 1u : 0u) << i;
      if constexpr (TIES) close |= is[i] == key && near_zero(i) ? 1 : 0;
    }
    const bool by_order = TIES && sum_of_waves(waves, __any(close));
    const auto place = [&](uint32_t i) -> uint64_t {
      if constexpr (TIES)
        if (by_order) return order(k.at + i);
      return k.at + i;
    };
    uint64_t until = 0;
#pragma unroll 1
    for (uint64_t bit = by_order ? 1ull << (kOrderBits - 1) : kBeamMerge / 2; bit; bit /= 2) {
      uint32_t lower = 0;
#pragma unroll 1
      for (uint32_t rest = equal; rest; rest &= rest - 1) lower += place(__builtin_ctz(rest)) < until + bit ? 1 : 0;
      if (sum_of_waves(waves, over_wave(lower, [](uint32_t x, uint32_t y) { return x + y; })) < more) until += bit;
    }
    __syncthreads();
    if (!t) listed = 0;
    __syncthreads();
    const auto add = [&](uint64_t v, uint32_t i) {
      const uint32_t to = atomicAdd(&listed, 1u);
      if (to < kMergeList) l.value[to] = v, places[to] = k.at + i;
    };
#pragma unroll
    for (uint32_t i = 0; i < kMergePer; ++i)
      if (is[i] > key) add(is[i], i);
#pragma unroll 1
    for (uint32_t rest = equal; rest; rest &= rest - 1)
      if (place(__builtin_ctz(rest)) <= until) add(key, __builtin_ctz(rest));
    __syncthreads();
    n = listed;
  }
  if (n > 2 * keep + 64) n = thin<kMerge>(l, places, numbers, waves, n, keep);
  constexpr uint32_t kMine = (kMergeList + kMerge - 1) / kMerge;
  uint32_t at[kMine];
  uint64_t v[kMine];
#pragma unroll 1
  for (uint32_t pass = 0;; ++pass) {  // by place; where that may not do, by order, whose ranks then take the places' place
    rank_list<kMerge, true>(l, places, n);
    if (pass != 1) {
      bool close = false;
#pragma unroll
      for (uint32_t i = 0; i < kMine; ++i) {
        const uint32_t c = i * kMerge + t;
        if (c < n && l.rank[c] < keep) close |= give(l.rank[c], l.value[c], pass ? at[i] : places[c]);
      }
      if (!TIES || pass) break;
      if (close) merged = 1;
      __syncthreads();
      if (!merged) break;
    }
#pragma unroll
    for (uint32_t i = 0; i < kMine; ++i) {
      const uint32_t c = i * kMerge + t;
      if (c >= n) continue;
      if (pass) {
        l.value[c] = v[i];
        places[c] = l.rank[c];
      } else {
        v[i] = l.value[c];
        at[i] = places[c];
        if constexpr (TIES) l.value[c] = ~order(at[i]);
      }
    }
    __syncthreads();
  }
  return n < keep ? n : keep;
}

// The best of a row's parts.
__global__ __launch_bounds__(kMerge) void beam_row_kernel(BeamArgs a) {
  const uint32_t row = blockIdx.x, n = a.splits * a.keep, t = threadIdx.x;
  if (!grows(a, row)) return;
  const Keys k(a.lists + static_cast<uint64_t>(row) * n, n, a.keep, a.splits);
  uint64_t* const out = a.rows + static_cast<uint64_t>(row) * a.keep;
  const uint32_t found = best_of<false>(k, a.keep, [&](uint32_t i) { return k.v[i]; }, nullptr, nullptr,
                                        [&](uint32_t rank, uint64_t key, uint32_t) {
                                          out[rank] = key;
                                          return false;
                                        });
  for (uint32_t i = found + t; i < a.keep; i += kMerge) out[i] = 0;
}

// A request: of each beam log-sum-exp of its parts, then the best over all.
// 24 requests of 640 keys 10.7 us, 8 of 8192 18.2: a chain of loads, the log, the bound, the list and the ranks, a barrier after each.
__global__ __launch_bounds__(kMerge) void beam_merge_kernel(BeamArgs a) {
  __shared__ double scores[kBeamMost], lses[kBeamMost];
  // Two logits x < y of a beam have one value only where 2^-24 |x|, the least that x and y are apart, is no more than v's two
  // roundings, 2^-53 of |x - lse| and of |v| each, make of both: |x| and |y| then are below 2^-27 (|score| + |lse|). Twice that.
  __shared__ float near[kBeamMost];
  __shared__ uint8_t state[kBeamMost];  // 0: no candidates, 1: from its logits, 2: done
  const uint32_t item = blockIdx.x, t = threadIdx.x;
  constexpr uint32_t kLanes = kMerge / kBeamMost;  // of a beam
  const uint32_t per = a.rows ? a.keep : a.splits * a.keep, n = a.beams * per;  // candidates of a beam, of all
  const uint64_t* const from = (a.rows ? a.rows : a.lists) + static_cast<uint64_t>(item) * n;
  const Keys k(from, n, a.keep, a.rows ? 1 : a.splits);  // lists of beams that have none hold anything
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
        return sum * (max > -INFINITY ? power_below(max, top) : 1.0);
      };
      double sum = part(m0, s0);
      for (uint32_t i = lane + kLanes; i < a.splits; i += kLanes) sum += part(m[i], s[i]);
      static_assert(kLanes == 16, "");
      sum = sum_of_row(sum);
      if (!(sum > 0)) is = 0;  // no logit above -infinity, or one that is no number or +infinity
      lse = top + log(sum);
    }
    if (!lane) {
      scores[beam] = score;
      lses[beam] = lse;
      state[beam] = is;
      near[beam] = is == 1 ? static_cast<float>(0x1p-26 * (fabs(score) + fabs(lse))) : -1.0f;
    }
  }
  __syncthreads();
  const auto value = [&](uint32_t i) -> uint64_t {
    const uint32_t beam = k.beam_of(i), is = state[beam];
    if (is == 1 && k.v[i]) return ordered(scores[beam] + (unordered(static_cast<uint32_t>(k.v[i] >> 32)) - lses[beam]) + 0.0);
    return is == 2 && k.at + i == beam * per ? ordered(scores[beam] + 0.0) : 0;
  };
  const auto close = [&](uint32_t beam, uint64_t key) { return fabsf(unordered(static_cast<uint32_t>(key >> 32))) <= near[beam]; };
  const auto near_zero = [&](uint32_t i) { return close(k.beam_of(i), k.v[i]); };
  const auto order = [&](uint32_t place) -> uint64_t {  // beam, the logit's complement, place
    const uint32_t beam = place / per, logit = state[beam] == 1 ? static_cast<uint32_t>(from[place] >> 32) : 0;
    return static_cast<uint64_t>(beam) << 46 | static_cast<uint64_t>(~logit) << 14 | place;
  };
  static_assert(kBeamMerge == 1u << 14 && kBeamMost <= 64 && kOrderBits == 52, "");
  const uint64_t to = static_cast<uint64_t>(item) * a.keep;
  const uint32_t found = best_of<true>(k, a.keep, value, near_zero, order, [&](uint32_t rank, uint64_t v, uint32_t at) {
    const uint32_t beam = at / per;
    const uint64_t key = from[at];
    a.tokens[to + rank] = state[beam] == 2 ? a.done_token : static_cast<int32_t>(0xffffffffu - static_cast<uint32_t>(key));
    a.parents[to + rank] = static_cast<int32_t>(item * a.beams + beam);
    a.scores_out[to + rank] = static_cast<float>(unordered(v));
    return close(beam, key);
  });
  for (uint32_t i = found + t; i < a.keep; i += kMerge) {
    a.tokens[to + i] = a.parents[to + i] = -1;
    a.scores_out[to + i] = -INFINITY;
  }
}

}  // namespace

hipError_t launch_beam(const BeamArgs& a, uint32_t type, hipStream_t stream) {
  const uint32_t rows = a.batch * a.beams, grid = rows * a.splits;
  hipError_t e = type == MMA_TYPE_F32   ? launch(beam_part_kernel<float>, grid, kThreads, stream, a)
                 : type == MMA_TYPE_F16 ? launch(beam_part_kernel<_Float16>, grid, kThreads, stream, a)
                                        : launch(beam_part_kernel<__bf16>, grid, kThreads, stream, a);
  if (e != hipSuccess) return e;
  if (a.rows && (e = launch(beam_row_kernel, rows, kMerge, stream, a)) != hipSuccess) return e;
  return launch(beam_merge_kernel, a.batch, kMerge, stream, a);
}

}  // namespace mma
