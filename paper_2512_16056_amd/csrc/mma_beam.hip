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

constexpr uint32_t kThreads = 256;
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
  const uint64_t b = __builtin_bit_cast(uint64_t, p) + (__builtin_bit_cast(uint64_t, t) << 52);  // times 2^n
  return __builtin_bit_cast(double, b);
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

// The value of rank `keep` - 1 of 256 in LDS, the largest first: as many different threads hold one at least as large.
template <class H>
__device__ __forceinline__ void bound_of(const H* h, uint32_t keep, H* bound) {
  if (threadIdx.x < 256) {
    const H mine = h[threadIdx.x];
    uint32_t rank = 0;
#pragma unroll 16
    for (uint32_t i = 0; i < 256; ++i) {
      const H x = h[i];
      rank += x > mine || (x == mine && i < threadIdx.x) ? 1 : 0;
    }
    if (rank == keep - 1) *bound = mine;
  }
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
// The `keep` best: the keep-th largest of the threads' maxima bounds them from below, since as many threads hold one
// as large; what reaches it (few more than keep) goes to a list, whose entries rank themselves. Where more reach it
// than the list holds, as of many equal logits, the bound is found bit by bit instead.
template <class T>
__global__ __launch_bounds__(kThreads) void beam_chunk_kernel(BeamArgs a) {
  constexpr uint32_t VEC = 16 / sizeof(T), NC = kPer / VEC;
  __shared__ uint64_t list[kList];
  __shared__ float maxima[kThreads], bound;
  __shared__ double sums[kThreads / kOpsWave];
  __shared__ uint32_t waves[kThreads / kOpsWave], listed;
  const uint32_t row = blockIdx.x / a.splits, split = blockIdx.x % a.splits, t = threadIdx.x;
  if (!grows(a, row)) return;  // the merge does not read its part
  const uint64_t start = reinterpret_cast<uint64_t>(a.logits) + row * a.row_bytes;
  const uint32_t ahead = static_cast<uint32_t>(start % 16) / sizeof(T);  // elements between there and the row's start
  const T* const from = reinterpret_cast<const T*>(start & ~15ull);
  const uint64_t first = static_cast<uint64_t>(split) * kBeamChunk, end = static_cast<uint64_t>(a.vocab) + ahead;
  u32x4 w[NC];
#pragma unroll
  for (uint32_t i = 0; i < NC; ++i) {
    const uint64_t v = first + (i * kThreads + t) * VEC;
    w[i] = v < end ? *reinterpret_cast<const u32x4*>(from + v) : u32x4{0, 0, 0, 0};
  }
  float x[kPer], top = -INFINITY;
  bool bad = false;
#pragma unroll
  for (uint32_t i = 0; i < kPer; ++i) {
    const uint64_t v = first + (i / VEC * kThreads + t) * VEC + i % VEC;
    const float y = to_float<T>(w[i / VEC], i % VEC) + 0.0f;
    x[i] = v >= ahead && v < end ? y : -INFINITY;
    bad = bad || x[i] != x[i] || x[i] == INFINITY;
    top = fmaxf(top, x[i]);
  }
  const auto token_of = [&](uint32_t i) {
    return static_cast<uint32_t>(first + (i / VEC * kThreads + t) * VEC + i % VEC - ahead);
  };
  maxima[t] = top;
  if (!t) listed = 0;
  __syncthreads();
  float all = top;
  {
    float m = max_of_wave(top);
    if (t % kOpsWave == 0) sums[t / kOpsWave] = m;
    bound_of(maxima, a.keep, &bound);
    __syncthreads();
    all = fmaxf(fmaxf(sums[0], sums[1]), fmaxf(sums[2], sums[3]));
  }
  const float least = bound;
  __syncthreads();

  // The sum, from the chunk's maximum. Logits far below it count for e^-600, nothing.
  double sum = 0;
  if (all > -INFINITY) {
    const float floor = all - 600.0f;
    const double from_top = all;
#pragma unroll
    for (uint32_t i = 0; i < kPer; ++i) sum += exp_of(static_cast<double>(fmaxf(x[i], floor)) - from_top);
  }
  if (bad) sum = NAN;
  sum = sum_of_wave(sum);
  if (t % kOpsWave == 0) sums[t / kOpsWave] = sum;

  // The candidates.
  if (top >= least && top > -INFINITY) {
#pragma unroll
    for (uint32_t i = 0; i < kPer; ++i)
      if (x[i] >= least && x[i] > -INFINITY) {
        const uint32_t at = atomicAdd(&listed, 1u);
        if (at < kList) list[at] = key_of(x[i], token_of(i));
      }
  }
  __syncthreads();
  const uint64_t part = static_cast<uint64_t>(row) * a.splits + split;
  if (!t) {
    a.part_max[part] = all;
    a.part_sum[part] = sums[0] + sums[1] + sums[2] + sums[3];
  }
  uint32_t n = listed;
  if (n > kList) {  // the largest key that at least `keep` candidates reach, which are then exactly so many
    uint64_t key = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t next = key | 1ull << bit;
      if (count_of<kPer>(waves, [&](int i) { return x[i] > -INFINITY && key_of(x[i], token_of(i)) >= next; }) >= a.keep) key = next;
    }
    __syncthreads();
    if (!t) listed = 0;
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < kPer; ++i)
      if (x[i] > -INFINITY && key_of(x[i], token_of(i)) >= key) list[atomicAdd(&listed, 1u)] = key_of(x[i], token_of(i));
    __syncthreads();
    n = listed;
  }
  uint64_t* const out = a.lists + part * a.keep;
  for (uint32_t i = t; i < n; i += kThreads) {
    const uint64_t mine = list[i];
    uint32_t rank = 0;
    for (uint32_t j = 0; j < n; ++j) rank += list[j] > mine ? 1 : 0;
    if (rank < a.keep) out[rank] = mine;
  }
  for (uint32_t i = n + t; i < a.keep; i += kThreads) out[i] = 0;
}

// The `keep` best of up to 16 values of each of 1024 threads (0: none), ties to the lower place i * 1024 + thread: found as
// in beam_chunk_kernel, with the maxima of four threads each. give(rank, value, place); returns how many there are.
template <class F>
__device__ __forceinline__ uint32_t best_of(const uint64_t (&v)[kMergePer], uint32_t keep, F give) {
  __shared__ uint64_t list[kList];
  __shared__ uint32_t places[kList], maxima[256], waves[kMerge / kOpsWave], bound, listed;
  const uint32_t t = threadIdx.x;
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
  if (!t) listed = 0;
  __syncthreads();
  bound_of(maxima, keep, &bound);
  __syncthreads();
  uint64_t least = static_cast<uint64_t>(bound) << 32;
  if (!least) least = 1;
#pragma unroll
  for (uint32_t i = 0; i < kMergePer; ++i)
    if (v[i] >= least) {
      const uint32_t at = atomicAdd(&listed, 1u);
      if (at < kList) list[at] = v[i], places[at] = i * kMerge + t;
    }
  __syncthreads();
  uint32_t n = listed;
  if (n > kList) {
    uint64_t key = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t next = key | 1ull << bit;
      if (count_of<kMergePer>(waves, [&](int i) { return v[i] >= next; }) >= keep) key = next;
    }
    // All above it, and of those that equal it the lowest places: below the smallest `until` that leaves enough of them.
    const uint32_t more = keep - count_of<kMergePer>(waves, [&](int i) { return v[i] > key; });
    uint32_t until = 0;
    for (uint32_t bit = kBeamMerge; bit; bit /= 2) {
      const uint32_t next = until + bit;
      if (next <= kBeamMerge && count_of<kMergePer>(waves, [&](int i) { return v[i] == key && i * kMerge + t < next; }) < more) until = next;
    }
    __syncthreads();
    if (!t) listed = 0;
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < kMergePer; ++i)
      if (v[i] > key || (v[i] == key && i * kMerge + t <= until)) {
        const uint32_t at = atomicAdd(&listed, 1u);
        if (at < kList) list[at] = v[i], places[at] = i * kMerge + t;
      }
    __syncthreads();
    n = listed;
  }
  for (uint32_t i = t; i < n; i += kMerge) {
    const uint64_t mine = list[i];
    const uint32_t place = places[i];
    uint32_t rank = 0;
    for (uint32_t j = 0; j < n; ++j) rank += list[j] > mine || (list[j] == mine && places[j] < place) ? 1 : 0;
    if (rank < keep) give(rank, mine, place);
  }
  return n < keep ? n : keep;
}

// The best of a row's parts.
__global__ __launch_bounds__(kMerge) void beam_row_kernel(BeamArgs a) {
  const uint32_t row = blockIdx.x, n = a.splits * a.keep, t = threadIdx.x;
  if (!grows(a, row)) return;
  const uint64_t* from = a.lists + static_cast<uint64_t>(row) * n;
  uint64_t v[kMergePer];
#pragma unroll
  for (uint32_t i = 0; i < kMergePer; ++i) v[i] = i * kMerge + t < n ? from[i * kMerge + t] : 0;
  uint64_t* const out = a.rows + static_cast<uint64_t>(row) * a.keep;
  const uint32_t found = best_of(v, a.keep, [&](uint32_t rank, uint64_t key, uint32_t) { out[rank] = key; });
  for (uint32_t i = found + t; i < a.keep; i += kMerge) out[i] = 0;
}

// A request: of each beam log-sum-exp of its parts, then the best over all.
__global__ __launch_bounds__(kMerge) void beam_merge_kernel(BeamArgs a) {
  __shared__ double scores[kBeamMost], lses[kBeamMost];
  __shared__ uint8_t state[kBeamMost];  // 0: no candidates, 1: from its logits, 2: done
  const uint32_t item = blockIdx.x, t = threadIdx.x, lane = t % kOpsWave;
  for (uint32_t beam = t / kOpsWave; beam < a.beams; beam += kMerge / kOpsWave) {
    const uint32_t row = item * a.beams + beam;
    uint8_t is = !finite(a.scores[row]) ? 0 : a.done && a.done[row] ? 2 : 1;
    double lse = 0;
    if (is == 1) {
      const float* m = a.part_max + static_cast<uint64_t>(row) * a.splits;
      const double* s = a.part_sum + static_cast<uint64_t>(row) * a.splits;
      float top = -INFINITY;
      for (uint32_t i = lane; i < a.splits; i += kOpsWave) top = fmaxf(top, m[i]);
      top = max_of_wave(top);
      double sum = 0;
      for (uint32_t i = lane; i < a.splits; i += kOpsWave) {
        const double from_top = static_cast<double>(m[i]) - top;
        sum += s[i] * (m[i] > -INFINITY ? exp(from_top) : 0.0);
      }
      sum = sum_of_wave(sum);
      if (!(sum > 0)) is = 0;  // no logit above -infinity, or one that is no number or +infinity
      lse = top + log(sum);
    }
    if (!lane) {
      scores[beam] = a.scores[row];
      lses[beam] = lse;
      state[beam] = is;
    }
  }
  __syncthreads();
  const uint64_t* const lists = a.rows ? a.rows : a.lists;
  const uint32_t per = a.rows ? a.keep : a.splits * a.keep, n = a.beams * per;  // candidates of a beam, of all
  const uint64_t* const from = lists + static_cast<uint64_t>(item) * n;
  uint64_t v[kMergePer];
#pragma unroll
  for (uint32_t i = 0; i < kMergePer; ++i) {
    const uint32_t at = i * kMerge + t;
    v[i] = 0;
    if (at >= n) continue;
    const uint32_t beam = at / per;
    if (state[beam] == 1) {
      const uint64_t key = from[at];
      if (key) v[i] = ordered(scores[beam] + (unordered(static_cast<uint32_t>(key >> 32)) - lses[beam]) + 0.0);
    } else if (state[beam] == 2 && at % per == 0) {
      v[i] = ordered(scores[beam] + 0.0);
    }
  }
  const uint64_t to = static_cast<uint64_t>(item) * a.keep;
  const uint32_t found = best_of(v, a.keep, [&](uint32_t rank, uint64_t value, uint32_t at) {
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
