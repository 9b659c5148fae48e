// Attention over the paged KV cache for gfx950 (MI355X): one token, a tree of drafted
// ones or a prompt chunk of each sequence against its entries, read where they lie.
//
// Notation: a "row" is one token and one query head of a KV head's group, so a KV head
// of one sequence has (tokens x group) rows, all of them over the same keys and values;
// they go in tiles of 16, the width of a matrix instruction. Entries go in tiles of 32.
//
// Of a tile the kernel forms S^T = K Q^T (keys down, rows across) with
// v_mfma_f32_16x16x32: lane (g, m), g = lane / 16, m = lane % 16, gives key row m, 8
// consecutive values of the head at 8 g, and gets 4 keys of query row m. The order of keys
// down a tile is free, so the two 16-key halves take keys 8 (m / 4) + m % 4 and + 4: then
// lane (g, m) holds the 8 consecutive keys 8 g .. 8 g + 7 of row m, which is the operand
// P^T of O^T = V^T P^T as it stands. Probabilities never change lanes, maxima and sums of
// a row are a lane's own but for two exchanges between its 4 lanes, and a lane's 8 keys lie
// in one block (if blocks hold a multiple of 8). The same holds for the head's values in
// Q K^T, which is what lets 8-bit keys be read 16 bytes at a time.
//
// Two kernels share that arithmetic. attention_stream_kernel, for up to 32 rows, reads keys
// and values from memory straight into the registers of the instructions; its waves split the
// entries. attention_rows_kernel, for more rows and for long 16-bit contexts, brings tiles to
// LDS once for the workgroup's 64 or 128 rows; its waves split the rows. Which of them takes a
// call, and in how many splits, is attention_plan's choice (mma_ops.cpp).
#include "mma_ops.h"

#include <algorithm>
#include <type_traits>

namespace mma {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr uint32_t kTile = 32;    // entries
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kLowest = -3.0e38f;  // maximum of a row that has seen nothing: finite, so that differences are numbers

template <class T>
struct Type;
template <>
struct Type<__bf16> {
  typedef bf16x8 x8;
  static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {  // round to nearest even
    const f32x2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
  }
  // Numbers from 0 on as the sum of two of 16 bits: the first cut off, the second what is left, and above 0 with the
  // number, so that an infinity times the two is no NaN.
  static __device__ __forceinline__ uint32_t split(float a, float b, uint32_t* rest) {
    const uint32_t x = __builtin_bit_cast(uint32_t, a), y = __builtin_bit_cast(uint32_t, b);
    *rest = pack(fmaxf(a - __builtin_bit_cast(float, x & 0xffff0000u), a * 0x1p-24f),
                 fmaxf(b - __builtin_bit_cast(float, y & 0xffff0000u), b * 0x1p-24f));
    return __builtin_amdgcn_perm(y, x, 0x07060302u);
  }
  static __device__ __forceinline__ uint32_t from_f8(uint32_t w, bool high) {  // exact
    return high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true))
                : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
  }
  static constexpr uint32_t kExponent = 0x7f80;
  static constexpr float kLift = 0, kRowsLift = 0, kRowsRoom = 8;
};
template <>
struct Type<_Float16> {
  typedef f16x8 x8;
  static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const f32x2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
  }
  static __device__ __forceinline__ uint32_t split(float a, float b, uint32_t* rest) {
    const auto cut = __builtin_amdgcn_cvt_pkrtz(a, b);
    *rest = pack(fmaxf(a - static_cast<float>(cut[0]), fminf(a, 0x1p-24f)),  // the least that there is
                 fmaxf(b - static_cast<float>(cut[1]), fminf(b, 0x1p-24f)));
    return __builtin_bit_cast(uint32_t, cut);
  }
  static __device__ __forceinline__ uint32_t from_f8(uint32_t w, bool high) {
    return high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true))
                : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false));
  }
  static constexpr uint32_t kExponent = 0x7c00;
  // f16 has normal numbers from 2^-14 on and nothing below 2^-25, and the many small weights of a long context beside a
  // few large ones are smaller. So p is held (and summed) times 2^kLift, below the largest number, 2^16.
  static constexpr float kLift = 15, kRowsLift = 11, kRowsRoom = 15;
};

// What V and the probabilities are multiplied in: 8-bit values are exact in f16, whose 11 bits lose less of p than bf16's 8.
template <class T, bool F8>
using ValueType = typename std::conditional<F8, _Float16, T>::type;

template <class T>
__device__ __forceinline__ float to_float(uint32_t bits16) {
  return static_cast<float>(__builtin_bit_cast(T, static_cast<uint16_t>(bits16)));
}

__device__ __forceinline__ float across(float v, int mask) { return __shfl_xor(v, mask, kOpsWave); }

// Maximum and sum over the 4 lanes that have a row's keys (16 and 32 apart), by exchanging rows of lanes between two
// registers instead of through LDS.
__device__ __forceinline__ float max_of_row(float v) {
  uint32_t x = __builtin_bit_cast(uint32_t, v);
  auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, static_cast<uint32_t>(a[0])), __builtin_bit_cast(float, static_cast<uint32_t>(a[1]))));
  a = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return fmaxf(__builtin_bit_cast(float, static_cast<uint32_t>(a[0])), __builtin_bit_cast(float, static_cast<uint32_t>(a[1])));
}

// 8 consecutive values of one row from global memory, elements at any alignment if not wide.
__device__ __forceinline__ u32x4 load_row8(const uint8_t* p, bool wide) {
  if (wide) return *reinterpret_cast<const u32x4*>(p);
  const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = h[2 * i] | (static_cast<uint32_t>(h[2 * i + 1]) << 16);
  return r;
}

// Q of 16 rows as the second operand of K Q^T. The head values of instruction s of lane
// group g start at 32 s + 8 g, or where 8-bit keys are in registers at 64 (s / 2) + 16 g + 8 (s % 2).
template <bool PAIRED, int KS>
__device__ __forceinline__ void load_q(const AttnArgs& a, uint32_t head, uint32_t token, bool live, uint32_t g, u32x4* q) {
  const uint8_t* p = a.q.data + 2 * (token * a.q.token + head * a.q.head);
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const uint32_t d = PAIRED ? (s / 2) * 64 + g * 16 + (s % 2) * 8 : s * 32 + g * 8;
    q[s] = live && d < a.c.dim ? load_row8(p + 2 * d, a.wide_q) : u32x4{0, 0, 0, 0};
  }
}

template <class T>
__device__ __forceinline__ u32x4 widen(uint32_t x, uint32_t y) {  // 8 values of 8 bits to 16 bits
  return u32x4{Type<T>::from_f8(x, false), Type<T>::from_f8(x, true), Type<T>::from_f8(y, false), Type<T>::from_f8(y, true)};
}

// Bit j: entry first + j, below `end`, has a block.
__device__ __forceinline__ uint32_t keys_there(const CacheArgs& c, const int32_t* row, uint32_t first, uint32_t end) {
  uint32_t ok = 0, token;
  if (c.tokens % 8 == 0) {
    if (first < end && block_at(c, row, first, &token) >= 0)
      ok = end - first >= 8 ? 0xffu : (1u << (end - first)) - 1;
    return ok;
  }
  for (uint32_t j = 0; j < 8 && first + j < end; ++j)
    if (block_at(c, row, first + j, &token) >= 0) ok |= 1u << j;
  return ok;
}

// Bit j: token `token` of a sequence (row `first` + token of the call) sees entry key + j.
__device__ __forceinline__ uint32_t keys_seen(const AttnArgs& a, const SeqSpan& sp, uint32_t token, uint32_t key) {
  const int32_t d = static_cast<int32_t>(key) - static_cast<int32_t>(sp.before);  // the first key's token, below 0 for the context
  if (d <= -8) return 0xff;
  if (!a.tree) {
    const int32_t n = static_cast<int32_t>(token) + 1 - d;  // keys up to its own
    return n >= 8 ? 0xffu : n <= 0 ? 0u : (1u << n) - 1;
  }
  const uint64_t* bits = a.tree + static_cast<uint64_t>(sp.first + token) * a.tree_words;
  const uint32_t from = d < 0 ? 0 : d, word = from / 64, shift = from % 64;
  uint64_t w = word < a.tree_words ? bits[word] >> shift : 0;
  if (shift > 56 && word + 1 < a.tree_words) w |= bits[word + 1] << (64 - shift);
  return d < 0 ? ((static_cast<uint32_t>(w) << -d) | ((1u << -d) - 1)) & 0xff : static_cast<uint32_t>(w) & 0xff;
}

// 16-bit halves of an operand whose keys' bits are set; the others 0.
__device__ __forceinline__ u32x4 only_keys(u32x4 w, uint32_t keys) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] &= (keys >> (2 * i) & 1 ? 0xffffu : 0u) | (keys >> (2 * i + 1) & 1 ? 0xffff0000u : 0u);
  return w;
}
// Bits of the keys whose value is infinite or NaN.
template <class T>
__device__ __forceinline__ uint32_t nonfinite_keys(u32x4 w) {
  uint32_t bad = 0;
  constexpr uint32_t x = Type<T>::kExponent;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    bad |= ((w[i] & x) == x ? 1u : 0u) << (2 * i) | ((w[i] >> 16 & x) == x ? 1u : 0u) << (2 * i + 1);
  return bad;
}

// O^T += V^T P^T over 32 keys: operand c of V^T from op(c); P in one term or two.
template <class T, int R, int NC, int TERMS, class Op>
__device__ __forceinline__ void add_values(Op op, const u32x4 (&p)[TERMS][R], f32x4 (&o)[R][NC]) {
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const u32x4 v = op(c);
#pragma unroll
    for (int t = 0; t < TERMS; ++t)
#pragma unroll
      for (int r = 0; r < R; ++r) o[r][c] = Type<T>::mfma(v, p[t][r], o[r][c]);
  }
}

// Probabilities y of 8 keys as the operand, in TERMS terms of 16 bits. Where a wave has one tile of rows, two: memory
// bounds it, and an error below 2^-15 of p (f16: 2^-21) costs 2 % at most (4 rows, 32 sequences of up to 8k, bf16, head-major: 124.5 us
// with one term, 125.6 with two). With two tiles one, rounded to nearest: 2^-8 of p in bf16, as the output is rounded,
// 2^-11 in f16 and over 8-bit caches. A second one would take a prompt of 2048 tokens behind 6144 entries, bf16, from 282
// us to 369, and 32 rows over 4 x 15k 8-bit x-packed entries, for lack of registers, from 32 to 38. The sum of p is of unrounded ones.
template <class T, int R, int TERMS>
__device__ __forceinline__ void operand_of(const float (&y)[8], u32x4 (&p)[TERMS][R], int r) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (TERMS == 2) {
      uint32_t rest;
      p[0][r][i] = Type<T>::split(y[2 * i], y[2 * i + 1], &rest);
      p[1][r][i] = rest;
    } else {
      p[0][r][i] = Type<T>::pack(y[2 * i], y[2 * i + 1]);
    }
  }
}

// The same where not every row sees every key: keys outside `ok` (stale ones in registers) count
// as 0, and an infinite or NaN value of a key reaches the rows that see the key, no others,
// though a product with a probability of 0 would bring NaN to all. Such keys are left out of the
// joint product and added one by one to the rows that see them.
template <class T, int R, int NC, int TERMS, class Op>
__device__ __forceinline__ void add_values_masked(Op op, const u32x4 (&p)[TERMS][R], const uint32_t (&seen)[R], uint32_t ok,
                                                  uint32_t g, uint32_t m, f32x4 (&o)[R][NC]) {
  uint32_t bad = 0;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    u32x4 v = only_keys(op(c), ok);
    const uint32_t n = nonfinite_keys<T>(v);
    bad |= n;
    v = only_keys(v, ~n);
#pragma unroll
    for (int t = 0; t < TERMS; ++t)
#pragma unroll
      for (int r = 0; r < R; ++r) o[r][c] = Type<T>::mfma(v, p[t][r], o[r][c]);
  }
  if (!__any(bad)) return;
  for (uint32_t j = 0; j < kTile; ++j) {
    if (!__any(g == j / 8 && (bad >> (j % 8) & 1))) continue;
    const uint32_t mine = g == j / 8 ? 1u << (j % 8) : 0u;
    uint32_t sees[R];
#pragma unroll
    for (int r = 0; r < R; ++r) sees[r] = __shfl(seen[r], (j / 8) * 16 + m, kOpsWave) >> (j % 8) & 1;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      u32x4 v = only_keys(op(c), mine & ok);
      v = only_keys(v, nonfinite_keys<T>(v));
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const f32x4 d = Type<T>::mfma(v, only_keys(p[0][r], mine), f32x4{0, 0, 0, 0});
#pragma unroll
        for (int i = 0; i < 4; ++i) o[r][c][i] = sees[r] ? o[r][c][i] + d[i] : o[r][c][i];
      }
    }
  }
}

// lse2 of a token's query head: rows of a KV head side by side.
__device__ __forceinline__ uint64_t lse2_at(const AttnArgs& a, uint32_t token, uint32_t qh) {
  return (static_cast<uint64_t>(qh / a.group) * a.s.num_tokens + token) * a.group + qh % a.group;
}

// What a row's result goes to: the output and lse, or with several splits this split's part of them.
// SIDE: a lane's 4 sums of an instruction are neighbours (value 16 c + 4 g); else the sums of CE instructions are, for
// each of the 4.
template <class T, int DP, int NC, int SIDE>
__device__ __forceinline__ void store_row(const AttnArgs& a, uint32_t token, uint32_t qh, uint32_t split, uint32_t g, float top,
                                          float sum, float v_scale, const f32x4 (&o)[NC]) {
  const uint64_t unit = static_cast<uint64_t>(token) * a.q_heads + qh;
  if (a.part_ml && !g) {
    float* ml = a.part_ml + 2 * (unit * a.splits + split);
    ml[0] = top;
    ml[1] = sum;
  }
  // The q-th four neighbours of the lane, and the head value of the first.
  const auto four = [&](int q) -> f32x4 {
    if constexpr (SIDE) return o[q];
    constexpr int CE = DP == 64 ? 4 : 8;
    const int i = q / (CE / 4) % 4, c = q / CE * CE + q % (CE / 4) * 4;
    return f32x4{o[c][i], o[c + 1][i], o[c + 2][i], o[c + 3][i]};
  };
  const auto value = [&](int q) -> uint32_t {
    if constexpr (SIDE) return q * 16 + g * 4;
    constexpr int CE = DP == 64 ? 4 : 8;
    return q / CE * 16 * CE + (g * 4 + q / (CE / 4) % 4) * CE + q % (CE / 4) * 4;
  };
  if (a.splits > 1) {
    float* to = a.part + (unit * a.splits + split) * DP;
#pragma unroll
    for (int q = 0; q < NC; ++q) *reinterpret_cast<f32x4*>(to + value(q)) = four(q) * v_scale;
    return;
  }
  const float by = sum == 0 ? 0.0f : v_scale / sum;
  T* to = reinterpret_cast<T*>(a.out.data) + token * a.out.token + qh * a.out.head;
#pragma unroll
  for (int q = 0; q < NC; ++q) {
    const f32x4 x = four(q) * by;
    const uint32_t d = value(q);
    if (d >= a.c.dim) continue;
    const u32x2 w = {Type<T>::pack(x[0], x[1]), Type<T>::pack(x[2], x[3])};
    if (a.wide_out) {
      *reinterpret_cast<u32x2*>(to + d) = w;
    } else {
      uint16_t* h = reinterpret_cast<uint16_t*>(to + d);
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] = static_cast<uint16_t>(w[i / 2] >> (i % 2 * 16));
    }
  }
  if (!g) {
    const float l2 = sum == 0 ? -INFINITY : top + __builtin_amdgcn_logf(sum);
    if (a.lse) a.lse[unit] = l2 * kLn2;
    if (a.lse2) a.lse2[lse2_at(a, token, qh)] = l2;
  }
}

// ---------------------------------------------------------------- few rows
// A workgroup has R tiles of rows of one sequence and KV head and one split of its
// entries; its 4 waves take the split's tiles in turn, each with its own running maximum
// and sum, and are joined in LDS at the end. Nothing is shared before that: a tile's
// bytes go from memory to the registers that the matrix instructions read. V^T comes as 8
// keys' rows of the lane's head values, turned in registers (v_perm), or from the x-packed
// layout, where 8 tokens of a value are contiguous, as it stands. Blocks hold a multiple of 8
// tokens here: a lane's keys of a tile and its values' keys are in one block each, whose
// table entries are read two tiles ahead, keys one tile ahead, values in the tile.
// Bound by the bytes in flight: its registers let two waves on a SIMD (a bound of three spilled: 32 sequences of 1k to 8k,
// 4 rows, heads of 128, x-packed, 179 us instead of 128 in bf16, 112 instead of 74 in 8 bits). 4 rows, one sequence of 64k
// entries, bf16, heads of 128, piece layout, logits kept: 63 us, 4.3 TB/s; the same entries of 8 bits, none kept, 32
// us with the join; 100 entries 7 us, the chain of loads from the length over the table to the entry.
template <bool F8, int DP, bool VX>
struct Stream {
  static constexpr int KS = DP / 32;                  // instructions of 32 head values
  static constexpr int NK = F8 ? KS / 2 : KS;         // 16-byte chunks of a key in one lane
  static constexpr int CE = DP == 64 ? 4 : 8;         // values of an entry's V in one lane and panel
  static constexpr int NP = DP / (16 * CE);           // panels
  static constexpr int NC = DP / 16;                  // instructions of 16 head values
  static constexpr int VW = VX ? (F8 ? 2 : 4) : CE / (F8 ? 4 : 2);  // dwords of a load of V
  static constexpr int NV = VX ? NC : NP * 8;                       // loads of V
  // Row r (0..15) of V^T of instruction c is head value 16 c + r (VX), else c / CE * 16 CE + r CE + c % CE.

  u32x4 k[2][NK];
  uint32_t v[NV][VW];

  // Loads have no conditions: lanes past head_dim read the row's start instead; their keys are then cleared, their
  // values come to nothing but outputs that are not stored.
  __device__ __forceinline__ void load_keys(const CacheArgs& c, int32_t id, uint32_t key, uint32_t head, uint32_t g) {
    const uint32_t token = key - block_of(c, key) * c.tokens;  // of the first half's key
    const uint8_t* p = c.k + static_cast<uint64_t>(static_cast<uint32_t>(id)) * c.block_bytes + head * c.k_head + token * c.k_token;
#pragma unroll
    for (int s = 0; s < NK; ++s) {
      const uint32_t chunk = s * 4 + g, at = chunk * (F8 ? 16 : 8) < c.dim ? chunk * c.k_chunk : 0;
#pragma unroll
      for (int t = 0; t < 2; ++t) k[t][s] = *reinterpret_cast<const u32x4*>(p + at + t * 4 * c.k_token);
    }
  }
  __device__ __forceinline__ void clear_keys(const CacheArgs& c, uint32_t g) {
    if (c.dim == DP) return;
#pragma unroll
    for (int s = 0; s < NK; ++s)
      if ((s * 4 + g) * (F8 ? 16 : 8) >= c.dim) k[0][s] = k[1][s] = u32x4{0, 0, 0, 0};
  }
  template <class T>
  __device__ __forceinline__ u32x4 key(int t, int s) const {
    if constexpr (!F8) return k[t][s];
    else return widen<T>(k[t][s / 2][s % 2 * 2], k[t][s / 2][s % 2 * 2 + 1]);
  }

  __device__ __forceinline__ void load_values(const CacheArgs& c, int32_t id, uint32_t first, uint32_t head, uint32_t m) {
    const uint32_t token = first - block_of(c, first) * c.tokens;
    const uint8_t* p = c.v + static_cast<uint64_t>(static_cast<uint32_t>(id)) * c.block_bytes + head * c.v_head + token * c.v_token;
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      uint32_t d = VX ? n * 16 + m : n / 8 * 16 * CE + m * CE;
      d = d < c.dim ? d : 0;
      const uint8_t* q = VX ? p + d * c.v_chunk : p + (n % 8) * c.v_token + d * (F8 ? 1 : 2);
      if constexpr (VW == 4) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(q);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[n][i] = x[i];
      } else if constexpr (VW == 2) {
        const u32x2 x = *reinterpret_cast<const u32x2*>(q);
        v[n][0] = x[0];
        v[n][1] = x[1];
      } else {
        v[n][0] = *reinterpret_cast<const uint32_t*>(q);
      }
    }
  }
  // Operand c of V^T: row m of instruction c, of the lane's 8 keys.
  template <class T>
  __device__ __forceinline__ u32x4 value(int c) const {
    if constexpr (VX) {
      if constexpr (F8) return widen<T>(v[c][0], v[c][1]);
      else return u32x4{v[c][0], v[c][1], v[c][2], v[c][3]};
    } else {
      const int n = c / CE * 8, e = c % CE;
      const uint32_t sel = e % 2 ? 0x07060302u : 0x05040100u;  // value e of keys 2 i and 2 i + 1 side by side
      u32x4 r;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (F8)
          r[i] = __builtin_amdgcn_perm(Type<T>::from_f8(v[n + 2 * i + 1][e / 4], e % 4 / 2),
                                       Type<T>::from_f8(v[n + 2 * i][e / 4], e % 4 / 2), sel);
        else
          r[i] = __builtin_amdgcn_perm(v[n + 2 * i + 1][e / 2], v[n + 2 * i][e / 2], sel);
      }
      return r;
    }
  }
};

template <class T, bool F8, int DP, bool VX, int R>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void attention_stream_kernel(AttnArgs a) {
  typedef Stream<F8, DP, VX> S;
  typedef ValueType<T, F8> TV;
  const uint32_t wave = threadIdx.x / kOpsWave, lane = threadIdx.x % kOpsWave, g = lane / 16, m = lane % 16;
  // Workgroups go to the 8 XCDs in turn: heads and sequences first, so that each XCD has early and late splits alike
  // (late ones exist of long sequences only; with splits first, counts of 4 and 8 left XCDs idle: 147 us instead of 128
  // for 32 sequences of 1k to 8k, 4 rows, x-packed bf16, and 86 instead of 74 in 8 bits).
  const uint32_t pairs = a.c.heads * a.s.num_seqs, pair = blockIdx.x % pairs, split = blockIdx.x / pairs;
  const uint32_t head = pair % a.c.heads, seq = pair / a.c.heads;
  const SeqSpan sp = span_of(a.s, seq);
  const uint32_t rows = sp.count * a.group;
  if (!rows) return;
  const uint32_t begin = split * a.split_len;
  if (begin >= sp.total && split) return;  // the first split also writes the rows that have no entries
  // Without a tree no row of the workgroup sees entries past its last token's.
  const uint32_t last_token = (R * 16 < rows ? R * 16 - 1 : rows - 1) / a.group;
  uint32_t end = begin + a.split_len < sp.total ? begin + a.split_len : sp.total;
  if (!a.tree && end > sp.before + last_token + 1) end = sp.before + last_token + 1;
  const int32_t* table = a.s.table + static_cast<uint64_t>(seq) * a.s.table_stride;

  u32x4 q[R][S::KS];
  uint32_t token[R];
  bool live[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const uint32_t row = r * 16 + m;
    live[r] = row < rows;
    token[r] = live[r] ? row / a.group : 0;
    load_q<F8, S::KS>(a, head * a.group + (live[r] ? row % a.group : 0), sp.first + token[r], live[r], g, q[r]);
  }
  const float to_log2 = a.scale * kLog2e * (a.k_scale ? a.k_scale[head] : 1.0f);

  f32x4 o[R][S::NC];
  float top[R], sum[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    top[r] = kLowest;
    sum[r] = 0;
#pragma unroll
    for (int c = 0; c < S::NC; ++c) o[r][c] = f32x4{0, 0, 0, 0};
  }

  // Keys of the first half: 8 (m / 4) + m % 4; a block's id of the lane's keys and of its values' keys,
  // 0 where there is none (then the tile is masked). Past the end: the last entry's.
  const uint32_t step = 4 * kTile;
  uint32_t base = begin + wave * kTile;
  // All 8 keys of a group at once: the group's first key decides, and past the end it is the last key's group.
  const auto clamp = [&](uint32_t first) { return first < end ? first : (end - 1) & ~7u; };
  const auto id_of = [&](uint32_t first) { return table[block_of(a.c, clamp(first))]; };
  const auto there = [&](int32_t id) { return static_cast<uint32_t>(id) < a.c.num_blocks; };
  S s;
  int32_t kid = 0, vid = 0;  // of this tile (values) and the next (keys)
  if (base < end) {
    kid = id_of(base + (m / 4) * 8);
    vid = id_of(base + g * 8);
    s.load_keys(a.c, there(kid) ? kid : 0, clamp(base + (m / 4) * 8) + m % 4, head, g);
  }
  int32_t next_kid = base + step < end ? id_of(base + step + (m / 4) * 8) : 0;
  float* logits[R];
#pragma unroll
  for (int r = 0; r < R; ++r)
    logits[r] = a.logits && live[r] ? a.logits + ((static_cast<uint64_t>(seq) * a.c.heads + head) * a.logit_rows + r * 16 + m) * a.logit_stride + g * 8
                                    : nullptr;
  const auto tile = [&](auto masked, bool have) {
    constexpr bool kMasked = decltype(masked)::value;
    s.load_values(a.c, have ? vid : 0, clamp(base + g * 8), head, m);
    s.clear_keys(a.c, g);
    f32x4 x[R][2];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int t = 0; t < 2; ++t) x[r][t] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < S::KS; ++i)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const u32x4 k = s.template key<T>(t, i);
#pragma unroll
        for (int r = 0; r < R; ++r) x[r][t] = Type<T>::mfma(k, q[r][i], x[r][t]);
      }
    if (base + step < end) {
      s.load_keys(a.c, there(next_kid) ? next_kid : 0, clamp(base + step + (m / 4) * 8) + m % 4, head, g);
      vid = id_of(base + step + g * 8);
      if (base + 2 * step < end) next_kid = id_of(base + 2 * step + (m / 4) * 8);
    }
    uint32_t okay = 0xff, seen[R];
    if constexpr (kMasked) {
      const uint32_t first = base + g * 8;
      okay = !have || first >= end ? 0 : end - first >= 8 ? 0xffu : (1u << (end - first)) - 1;
    }
    u32x4 p[R == 1 ? 2 : 1][R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = x[r][j / 4][j % 4] * to_log2;
      if constexpr (kMasked) {
        seen[r] = okay & keys_seen(a, sp, token[r], base + g * 8);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = seen[r] >> j & 1 ? y[j] : -INFINITY;
      }
      if (logits[r]) {  // kept for the entries' weights
        *reinterpret_cast<f32x4*>(logits[r] + base) = f32x4{y[0], y[1], y[2], y[3]};
        *reinterpret_cast<f32x4*>(logits[r] + base + 4) = f32x4{y[4], y[5], y[6], y[7]};
      }
      float mx = top[r];
#pragma unroll
      for (int j = 0; j < 8; ++j) mx = fmaxf(mx, y[j]);
      mx = max_of_row(mx);
      const float fade = __builtin_amdgcn_exp2f(top[r] - mx), from = mx - Type<TV>::kLift;
      top[r] = mx;
      float add = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        y[j] = __builtin_amdgcn_exp2f(y[j] - from);
        add += y[j];
      }
      sum[r] = sum[r] * fade + add;  // this lane's keys; its 4 lanes are joined at the end
      operand_of<TV>(y, p, r);
#pragma unroll
      for (int c = 0; c < S::NC; ++c) o[r][c] *= fade;
    }
    const auto op = [&](int c) { return s.template value<TV>(c); };
    if constexpr (kMasked)
      add_values_masked<TV>(op, p, seen, okay, g, m, o);
    else
      add_values<TV>(op, p, o);
    base += step;
  };
  // Tiles that every row sees whole; from the first other one on (drafted tokens, the end, or a block that is not
  // there), masked ones.
  uint32_t whole = a.tree ? sp.before : sp.before + 1;
  if (whole > end) whole = end;
  bool have = there(vid);
  while (base + kTile <= whole && __all(have)) {
    tile(std::false_type(), true);
    have = there(vid);
  }
  while (base < end) {
    tile(std::true_type(), have);
    have = there(vid);
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    sum[r] += across(sum[r], 16);
    sum[r] += across(sum[r], 32);
    top[r] -= Type<TV>::kLift;  // what the sums are taken from
  }

  // Waves 2, 3 to 0, 1, then 1 to 0. A value's lane and register are the same in every wave.
  constexpr int NO = R * S::NC * 4;
  __shared__ float part[2][NO + 2 * R][kOpsWave];
#pragma unroll
  for (uint32_t half = 2; half >= 1; half /= 2) {
    if (wave >= half && wave < 2 * half) {
      float(*to)[kOpsWave] = part[wave - half];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        to[NO + 2 * r][lane] = top[r];
        to[NO + 2 * r + 1][lane] = sum[r];
#pragma unroll
        for (int c = 0; c < S::NC; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) to[(r * S::NC + c) * 4 + i][lane] = o[r][c][i];
      }
    }
    __syncthreads();
    if (wave < half) {
      const float(*from)[kOpsWave] = part[wave];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float t = from[NO + 2 * r][lane], u = from[NO + 2 * r + 1][lane];
        const float mx = fmaxf(top[r], t);
        const float f = __builtin_amdgcn_exp2f(top[r] - mx), h = __builtin_amdgcn_exp2f(t - mx);
        top[r] = mx;
        sum[r] = sum[r] * f + u * h;
#pragma unroll
        for (int c = 0; c < S::NC; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[r][c][i] = o[r][c][i] * f + from[(r * S::NC + c) * 4 + i][lane] * h;
      }
    }
    __syncthreads();
  }
  if (wave) return;
  const float v_scale = a.v_scale ? a.v_scale[head] : 1.0f;
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (live[r])
      store_row<T, DP, S::NC, VX>(a, sp.first + token[r], head * a.group + (r * 16 + m) % a.group, split, g, top[r], sum[r], v_scale, o[r]);
}

// ---------------------------------------------------------------- many rows
// A workgroup has 64 RW rows of one sequence and KV head and one split of its entries; each
// of its 4 waves has RW tiles of 16 rows and goes through all tiles of KT entries, which
// the workgroup brings to LDS, two buffers in turn, one barrier a tile.
//
// 16-bit caches go from memory to LDS without registers (a lane's 16 bytes land at 16 times
// its index, so the order within the tile is made by which chunk a lane asks for); 8-bit ones
// pass through registers, where they are widened once for all waves. Rows of an entry lie
// DP values apart with their 16-byte chunks exchanged by the entry's number in the tile (bits
// 0, 1, 3, 4: what tells the 16 lanes of a read apart), so that neither the 16-byte reads of K
// nor the transposing 8-byte reads of V (ds_read_b64_tr_b16: of 4 entries' 16 values each lane of
// 16 gets one value of the 4) meet in a bank. x-packed values are V^T already.
//
// What probabilities are taken from follows the row's maximum only where one would pass
// 2^kRowsRoom (2^8 in bf16): the factor is 1 otherwise and nothing is scaled.
//
// 2048 tokens of 32 heads behind 6144 entries (8 KV heads, 128 values, bf16, head-major): 284 us, 0.85
// PFLOP/s, where a plain matrix product of the library reaches 1.37 (8192^3, both over hundreds of
// passes; over 40 after a rest of the GPU, 331 us, 0.73 PFLOP/s, and 1.29). Without the fetches a tile
// takes 12 % less, without the exponentials the same, without the reads of V 10 %: no one of
// them bounds it, the chain through a tile of few waves does. 4 trees of 13 to 24 tokens over 3k to 15k 8-bit
// x-packed entries: 56 us; splits are cut for the longest, so that 248 of 480 workgroups have entries, up to 1024 each,
// and pass a widened tile every 1.7 us. 4 rows over 32 sequences of 1k to 8k, bf16, head-major: 114 us, 5.4 TB/s.
template <bool F8, int DP, bool VX>
struct Tiles {
  static constexpr int KT = DP == 256 || (F8 && DP == 128) ? 32 : 64;  // entries of a tile
  static constexpr int AHEAD = F8 ? 4 : 1;        // tiles on their way while one is worked on
  static constexpr int SUB = KT / 32;
  static constexpr int KS = DP / 32;
  static constexpr int NC = DP / 16;
  static constexpr int C = DP / 8;                // 16-byte chunks of an entry
  static constexpr int VC = KT / 8;               // x-packed: 16-byte chunks of a value
  static constexpr uint32_t kBytes = KT * DP * 2; // of K or V of a tile
  static constexpr int N = KT * C / 256;          // chunks of a thread (16-bit)
  static constexpr int NL = F8 ? N / 2 : N;        // 16-byte loads of a thread

  static __device__ __forceinline__ uint32_t swizzle(uint32_t entry) {
    const uint32_t f = (entry & 3) | (entry >> 3 & 3) << 2;
    return C == 8 ? f >> 1 : f;
  }
  static __device__ __forceinline__ uint32_t at(uint32_t entry, uint32_t chunk) {
    return (entry * C + (chunk ^ swizzle(entry))) * 16;
  }
  static __device__ __forceinline__ uint32_t at_x(uint32_t d, uint32_t chunk) {  // V^T: chunk of 8 entries of value d
    return (d * VC + (chunk ^ (VC == 8 ? d >> 1 & 7 : d >> 2 & 3))) * 16;
  }
};

typedef __attribute__((address_space(3))) uint8_t lds_u8;
constexpr int kMfma = 0x008, kDsRead = 0x100;  // groups of instructions for the scheduler
typedef __attribute__((address_space(1))) const uint8_t global_u8;

__device__ __forceinline__ u32x2 read_turned(const uint8_t* p) {  // 16 lanes: 4 rows of 16 values, a column to each
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p)));
}

template <class T, bool F8, int DP, bool VX, int RW>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void attention_rows_kernel(AttnArgs a, uint32_t row_groups, uint32_t cells) {
  typedef Tiles<F8, DP, VX> S;
  typedef ValueType<T, F8> TV;
  // Two buffers, each of its own so that the compiler can tell reads of one from loads on their way to the other and
  // does not wait for those: code that knows its buffer takes it as a constant B.
  __shared__ __attribute__((aligned(1024))) uint8_t k0[S::kBytes], v0[S::kBytes], k1[S::kBytes], v1[S::kBytes];
  const auto k_of = [&](auto b) -> uint8_t* {
    if constexpr (std::is_same<decltype(b), int>::value) return b ? k1 : k0;
    else if constexpr (decltype(b)::value) return k1;
    else return k0;
  };
  const auto v_of = [&](auto b) -> uint8_t* {
    if constexpr (std::is_same<decltype(b), int>::value) return b ? v1 : v0;
    else if constexpr (decltype(b)::value) return v1;
    else return v0;
  };
  const auto other = [](auto b) {
    if constexpr (std::is_same<decltype(b), int>::value) return b ^ 1;
    else return std::bool_constant<!decltype(b)::value>();
  };
  constexpr uint32_t kRing = F8 ? 8 : 4;  // more than the tiles between a publication and the last use of it
  __shared__ uint64_t rows_at[kRing][S::KT], groups_at[kRing][VX ? S::VC : 1];  // of the last tiles, addresses of their entries, 0 where there is none
  __shared__ uint32_t absent[8];  // number of the last tile of every eight that had entries without a block
  // 8 bits: tiles as they come, 4 in turn; a thread's 16 bytes of K at 16 i of its chunk i, then those of V.
  constexpr uint32_t kRaw = F8 ? S::NL * 2 * 4096 : 16;
  __shared__ __attribute__((aligned(1024))) uint8_t raw[F8 ? 4 : 1][kRaw];
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kOpsWave), lane = threadIdx.x % kOpsWave, g = lane / 16, m = lane % 16;
  // Workgroups go to the 8 XCDs in turn. Row groups with the same keys follow each other on one XCD, so that they
  // share its L2; what they belong to (heads and sequences first, then splits) goes round the XCDs.
  const uint32_t slot = blockIdx.x / 8, cell = slot / row_groups * 8 + blockIdx.x % 8;
  if (cell >= cells) return;
  const uint32_t group = row_groups - 1 - slot % row_groups;  // the last rows first: without a tree they see most
  const uint32_t pairs = a.c.heads * a.s.num_seqs, split = cell / pairs, u = cell % pairs;
  const uint32_t head = u % a.c.heads, seq = u / a.c.heads;
  const SeqSpan sp = span_of(a.s, seq);
  const uint32_t rows = sp.count * a.group;
  const uint32_t row0 = group * 64 * RW;
  if (row0 >= rows) return;
  const uint32_t begin = split * a.split_len;
  if (begin >= sp.total && split) return;
  const auto last_token = [&](uint32_t first, uint32_t n) { return (first + n < rows ? first + n - 1 : rows - 1) / a.group; };
  uint32_t end = begin + a.split_len < sp.total ? begin + a.split_len : sp.total;
  if (!a.tree && end > sp.before + last_token(row0, 64 * RW) + 1) end = sp.before + last_token(row0, 64 * RW) + 1;
  const int32_t* table = a.s.table + static_cast<uint64_t>(seq) * a.s.table_stride;

  float to_log2 = a.scale * kLog2e * (a.k_scale ? a.k_scale[head] : 1.0f);
  // A negative factor goes into Q, so that the largest product is the largest logit; 0 becomes a number that keeps -infinity.
  const uint32_t flip = to_log2 < 0 ? 0x80008000u : 0u;
  to_log2 = fabsf(to_log2);
  if (to_log2 < 1e-30f) to_log2 = 1e-30f;  // not a maximum, which would drop NaN
  u32x4 q[RW][S::KS];
  uint32_t token[RW];
  bool live[RW];
  const uint32_t my_row0 = row0 + wave * RW * 16;
#pragma unroll
  for (int r = 0; r < RW; ++r) {
    const uint32_t row = my_row0 + r * 16 + m;
    live[r] = row < rows;
    token[r] = live[r] ? row / a.group : 0;
    load_q<false, S::KS>(a, head * a.group + (live[r] ? row % a.group : 0), sp.first + token[r], live[r], g, q[r]);
#pragma unroll
    for (int i = 0; i < S::KS; ++i) q[r][i] ^= flip;
  }
  // Entries that this wave's rows may see.
  const bool work = my_row0 < rows;
  const uint32_t my_end = !work ? 0 : a.tree ? end : sp.before + last_token(my_row0, RW * 16) + 1;

  f32x4 o[RW][S::NC];
  float top[RW], sum[RW];
#pragma unroll
  for (int r = 0; r < RW; ++r) {
    top[r] = kLowest;
    sum[r] = 0;
#pragma unroll
    for (int c = 0; c < S::NC; ++c) o[r][c] = f32x4{0, 0, 0, 0};
  }

  // Chunks past head_dim that no tile brings count as 0: K's in the products, and V's would be looked through for
  // infinities, as whatever the last kernel left there (8-bit and x-packed tiles bring zeros themselves).
  if (a.c.dim < DP)
    for (uint32_t i = threadIdx.x; i < S::kBytes / 16; i += 256) {
      reinterpret_cast<u32x4*>(k0)[i] = u32x4{0, 0, 0, 0};
      reinterpret_cast<u32x4*>(k1)[i] = u32x4{0, 0, 0, 0};
      if constexpr (!F8 && !VX) {
        reinterpret_cast<u32x4*>(v0)[i] = u32x4{0, 0, 0, 0};
        reinterpret_cast<u32x4*>(v1)[i] = u32x4{0, 0, 0, 0};
      }
    }
  if (threadIdx.x < 8) absent[threadIdx.x] = 0;
  __syncthreads();

  // Where a tile's entries (and, x-packed, the 8 or 16 entries of a chunk of values) lie, found once for all threads that
  // bring parts of them: a thread an entry, its address a tile before it is used, its block a tile before that.
  constexpr uint32_t kPer = F8 ? 16 : 8, kGroups = VX ? S::KT / kPer : 0;
  const bool finds = threadIdx.x < S::KT, finds_x = VX && threadIdx.x >= S::KT && threadIdx.x < S::KT + kGroups;
  const uint32_t found = finds ? threadIdx.x : (threadIdx.x - S::KT) * kPer;  // the entry of the tile
  int32_t id = 0;
  const auto look_up = [&](uint32_t base) {
    const uint32_t e = base + found;
    if (finds || finds_x) id = table[block_of(a.c, e < end ? e : end - 1)];
  };
  const auto publish = [&](uint32_t base, uint32_t n) {
    if (!finds && !finds_x) return;
    const uint32_t e = base + found;
    const bool has = static_cast<uint32_t>(id) < a.c.num_blocks;
    uint64_t p = 0;
    if (e < end && has) {
      const uint32_t t = e - block_of(a.c, e) * a.c.tokens;
      p = static_cast<uint64_t>(static_cast<uint32_t>(id)) * a.c.block_bytes;
      if (finds)
        p += reinterpret_cast<uint64_t>(a.c.k) + head * a.c.k_head + static_cast<uint64_t>(t) * a.c.k_token;
      else
        p += reinterpret_cast<uint64_t>(a.c.v) + head * a.c.v_head + static_cast<uint64_t>(t) * a.c.v_token;
    }
    if (finds) {
      rows_at[n % kRing][threadIdx.x] = p;
      if (e < end && !has) absent[n % 8] = n;
    } else {
      groups_at[n % kRing][threadIdx.x - S::KT] = p;
    }
  };

  // This thread's part of a tile: chunk i of K (and V) is slot 256 i + thread; 16 bits: of the tile in LDS, 8 bits: of the
  // tile in memory.
  constexpr uint32_t kRowChunks = F8 ? S::C / 2 : S::C, kXChunks = F8 ? S::VC / 2 : S::VC;
  const auto k_entry = [&](int i) { return (i * 256 + threadIdx.x) / kRowChunks; };
  const auto k_chunk = [&](int i) { return F8 ? threadIdx.x % kRowChunks : (threadIdx.x % kRowChunks) ^ S::swizzle(k_entry(i)); };
  const auto x_value = [&](int i) { return (i * 256 + threadIdx.x) / kXChunks; };
  const auto x_chunk = [&](int i) -> uint32_t {
    const uint32_t d = x_value(i), c = threadIdx.x % kXChunks;
    return F8 ? c : c ^ (S::VC == 8 ? d >> 1 & 7 : d >> 2 & 3);
  };
  const uint64_t v_from_k = a.c.v - a.c.k;
  uint32_t in_full = 0;  // 8 bits: how many tiles in a row this wave asked for every chunk of
  // Start bringing tile n, at `base`, to buffer b (8 bits: to its turn of `raw`).
  const auto fetch = [&](uint32_t base, uint32_t n, auto b) {
    uint8_t* const kl = k_of(b);
    uint8_t* const vl = v_of(b);
    uint8_t* const rl = raw[F8 ? n % 4 : 0];
    bool full = true;
    const bool tail = base + S::KT > end;
    if constexpr (!F8 && !VX) {
      // All of the tile there and no padding, as almost always: nothing but the loads.
      uint64_t at[S::NL];
      bool all = a.c.dim == DP;
#pragma unroll
      for (int i = 0; i < S::NL; ++i) {
        at[i] = rows_at[n % kRing][k_entry(i)];
        all = all && at[i];
      }
      if (__all(all)) {
#pragma unroll
        for (int i = 0; i < S::NL; ++i) {
          const uint8_t* kp = reinterpret_cast<const uint8_t*>(at[i]) + k_chunk(i) * 16;  // rows: chunks follow each other
          __builtin_amdgcn_global_load_lds((global_u8*)kp, (lds_u8*)(kl + (i * 256 + wave * 64) * 16), 16, 0, 0);
          __builtin_amdgcn_global_load_lds((global_u8*)(kp + v_from_k), (lds_u8*)(vl + (i * 256 + wave * 64) * 16), 16, 0, 0);
        }
        return;
      }
    }
#pragma unroll
    for (int i = 0; i < S::NL; ++i) {
      const uint32_t chunk = k_chunk(i);
      const uint64_t at = rows_at[n % kRing][k_entry(i)];
      const uint8_t* kp = reinterpret_cast<const uint8_t*>(at) + chunk * a.c.k_chunk;
      const uint8_t* vp = reinterpret_cast<const uint8_t*>(at) + v_from_k + chunk * 16;  // not x-packed: as far from V's start
      const bool live = chunk * (F8 ? 16 : 8) < a.c.dim;
      if constexpr (F8) {
        const uint32_t slot = i * 256 + threadIdx.x, to = (i * 256 + wave * 64) * 16;
        const bool in = at && live;
        full = full && in;
        if (in) {
          __builtin_amdgcn_global_load_lds((global_u8*)kp, (lds_u8*)(rl + to), 16, 0, 0);
          if constexpr (!VX) __builtin_amdgcn_global_load_lds((global_u8*)vp, (lds_u8*)(rl + S::NL * 4096 + to), 16, 0, 0);
        } else {
          *reinterpret_cast<u32x4*>(rl + slot * 16) = u32x4{0, 0, 0, 0};
          if constexpr (!VX) *reinterpret_cast<u32x4*>(rl + S::NL * 4096 + slot * 16) = u32x4{0, 0, 0, 0};
        }
      } else if (live) {
        if (at) {
          __builtin_amdgcn_global_load_lds((global_u8*)kp, (lds_u8*)(kl + (i * 256 + wave * 64) * 16), 16, 0, 0);
          if constexpr (!VX)
            __builtin_amdgcn_global_load_lds((global_u8*)vp, (lds_u8*)(vl + (i * 256 + wave * 64) * 16), 16, 0, 0);
        } else {
          const uint32_t slot = i * 256 + threadIdx.x;
          *reinterpret_cast<u32x4*>(kl + slot * 16) = u32x4{0, 0, 0, 0};
          if constexpr (!VX) *reinterpret_cast<u32x4*>(vl + slot * 16) = u32x4{0, 0, 0, 0};
        }
      }
      if constexpr (VX) {
        const uint32_t d = x_value(i), c = x_chunk(i);
        const uint64_t from = groups_at[n % kRing][c];
        const uint8_t* xp = reinterpret_cast<const uint8_t*>(from) + d * a.c.v_chunk;
        const bool in = from && d < a.c.dim;
        const uint32_t e = base + c * kPer, left = !tail ? kPer : e < end ? end - e : 0;  // of the chunk's entries, those before the end
        if constexpr (F8) {
          const uint32_t slot = i * 256 + threadIdx.x;
          full = full && in && left >= kPer;
          if (in && left >= kPer) {
            __builtin_amdgcn_global_load_lds((global_u8*)xp, (lds_u8*)(rl + S::NL * 4096 + (i * 256 + wave * 64) * 16), 16, 0, 0);
          } else {
            u32x4 w = in ? *reinterpret_cast<const u32x4*>(xp) : u32x4{0, 0, 0, 0};
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) w[j] &= left >= 4 * j + 4 ? ~0u : left <= 4 * j ? 0u : (1u << (left - 4 * j) * 8) - 1;
            *reinterpret_cast<u32x4*>(rl + S::NL * 4096 + slot * 16) = w;
          }
        } else if (in && left >= kPer) {
          __builtin_amdgcn_global_load_lds((global_u8*)xp, (lds_u8*)(vl + (i * 256 + wave * 64) * 16), 16, 0, 0);
        } else {
          const u32x4 w = in ? *reinterpret_cast<const u32x4*>(xp) : u32x4{0, 0, 0, 0};
          *reinterpret_cast<u32x4*>(vl + (i * 256 + threadIdx.x) * 16) = only_keys(w, (1u << left) - 1);
        }
      }
    }
    if constexpr (F8) in_full = __all(full) ? in_full + 1 : 0;
  };
  // 8 bits: widen tile n from its turn of `raw` into buffer b, for all waves once. A thread widens what it asked for, so it
  // waits for its own loads alone, and not for those of the `later` tiles asked for since where their number is sure.
  // (The reads are written out, with their wait: the compiler would wait for all loads that are on their way to `raw`.)
  const auto widen_to = [&](auto b, uint32_t n, bool later) {
    if constexpr (F8) {
      uint8_t* const kl = k_of(b);
      uint8_t* const vl = v_of(b);
      if (later && in_full >= S::AHEAD - 1)
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S::AHEAD - 1) * 2 * S::NL) : "memory");
      else
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      const uint32_t at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_u8*)raw[n % 4])) + threadIdx.x * 16;
#pragma unroll
      for (int i = 0; i < S::NL; ++i) {
        const uint32_t e = k_entry(i), chunk = k_chunk(i) * 2;
        u32x4 x, y;
        asm volatile("s_waitcnt lgkmcnt(0)\n\tds_read_b128 %0, %2\n\tds_read_b128 %1, %3\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(x), "=&v"(y)
                     : "v"(at + i * 4096), "v"(at + (S::NL + i) * 4096)
                     : "memory");
        *reinterpret_cast<u32x4*>(kl + S::at(e, chunk)) = widen<T>(x[0], x[1]);
        *reinterpret_cast<u32x4*>(kl + S::at(e, chunk + 1)) = widen<T>(x[2], x[3]);
        if constexpr (VX) {
          const uint32_t d = x_value(i), c = x_chunk(i) * 2;
          *reinterpret_cast<u32x4*>(vl + S::at_x(d, c)) = widen<TV>(y[0], y[1]);
          *reinterpret_cast<u32x4*>(vl + S::at_x(d, c + 1)) = widen<TV>(y[2], y[3]);
        } else {
          *reinterpret_cast<u32x4*>(vl + S::at(e, chunk)) = widen<TV>(y[0], y[1]);
          *reinterpret_cast<u32x4*>(vl + S::at(e, chunk + 1)) = widen<TV>(y[2], y[3]);
        }
      }
    }
  };

  // Where this lane reads: instruction s of K is at k_at ^ 64 s, halves 4 entries apart; of V
  // instruction c at v_at ^ 32 c (16 values are 2 chunks), halves 4 entries apart too.
  const uint32_t k_at = S::at((m / 4) * 8 + m % 4, g);
  const uint32_t v_at = VX ? 0 : S::at(g * 8 + m / 4, m >> 1 & 1) + (m & 1) * 8;

  constexpr uint32_t kAhead = S::AHEAD, KT = S::KT;
  uint32_t number = 1;
  if (begin < end) {
#pragma unroll
    for (uint32_t i = 0; i <= kAhead; ++i) {
      look_up(begin + i * KT);
      publish(begin + i * KT, number + i);
    }
    look_up(begin + (kAhead + 1) * KT);
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < (F8 ? kAhead : 1); ++i)
      if (begin + i * KT < end) fetch(begin + i * KT, number + i, std::false_type());
    widen_to(std::false_type(), number, false);
  }
  uint32_t base = begin;
  const auto arrive = [&](auto b) {  // the tile at `base` is in buffer b, and the next ones are on their way
    if constexpr (!F8) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this thread's part of the tile is in LDS
    __syncthreads();                                                     // and everyone's, and the other buffer is no longer read
    if (base + kAhead * KT < end) {
      // In this order, so that the block looked up last time is not waited for behind the tile's own loads.
      publish(base + (kAhead + 1) * KT, number + kAhead + 1);
      look_up(base + (kAhead + 2) * KT);
      fetch(base + kAhead * KT, number + kAhead, other(b));
    }
  };
  const auto leave = [&](auto b) {
    if (base + KT < end) widen_to(other(b), number + 1, base + kAhead * KT < end);
    base += KT;
    ++number;
  };
  const auto tile = [&](auto masked, auto b) {
    constexpr bool kMasked = decltype(masked)::value;
    const uint8_t* const kl = k_of(b);
    const uint8_t* const vl = v_of(b);
    f32x4 x[RW][S::SUB][2];
#pragma unroll
    for (int r = 0; r < RW; ++r)
#pragma unroll
      for (int j = 0; j < S::SUB; ++j)
#pragma unroll
        for (int t = 0; t < 2; ++t) x[r][j][t] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < S::KS; ++i)
#pragma unroll
      for (int j = 0; j < S::SUB; ++j)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const u32x4 k = *reinterpret_cast<const u32x4*>(kl + (k_at ^ (i * 64)) + (j * 32 + t * 4) * S::C * 16);
#pragma unroll
          for (int r = 0; r < RW; ++r) x[r][j][t] = Type<T>::mfma(k, q[r][i], x[r][j][t]);
        }
    if constexpr (!kMasked) {
      constexpr int kReads = S::KS * S::SUB * 2;
      __builtin_amdgcn_sched_group_barrier(kDsRead, kReads / 2, 0);
#pragma unroll
      for (int i = 0; i < kReads / 2; ++i) {
        __builtin_amdgcn_sched_group_barrier(kMfma, RW, 0);
        __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(kMfma, RW * kReads / 2, 0);
    }
    uint32_t seen[S::SUB][RW];
    if constexpr (kMasked) {
#pragma unroll
      for (int j = 0; j < S::SUB; ++j) {
        const uint32_t okay = keys_there(a.c, table, base + j * 32 + g * 8, end);
#pragma unroll
        for (int r = 0; r < RW; ++r) {
          seen[j][r] = okay & keys_seen(a, sp, token[r], base + j * 32 + g * 8);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[r][j][i / 4][i % 4] = seen[j][r] >> i & 1 ? x[r][j][i / 4][i % 4] : -INFINITY;
        }
      }
    }
    float mx[RW];
    bool rise = false;
#pragma unroll
    for (int r = 0; r < RW; ++r) {
      float y = x[r][0][0][0];
#pragma unroll
      for (int j = 0; j < S::SUB; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) y = fmaxf(y, x[r][j][i / 4][i % 4]);
      mx[r] = max_of_row(y) * to_log2;
      rise |= mx[r] > top[r] + Type<TV>::kRowsRoom;
    }
    if (__any(rise)) {
#pragma unroll
      for (int r = 0; r < RW; ++r) {
        const float y = fmaxf(top[r], mx[r] - Type<TV>::kRowsLift);
        const float fade = __builtin_amdgcn_exp2f(top[r] - y);
        top[r] = y;
        sum[r] *= fade;
#pragma unroll
        for (int c = 0; c < S::NC; ++c) o[r][c] *= fade;
      }
    }
#pragma unroll
    for (int j = 0; j < S::SUB; ++j) {
      u32x4 p[RW == 1 ? 2 : 1][RW];
#pragma unroll
      for (int r = 0; r < RW; ++r) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          y[i] = __builtin_amdgcn_exp2f(fmaf(x[r][j][i / 4][i % 4], to_log2, -top[r]));
          sum[r] += y[i];
        }
        operand_of<TV>(y, p, r);
      }
      const auto op = [&](int c) {
        if constexpr (VX) {
          return *reinterpret_cast<const u32x4*>(vl + S::at_x(c * 16 + m, j * 4 + g));
        } else {
          const uint8_t* at = vl + (v_at ^ (c * 32)) + j * 32 * S::C * 16;
          const u32x2 lo = read_turned(at), hi = read_turned(at + 4 * S::C * 16);
          return u32x4{lo[0], lo[1], hi[0], hi[1]};
        }
      };
      if constexpr (kMasked)
        add_values_masked<TV>(op, p, seen[j], 0xff, g, m, o);  // entries that are not there are 0 in LDS
      else
        add_values<TV>(op, p, o);
    }
  };
  // Tiles that every row of the workgroup sees whole, the two buffers in turn; from the first other one on, masked ones.
  uint32_t whole = a.tree ? sp.before : sp.before + row0 / a.group + 1;
  if (whole > end) whole = end;
  bool arrived = false;
  const auto go = [&](auto b) {
    if (base + S::KT > whole) return false;
    arrive(b);
    arrived = absent[number % 8] == number;
    if (arrived) return false;
    if (work) tile(std::false_type(), b);
    leave(b);
    return true;
  };
  int b = 0;
  while (true) {
    b = 0;
    if (!go(std::false_type())) break;
    b = 1;
    if (!go(std::true_type())) break;
  }
  while (base < end) {
    if (!arrived) b ? arrive(std::true_type()) : arrive(std::false_type());
    arrived = false;
    if (base < my_end) tile(std::true_type(), b);
    b ? leave(std::true_type()) : leave(std::false_type());
    b ^= 1;
  }
  const float v_scale = a.v_scale ? a.v_scale[head] : 1.0f;
#pragma unroll
  for (int r = 0; r < RW; ++r) {
    sum[r] += across(sum[r], 16);
    sum[r] += across(sum[r], 32);
    if (live[r])
      store_row<T, DP, S::NC, 1>(a, sp.first + token[r], head * a.group + (my_row0 + r * 16 + m) % a.group, split, g, top[r], sum[r], v_scale, o[r]);
  }
}

// ---------------------------------------------------------------- joining the splits
// Splits that a sequence with `total` entries has.
__device__ __forceinline__ uint32_t splits_of(const AttnArgs& a, uint32_t total) {
  const uint32_t n = (total + a.split_len - 1) / a.split_len;
  return n ? n : 1;
}

// Maximum and sum of a row over its n splits, by a whole wave.
__device__ __forceinline__ void join_ml(const float* ml, uint32_t n, float* top, float* sum) {
  const uint32_t lane = threadIdx.x % kOpsWave;
  float t = kLowest, s = 0;
  for (uint32_t i = lane; i < n; i += kOpsWave) {
    const float y = fmaxf(t, ml[2 * i]);
    s = s * __builtin_amdgcn_exp2f(t - y) + ml[2 * i + 1] * __builtin_amdgcn_exp2f(ml[2 * i] - y);
    t = y;
  }
#pragma unroll
  for (int x = 1; x < kOpsWave; x *= 2) {
    const float u = across(t, x), v = across(s, x), y = fmaxf(t, u);
    s = s * __builtin_amdgcn_exp2f(t - y) + v * __builtin_amdgcn_exp2f(u - y);
    t = y;
  }
  *top = t;
  *sum = s;
}

// A row: out = sum 2^(m_i - M) o_i / sum 2^(m_i - M) l_i over its splits. A workgroup has one
// row; DP / 4 lanes read a split, and 1024 / DP splits are read at once. 6 us for 32 rows of 64
// splits and the weights of 64k entries: a launch and two dependent reads.
template <class T, int DP>
__device__ __forceinline__ void join_row(const AttnArgs& a, const SeqSpan& sp, uint32_t row, uint32_t head, f32x4* lds) {
  constexpr uint32_t L = DP / 4, W = 256 / L;
  const uint32_t token = sp.first + row / a.group, qh = head * a.group + row % a.group;
  const uint64_t unit = static_cast<uint64_t>(token) * a.q_heads + qh;
  const uint32_t n = splits_of(a, sp.total), l = threadIdx.x % L, w = threadIdx.x / L;
  const float* ml = a.part_ml + 2 * unit * a.splits;
  float top, sum;
  join_ml(ml, n, &top, &sum);
  if (threadIdx.x == 0) {
    const float l2 = sum == 0 ? -INFINITY : top + __builtin_amdgcn_logf(sum);
    if (a.lse) a.lse[unit] = l2 * kLn2;
    if (a.lse2) a.lse2[lse2_at(a, token, qh)] = l2;
  }
  const f32x4* part = reinterpret_cast<const f32x4*>(a.part + unit * a.splits * DP) + l;
  f32x4 o = {0, 0, 0, 0};
#pragma unroll 4
  for (uint32_t i = w; i < n; i += W) o += part[static_cast<uint64_t>(i) * L] * __builtin_amdgcn_exp2f(ml[2 * i] - top);
  lds[threadIdx.x] = o;
  __syncthreads();
  if (w) return;
  for (uint32_t i = 1; i < W; ++i) o += lds[i * L + l];
  const float by = sum == 0 ? 0.0f : 1.0f / sum;
  T* to = reinterpret_cast<T*>(a.out.data) + token * a.out.token + qh * a.out.head;
  if (l * 4 >= a.c.dim) return;
  const u32x2 y = {Type<T>::pack(o[0] * by, o[1] * by), Type<T>::pack(o[2] * by, o[3] * by)};
  if (a.wide_out) {
    *reinterpret_cast<u32x2*>(to + l * 4) = y;
  } else {
    uint16_t* h = reinterpret_cast<uint16_t*>(to + l * 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) h[j] = static_cast<uint16_t>(y[j / 2] >> (j % 2 * 16));
  }
}

constexpr uint32_t kWeigh = 1024;  // entries of a workgroup that adds up kept logits

// Rows of the call first (`joins` of them), then, where logits were kept or the call has no rows, the weights of the
// entries: scores_out = decay scores_in + sum over the rows of 2^(logit - lse).
template <class T, int DP>
__global__ __launch_bounds__(256) void attention_finish_kernel(AttnArgs a, uint32_t joins) {
  __shared__ f32x4 lds[256];
  const uint32_t head = blockIdx.y, seq = blockIdx.z;
  const SeqSpan sp = span_of(a.s, seq);
  const uint32_t rows = sp.count * a.group;
  if (blockIdx.x < joins) {
    if (blockIdx.x < rows) join_row<T, DP>(a, sp, blockIdx.x, head, lds);
    return;
  }
  const uint32_t first = (blockIdx.x - joins) * kWeigh;
  if (first >= sp.total) return;
  float* l2 = reinterpret_cast<float*>(lds);  // of the rows: at most 16
  const uint32_t n = rows ? splits_of(a, sp.total) : 0;
  for (uint32_t r = threadIdx.x / kOpsWave; r < rows; r += 4) {
    const uint64_t unit = static_cast<uint64_t>(sp.first + r / a.group) * a.q_heads + head * a.group + r % a.group;
    float top, sum;
    join_ml(a.part_ml + 2 * unit * a.splits, n, &top, &sum);
    if (threadIdx.x % kOpsWave == 0) l2[r] = sum == 0 ? INFINITY : top + __builtin_amdgcn_logf(sum);
  }
  __syncthreads();
  const uint32_t key = first + threadIdx.x * 4;
  if (key >= sp.total) return;
  const uint64_t pair = static_cast<uint64_t>(seq) * a.c.heads + head;
  const float* x = a.logits + pair * a.logit_rows * a.logit_stride + key;
  f32x4 w = {0, 0, 0, 0};
  for (uint32_t r = 0; r < rows; ++r) {
    const f32x4 y = *reinterpret_cast<const f32x4*>(x + static_cast<uint64_t>(r) * a.logit_stride);
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] += y[j] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(y[j] - l2[r]);  // 0 though l2 be NaN
  }
  const uint64_t at = pair * a.scores_stride + key;
#pragma unroll
  for (uint32_t j = 0; j < 4; ++j)
    if (key + j < sp.total) a.scores_out[at + j] = (a.scores_in && key + j < sp.before ? a.decay * a.scores_in[at + j] : 0.0f) + w[j];
}

// The queries kept for the weights where the output is written over them: 8 values a thread.
__global__ __launch_bounds__(256) void attention_keep_queries_kernel(AttnArgs a) {
  const uint32_t chunks = a.c.dim / 8;
  const uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x, row = i / chunks;
  if (row >= static_cast<uint64_t>(a.s.num_tokens) * a.q_heads) return;
  const uint64_t token = row / a.q_heads, head = row % a.q_heads, d = i % chunks * 8;
  const u32x4 w = load_row8(a.q.data + 2 * (token * a.q.token + head * a.q.head + d), a.wide_q);
  *reinterpret_cast<u32x4*>(a.score_q.data + 2 * (token * a.score_q.token + head * a.score_q.head + d)) = w;
}

// ---------------------------------------------------------------- weights of the entries, many rows
// With every row's sum known, Q K^T once more, this time rows down and keys across, so that a
// lane adds up its key's rows. Rows come to LDS with their lse. Each score has one writer and its
// sum one order.
//
// Up to some hundred rows a workgroup has up to kScored keys (score_len) and brings kRows rows at
// a time; its waves take the keys, 32 at a time, in turn, the next ones on their way: what bounds
// it is how many different keys are on their way at once. With more rows (STAY) a wave's 32 keys
// stay in its registers and the rows pass by in two buffers, the next ones on their way to
// registers: bound by the exponentials and LDS, about 300 us for 8192 rows and 8192 entries of
// 8 KV heads.
constexpr uint32_t kScored = 1024;

template <class T, bool F8, int DP, bool STAY>
__global__ __launch_bounds__(256) void attention_scores_kernel(AttnArgs a) {
  constexpr int KS = DP / 32, NK = F8 ? KS / 2 : KS, C = DP / 8, kRows = STAY || DP == 256 ? 64 : 128;
  constexpr int kChunks = kRows * C / 256;  // 16-byte chunks of the rows that a thread brings
  __shared__ __attribute__((aligned(16))) uint8_t ql[(STAY ? 2 : 1) * kRows * C * 16];
  __shared__ __attribute__((aligned(16))) float ll[(STAY ? 2 : 1) * kRows];
  __shared__ float sums[STAY ? 4 * kTile : kScored];
  const uint32_t wave = threadIdx.x / kOpsWave, lane = threadIdx.x % kOpsWave, g = lane / 16, m = lane % 16;
  const uint32_t head = blockIdx.y, seq = blockIdx.z;
  const SeqSpan sp = span_of(a.s, seq);
  const uint32_t begin = blockIdx.x * a.score_len;
  if (begin >= sp.total) return;
  const uint32_t end = begin + a.score_len < sp.total ? begin + a.score_len : sp.total;
  const int32_t* table = a.s.table + static_cast<uint64_t>(seq) * a.s.table_stride;
  const uint32_t rows = sp.count * a.group;
  const float to_log2 = a.scale * kLog2e * (a.k_scale ? a.k_scale[head] : 1.0f);
  // lse2 has a sequence's and KV head's rows side by side.
  const float* l2_at = a.lse2 + (static_cast<uint64_t>(head) * a.s.num_tokens + sp.first) * a.group;
  // 16 bytes of a row in LDS: chunks exchanged by the row's number, so that 16 rows' do not meet in a bank.
  const auto at = [&](uint32_t row, uint32_t chunk) {
    return (row * C + (chunk ^ (C == 8 ? row >> 1 & 7 : row & 15))) * 16;
  };
  const auto load = [&](uint32_t base, u32x4 (&k)[2][NK], uint32_t* there) {
    uint32_t have = 0;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      uint32_t in_block;
      const uint32_t key = base + t * 16 + m;
      const int32_t id = block_at(a.c, table, key < end ? key : end - 1, &in_block);
      have |= (key < end && id >= 0 ? 1u : 0u) << t;
      const uint8_t* p = a.c.k + static_cast<uint64_t>(id < 0 ? 0 : id) * a.c.block_bytes + head * a.c.k_head +
                         in_block * a.c.k_token;
#pragma unroll
      for (int s = 0; s < NK; ++s) {
        const uint32_t chunk = s * 4 + g;
        k[t][s] = *reinterpret_cast<const u32x4*>(p + (chunk * (F8 ? 16 : 8) < a.c.dim ? chunk * a.c.k_chunk : 0));
      }
    }
    *there = have;
  };
  const auto operands = [&](const u32x4 (&k)[2][NK], u32x4 (&kw)[2][KS]) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        const bool live = F8 ? ((i / 2) * 4 + g) * 16 < a.c.dim : (i * 4 + g) * 8 < a.c.dim;
        if constexpr (F8) kw[t][i] = widen<T>(k[t][i / 2][i % 2 * 2], k[t][i / 2][i % 2 * 2 + 1]);
        else kw[t][i] = k[t][i];
        if (a.c.dim < DP && !live) kw[t][i] = u32x4{0, 0, 0, 0};
      }
  };
  const auto row_chunk = [&](uint32_t row0, uint32_t i) {
    const uint32_t row = row0 + i / C, d = i % C * 8;
    u32x4 w = {0, 0, 0, 0};
    if (row < rows && d < a.c.dim)
      w = load_row8(a.score_q.data + 2 * ((sp.first + row / a.group) * a.score_q.token +
                                          (head * a.group + row % a.group) * a.score_q.head + d), a.wide_score_q);
    return w;
  };
  const auto row_lse = [&](uint32_t row) {
    const float l = row < rows ? l2_at[row] : INFINITY;
    return l == -INFINITY ? INFINITY : l;  // a row that sees nothing
  };
  // Adds to a lane's two keys' sums what `some` rows from row0 on, in LDS at q_at and l_at, give them. A loop of its own
  // for keys that every row sees, for drafted ones of a chain, seen from row `from` on, and for those of a tree.
  const auto weigh = [&](uint32_t base, const u32x4 (&kw)[2][KS], const uint8_t* q_at, const float* l_at, uint32_t row0,
                         uint32_t some, float (&sum)[2]) {
    const auto run = [&](auto mode) {
      constexpr int kMode = decltype(mode)::value;
      uint32_t from[2], draft[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint32_t key = base + t * 16 + m;
        draft[t] = key < sp.before ? 0 : key - sp.before;
        from[t] = draft[t] * a.group;
      }
      for (uint32_t r0 = 0; r0 < some; r0 += 16) {
        f32x4 x[2] = {f32x4{0, 0, 0, 0}, f32x4{0, 0, 0, 0}};
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          const u32x4 q = *reinterpret_cast<const u32x4*>(q_at + at(r0 + m, F8 ? i / 2 * 8 + g * 2 + i % 2 : i * 4 + g));
          x[0] = Type<T>::mfma(q, kw[0][i], x[0]);
          x[1] = Type<T>::mfma(q, kw[1][i], x[1]);
        }
        const f32x4 l2 = *reinterpret_cast<const f32x4*>(l_at + r0 + g * 4);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p = __builtin_amdgcn_exp2f(x[t][i] * to_log2 - l2[i]);
            const uint32_t row = row0 + r0 + g * 4 + i;
            bool see = l2[i] != INFINITY;  // NaN does: its entries' weights are no numbers
            if constexpr (kMode == 1) see = see && row >= from[t];
            if constexpr (kMode == 2)
              if (see && base + t * 16 + m >= sp.before) {
                const uint32_t d = draft[t];
                see = d / 64 < a.tree_words &&
                      (a.tree[static_cast<uint64_t>(sp.first + row / a.group) * a.tree_words + d / 64] >> (d % 64) & 1);
              }
            sum[t] += see ? p : 0.0f;
          }
      }
    };
    if (base + kTile <= sp.before)
      run(std::integral_constant<int, 0>());
    else if (!a.tree)
      run(std::integral_constant<int, 1>());
    else
      run(std::integral_constant<int, 2>());
  };
  // A key's rows are in the lanes 16 apart.
  const auto joined = [&](const float (&sum)[2], uint32_t there, int t) {
    float w = there >> t & 1 ? sum[t] : 0.0f;
    w += across(w, 16);
    return w + across(w, 32);
  };
  // Rows of tokens before the first key's do not see these keys.
  const uint32_t start = !a.tree && begin > sp.before ? (begin - sp.before) * a.group / 16 * 16 : 0;
  if constexpr (STAY) {
    const uint32_t base = begin + wave * kTile;
    u32x4 k[2][NK], kw[2][KS], next[kChunks];
    uint32_t there = 0;
    float next_lse = 0, sum[2] = {0, 0};
    const auto fetch = [&](uint32_t row0) {
#pragma unroll
      for (int i = 0; i < kChunks; ++i) next[i] = row_chunk(row0, i * 256 + threadIdx.x);
      if (threadIdx.x < kRows) next_lse = row_lse(row0 + threadIdx.x);
    };
    if (start < rows) fetch(start);
    load(base, k, &there);
    operands(k, kw);
    uint32_t b = 0;
    for (uint32_t row0 = start; row0 < rows; row0 += kRows, b ^= 1) {
      uint8_t* q_at = ql + b * kRows * C * 16;
#pragma unroll
      for (int i = 0; i < kChunks; ++i) {
        const uint32_t n = i * 256 + threadIdx.x;
        *reinterpret_cast<u32x4*>(q_at + at(n / C, n % C)) = next[i];
      }
      if (threadIdx.x < kRows) ll[b * kRows + threadIdx.x] = next_lse;
      __syncthreads();
      if (row0 + kRows < rows) fetch(row0 + kRows);
      if (base < end) weigh(base, kw, q_at, ll + b * kRows, row0, rows - row0 < kRows ? rows - row0 : kRows, sum);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float w = joined(sum, there, t);
      if (!g) sums[wave * kTile + t * 16 + m] = w;
    }
  } else {
    const uint32_t step = 4 * kTile;
    bool first = true;
    for (uint32_t row0 = start; row0 < rows || first; row0 += kRows, first = false) {
      if (!first) __syncthreads();
      for (uint32_t i = threadIdx.x; i < kRows * C; i += 256)
        *reinterpret_cast<u32x4*>(ql + at(i / C, i % C)) = row_chunk(row0, i);
      for (uint32_t i = threadIdx.x; i < kRows; i += 256) ll[i] = row_lse(row0 + i);
      __syncthreads();
      const uint32_t some = row0 < rows ? (rows - row0 < kRows ? rows - row0 : kRows) : 0;
      u32x4 k[2][2][NK];
      uint32_t there[2];
      const auto add = [&](uint32_t base, auto b) {
        u32x4 kw[2][KS];
        float sum[2] = {0, 0};
        operands(k[b], kw);
        weigh(base, kw, ql, ll, row0, some, sum);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const float w = joined(sum, there[b], t);
          if (!g) {
            float* to = &sums[base - begin + t * 16 + m];
            *to = first ? w : *to + w;
          }
        }
      };
      uint32_t base = begin + wave * kTile;
      if (base < end) load(base, k[0], &there[0]);
      for (; base < end; base += 2 * step) {
        if (base + step < end) load(base + step, k[1], &there[1]);
        add(base, std::false_type());
        if (base + step >= end) break;
        if (base + 2 * step < end) load(base + 2 * step, k[0], &there[0]);
        add(base + step, std::true_type());
      }
    }
  }
  __syncthreads();
  for (uint32_t i = threadIdx.x; begin + i < end; i += 256) {
    const uint32_t key = begin + i;
    const uint64_t to = (static_cast<uint64_t>(seq) * a.c.heads + head) * a.scores_stride + key;
    a.scores_out[to] = (a.scores_in && key < sp.before ? a.decay * a.scores_in[to] : 0.0f) + sums[i];
  }
}

template <class T, bool F8, int DP, bool VX>
hipError_t launch_of(const AttnArgs& a, const AttnPlan& p, hipStream_t stream) {
  const uint32_t cells = p.splits * a.c.heads * a.s.num_seqs;
  hipError_t e = hipSuccess;
  if (a.score_q.data != a.q.data) {
    const uint64_t chunks = static_cast<uint64_t>(a.s.num_tokens) * a.q_heads * (a.c.dim / 8);
    e = launch(attention_keep_queries_kernel, static_cast<uint32_t>((chunks + 255) / 256), 256, stream, a);
    if (e != hipSuccess) return e;
  }
  if (!p.rows) {  // the weights fade, that is all
    const dim3 grid((a.s.max_len + kWeigh - 1) / kWeigh, a.c.heads, a.s.num_seqs);
    return launch(attention_finish_kernel<T, DP>, grid, 256, stream, a, 0);
  }
  if (p.stream) {
    if (p.tiles_per_wave == 1) {
      e = launch(attention_stream_kernel<T, F8, DP, VX, 1>, cells, 256, stream, a);
    } else {
      e = hipErrorInvalidValue;  // no plan has it
      if constexpr (stream_two_tiles(DP, F8, VX)) e = launch(attention_stream_kernel<T, F8, DP, VX, 2>, cells, 256, stream, a);
    }
  } else {
    const uint32_t grid = (cells + 7) / 8 * 8 * p.row_groups;
    e = p.tiles_per_wave == 1 ? launch(attention_rows_kernel<T, F8, DP, VX, 1>, grid, 256, stream, a, p.row_groups, cells)
                              : launch(attention_rows_kernel<T, F8, DP, VX, 2>, grid, 256, stream, a, p.row_groups, cells);
  }
  if (e != hipSuccess) return e;
  const uint32_t joins = p.splits > 1 ? p.rows : 0;
  const uint32_t weighs = a.logits ? (a.s.max_len + kWeigh - 1) / kWeigh : 0;
  if (joins + weighs) {
    e = launch(attention_finish_kernel<T, DP>, dim3(joins + weighs, a.c.heads, a.s.num_seqs), 256, stream, a, joins);
    if (e != hipSuccess) return e;
  }
  if (a.lse2) {
    const dim3 grid((a.s.max_len + a.score_len - 1) / a.score_len, a.c.heads, a.s.num_seqs);
    e = p.keys_stay ? launch(attention_scores_kernel<T, F8, DP, true>, grid, 256, stream, a)
                    : launch(attention_scores_kernel<T, F8, DP, false>, grid, 256, stream, a);
  }
  return e;
}

template <class T, bool F8, int DP>
hipError_t by_layout(const AttnArgs& a, const AttnPlan& p, const OpsKind& k, hipStream_t stream) {
  return k.layout == MMA_KV_LAYOUT_XPACKED ? launch_of<T, F8, DP, true>(a, p, stream)
                                           : launch_of<T, F8, DP, false>(a, p, stream);
}

template <class T, bool F8>
hipError_t by_dim(const AttnArgs& a, const AttnPlan& p, const OpsKind& k, hipStream_t stream) {
  return p.dim_pad == 64    ? by_layout<T, F8, 64>(a, p, k, stream)
         : p.dim_pad == 128 ? by_layout<T, F8, 128>(a, p, k, stream)
                            : by_layout<T, F8, 256>(a, p, k, stream);
}

}  // namespace

hipError_t launch_attention(const AttnArgs& a, const AttnPlan& p, const OpsKind& k, hipStream_t stream) {
  const bool f8 = k.cache_type == MMA_TYPE_F8;
  if (k.type == MMA_TYPE_BF16) return f8 ? by_dim<__bf16, true>(a, p, k, stream) : by_dim<__bf16, false>(a, p, k, stream);
  return f8 ? by_dim<_Float16, true>(a, p, k, stream) : by_dim<_Float16, false>(a, p, k, stream);
}

}  // namespace mma
