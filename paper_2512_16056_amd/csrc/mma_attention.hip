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
// V^T comes as 8 keys' rows of the lane's head values, turned in registers (v_perm), or
// from the x-packed layout, where 8 tokens of a value are contiguous, as it stands.
#include "mma_ops.h"

#include <algorithm>

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
  static __device__ __forceinline__ uint32_t from_f8(uint32_t w, bool high) {  // exact
    return high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true))
                : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
  }
  static constexpr uint32_t kExponent = 0x7f80;
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
  static __device__ __forceinline__ uint32_t from_f8(uint32_t w, bool high) {
    return high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true))
                : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false));
  }
  static constexpr uint32_t kExponent = 0x7c00;
};

template <class T>
__device__ __forceinline__ float to_float(uint32_t bits16) {
  return static_cast<float>(__builtin_bit_cast(T, static_cast<uint16_t>(bits16)));
}

__device__ __forceinline__ float across(float v, int mask) { return __shfl_xor(v, mask, kOpsWave); }

// Shape of a kernel: head padded to DP values; CE values of an entry's V in one lane, over
// 16 lanes and NP panels; KS instructions of 32 values for a tile of keys.
template <bool F8, int DP, bool VX>
struct Shape {
  static constexpr int E = F8 ? 1 : 2;
  static constexpr int KS = DP / 32;
  static constexpr int CE = DP == 64 ? 4 : 8;
  static constexpr int NP = DP / (16 * CE);
  static constexpr int NC = NP * CE;  // instructions of 16 head values
  // Head value of V^T row r (0..15) of instruction c.
  static __device__ __forceinline__ uint32_t value_at(int c, uint32_t r) {
    return VX ? c * 16 + r : (c / CE) * 16 * CE + r * CE + c % CE;
  }
};

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
// group g start at 32 s + 8 g, or for 8-bit keys at 64 (s / 2) + 16 g + 8 (s % 2).
template <bool F8, int KS>
__device__ __forceinline__ void load_q(const AttnArgs& a, uint32_t head, uint32_t token, bool live, uint32_t g, u32x4* q) {
  const uint8_t* p = a.q.data + 2 * (token * a.q.token + head * a.q.head);
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const uint32_t d = F8 ? (s / 2) * 64 + g * 16 + (s % 2) * 8 : s * 32 + g * 8;
    q[s] = live && d < a.c.dim ? load_row8(p + 2 * d, a.wide_q) : u32x4{0, 0, 0, 0};
  }
}

// Blocks of the 8 keys key .. key + 7 (a lane's own): one if blocks hold a multiple of 8.
struct Keys {
  int32_t block[8];
  uint32_t token[8];
  uint32_t ok;  // bit j: key + j is below `end` and its block is there
};

// A tile of keys as the first operand: halves t, instruction s. Raw bytes for 8-bit keys:
// 16 of them serve instructions 2 s and 2 s + 1.
template <bool F8, int KS>
struct KeyTile {
  static constexpr int N = F8 ? KS / 2 : KS;
  u32x4 w[2][N];
  template <class T>
  __device__ __forceinline__ u32x4 operand(int t, int s) const {
    if constexpr (!F8) {
      return w[t][s];
    } else {
      const uint32_t x = w[t][s / 2][(s % 2) * 2], y = w[t][s / 2][(s % 2) * 2 + 1];
      return u32x4{Type<T>::from_f8(x, false), Type<T>::from_f8(x, true), Type<T>::from_f8(y, false),
                   Type<T>::from_f8(y, true)};
    }
  }
};

// Address of a key's first byte, with its block clamped into the cache.
__device__ __forceinline__ const uint8_t* key_at(const CacheArgs& c, const int32_t* row, uint32_t key, uint32_t head) {
  uint32_t token;
  const int32_t id = block_at(c, row, key, &token);
  return c.k + static_cast<uint64_t>(id < 0 ? 0 : id) * c.block_bytes + head * c.k_head + token * c.k_token;
}

// Keys base .. base + 31 of one head; `last` is the last entry that may be looked up.
template <bool F8, int KS>
__device__ __forceinline__ void load_keys(const CacheArgs& c, const int32_t* row, uint32_t base, uint32_t last, uint32_t head,
                                          uint32_t g, uint32_t m, KeyTile<F8, KS>& k) {
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    uint32_t key = base + (m / 4) * 8 + t * 4 + m % 4;
    if (key > last) key = last;
    const uint8_t* p = key_at(c, row, key, head);
#pragma unroll
    for (int s = 0; s < KeyTile<F8, KS>::N; ++s) {
      const uint32_t chunk = s * 4 + g;  // of 16 bytes
      k.w[t][s] = chunk * (F8 ? 16 : 8) < c.dim ? *reinterpret_cast<const u32x4*>(p + static_cast<uint64_t>(chunk) * c.k_chunk)
                                                : u32x4{0, 0, 0, 0};
    }
  }
}

// V^T of a tile: operand c has head value value_at(c, m) of keys base + 8 g .. + 7.
template <class T, bool F8, int DP, bool VX>
struct ValueTile {
  typedef Shape<F8, DP, VX> S;
  u32x4 op[S::NC];

  __device__ __forceinline__ void load(const CacheArgs& c, const int32_t* row, uint32_t base, uint32_t last, uint32_t head,
                                       uint32_t g, uint32_t m) {
    const uint8_t* at[8];
    const uint32_t first = base + g * 8;
    const bool one = c.tokens % 8 == 0;
    if constexpr (VX) {
      uint32_t token;
      const int32_t id = block_at(c, row, first > last ? last - last % 8 : first, &token);
      const uint8_t* p = c.v + static_cast<uint64_t>(id < 0 ? 0 : id) * c.block_bytes + head * c.v_head + token * c.v_token;
#pragma unroll
      for (int n = 0; n < S::NC; ++n) {
        const uint32_t d = S::value_at(n, m);
        const uint8_t* q = p + static_cast<uint64_t>(d) * c.v_chunk;
        if constexpr (F8) {
          const u32x2 w = d < c.dim ? *reinterpret_cast<const u32x2*>(q) : u32x2{0, 0};
          op[n] = u32x4{Type<T>::from_f8(w[0], false), Type<T>::from_f8(w[0], true), Type<T>::from_f8(w[1], false),
                        Type<T>::from_f8(w[1], true)};
        } else {
          op[n] = d < c.dim ? *reinterpret_cast<const u32x4*>(q) : u32x4{0, 0, 0, 0};
        }
      }
    } else {
      if (one) {
        uint32_t token;
        const int32_t id = block_at(c, row, first > last ? last : first, &token);
        const uint32_t stay = first > last ? 0 : 1;  // past the end: the last entry, eight times
        const uint8_t* p = c.v + static_cast<uint64_t>(id < 0 ? 0 : id) * c.block_bytes + head * c.v_head;
#pragma unroll
        for (int j = 0; j < 8; ++j) at[j] = p + static_cast<uint64_t>(token + j * stay) * c.v_token;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          uint32_t token;
          const int32_t id = block_at(c, row, first + j > last ? last : first + j, &token);
          at[j] = c.v + static_cast<uint64_t>(id < 0 ? 0 : id) * c.block_bytes + head * c.v_head +
                  static_cast<uint64_t>(token) * c.v_token;
        }
      }
      constexpr int W = S::CE / 2;  // dwords of 16-bit values in a lane's part of a panel
#pragma unroll
      for (int n = 0; n < S::NP; ++n) {
        const uint32_t d = n * 16 * S::CE + m * S::CE;
        const bool live = d < c.dim;
        uint32_t w[8][W];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint8_t* q = at[j] + d * S::E;  // a row is contiguous
          if constexpr (F8) {
            uint32_t b[W / 2];
            if constexpr (W == 4) {
              const u32x2 x = live ? *reinterpret_cast<const u32x2*>(q) : u32x2{0, 0};
              b[0] = x[0];
              b[1] = x[1];
            } else {
              b[0] = live ? *reinterpret_cast<const uint32_t*>(q) : 0;
            }
#pragma unroll
            for (int i = 0; i < W; ++i) w[j][i] = Type<T>::from_f8(b[i / 2], i % 2);
          } else if constexpr (W == 4) {
            const u32x4 x = live ? *reinterpret_cast<const u32x4*>(q) : u32x4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < W; ++i) w[j][i] = x[i];
          } else {
            const u32x2 x = live ? *reinterpret_cast<const u32x2*>(q) : u32x2{0, 0};
            w[j][0] = x[0];
            w[j][1] = x[1];
          }
        }
        // 8 keys x CE values: value e of keys 2 i and 2 i + 1 side by side
#pragma unroll
        for (int e = 0; e < S::CE; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            op[n * S::CE + e][i] =
                __builtin_amdgcn_perm(w[2 * i + 1][e / 2], w[2 * i][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
      }
    }
  }

  // Keys whose bit in `ok` is clear count as 0.
  __device__ __forceinline__ void keep(uint32_t ok) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t mask = (ok >> (2 * i) & 1 ? 0xffffu : 0u) | (ok >> (2 * i + 1) & 1 ? 0xffff0000u : 0u);
#pragma unroll
      for (int n = 0; n < S::NC; ++n) op[n][i] &= mask;
    }
  }
  // Bits of the keys with an infinity or NaN among the lane's values, which become 0.
  __device__ __forceinline__ uint32_t drop_nonfinite() {
    uint32_t bad = 0;
#pragma unroll
    for (int n = 0; n < S::NC; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t w = op[n][i], lo = w & 0xffffu, hi = w >> 16, x = Type<T>::kExponent;
        const bool l = (lo & x) == x, h = (hi & x) == x;
        bad |= (l ? 1u : 0u) << (2 * i) | (h ? 1u : 0u) << (2 * i + 1);
        op[n][i] = (l ? 0 : lo) | (h ? 0 : hi << 16);
      }
    return bad;
  }
};

// The value at head value d of one entry, as a float.
template <class T, bool F8, bool VX>
__device__ __forceinline__ float value_of(const CacheArgs& c, const int32_t* row, uint32_t key, uint32_t head, uint32_t d) {
  uint32_t token;
  const int32_t id = block_at(c, row, key, &token);
  if (id < 0 || d >= c.dim) return 0;
  const uint8_t* p = c.v + static_cast<uint64_t>(id) * c.block_bytes + head * c.v_head + static_cast<uint64_t>(token) * c.v_token +
                     (VX ? static_cast<uint64_t>(d) * c.v_chunk : static_cast<uint64_t>(d) * (F8 ? 1 : 2));
  if constexpr (F8) return to_float<T>(Type<T>::from_f8(*p, false));
  return to_float<T>(*reinterpret_cast<const uint16_t*>(p));
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
  uint32_t seen = 0;
#pragma unroll
  for (uint32_t j = 0; j < 8; ++j) {
    bool see = key + j < sp.before;
    if (!see) {
      const uint32_t d = key + j - sp.before;
      if (!a.tree)
        see = d <= token;
      else if (d / 64 < a.tree_words)
        see = a.tree[static_cast<uint64_t>(sp.first + token) * a.tree_words + d / 64] >> (d % 64) & 1;
    }
    seen |= (see ? 1u : 0u) << j;
  }
  return seen;
}

// ---------------------------------------------------------------- the main kernel
// A workgroup has R tiles of rows of one sequence and KV head and one split of its
// entries; its 4 waves take the split's tiles in turn, each with its own running maximum
// and sum, and are joined in LDS at the end. Nothing is shared before that: a tile's
// bytes go from memory to the registers that the matrix instructions read.
template <class T, bool F8, int DP, bool VX, int R>
__global__ __launch_bounds__(256) void attention_kernel(AttnArgs a) {
  typedef Shape<F8, DP, VX> S;
  const uint32_t wave = threadIdx.x / kOpsWave, lane = threadIdx.x % kOpsWave, g = lane / 16, m = lane % 16;
  const uint32_t split = blockIdx.x % a.splits, group = blockIdx.x / a.splits;
  const uint32_t head = blockIdx.y, seq = blockIdx.z;
  const SeqSpan sp = span_of(a.s, seq);
  const uint32_t rows = sp.count * a.group;
  const uint32_t row0 = group * R * 16;
  if (row0 >= rows) return;
  const uint32_t begin = split * a.split_len;
  if (begin >= sp.total && split) return;  // the first split also writes the rows that have no entries
  // Without a tree no row of the workgroup sees entries past its last token's.
  const uint32_t last_token = (row0 + R * 16 < rows ? row0 + R * 16 - 1 : rows - 1) / a.group;
  uint32_t end = begin + a.split_len < sp.total ? begin + a.split_len : sp.total;
  if (!a.tree && end > sp.before + last_token + 1) end = sp.before + last_token + 1;
  const int32_t* table = a.s.table + static_cast<uint64_t>(seq) * a.s.table_stride;

  u32x4 q[R][S::KS];
  uint32_t token[R];
  bool live[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const uint32_t row = row0 + r * 16 + m;
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

  uint32_t base = begin + wave * kTile;
  KeyTile<F8, S::KS> k;
  if (base < end) load_keys<F8, S::KS>(a.c, table, base, end - 1, head, g, m, k);
  for (; base < end; base += 4 * kTile) {
    ValueTile<T, F8, DP, VX> v;
    v.load(a.c, table, base, end - 1, head, g, m);
    f32x4 s[R][2];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int t = 0; t < 2; ++t) s[r][t] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < S::KS; ++i)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const u32x4 x = k.template operand<T>(t, i);
#pragma unroll
        for (int r = 0; r < R; ++r) s[r][t] = Type<T>::mfma(x, q[r][i], s[r][t]);
      }
    if (base + 4 * kTile < end) load_keys<F8, S::KS>(a.c, table, base + 4 * kTile, end - 1, head, g, m, k);

    const uint32_t ok = keys_there(a.c, table, base + g * 8, end);
    const bool inner = base + kTile <= sp.before;  // every row sees every entry
    const bool plain = __all(ok == 0xff) && inner;
    u32x4 p[R];
    uint32_t seen[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = s[r][j / 4][j % 4] * to_log2;
      seen[r] = 0xff;
      if (!plain) {
        seen[r] = inner ? ok : ok & keys_seen(a, sp, token[r], base + g * 8);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = seen[r] >> j & 1 ? x[j] : -INFINITY;
      }
      float mx = top[r];
#pragma unroll
      for (int j = 0; j < 8; ++j) mx = fmaxf(mx, x[j]);
      mx = fmaxf(mx, across(mx, 16));
      mx = fmaxf(mx, across(mx, 32));
      const float fade = __builtin_amdgcn_exp2f(top[r] - mx);
      top[r] = mx;
      float add = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[j] = __builtin_amdgcn_exp2f(x[j] - mx);
        add += x[j];
      }
      sum[r] = sum[r] * fade + add;  // this lane's keys; its 4 lanes are joined at the end
      // The probabilities are rounded to the type's 16 bits for the product with V, as the
      // output is: an error of the same size as the output's own. Their sum is not rounded.
#pragma unroll
      for (int i = 0; i < 4; ++i) p[r][i] = Type<T>::pack(x[2 * i], x[2 * i + 1]);
#pragma unroll
      for (int c = 0; c < S::NC; ++c) o[r][c] *= fade;
    }
    uint32_t bad = 0;
    if (!plain) {
      v.keep(ok);
      if (!inner) bad = v.drop_nonfinite();
    }
#pragma unroll
    for (int c = 0; c < S::NC; ++c)
#pragma unroll
      for (int r = 0; r < R; ++r) o[r][c] = Type<T>::mfma(v.op[c], p[r], o[r][c]);
    if (!plain && !inner && __any(bad)) {
      // A drafted token's V is infinite or NaN: it reaches the rows that see it, no others.
      for (uint32_t j = 0; j < kTile; ++j) {
        if (!__any(bad >> (j % 8) & 1 && g == j / 8)) continue;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const uint32_t from = (j / 8) * 16 + m;
          const uint32_t sees = __shfl(seen[r], from, kOpsWave) >> (j % 8) & 1;
          const uint32_t pw = j % 8 < 2 ? p[r][0] : j % 8 < 4 ? p[r][1] : j % 8 < 6 ? p[r][2] : p[r][3];
          const uint32_t pj = __shfl(pw, from, kOpsWave) >> (j % 2 * 16) & 0xffff;
          if (!sees || !live[r]) continue;
#pragma unroll
          for (int c = 0; c < S::NC; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float x = value_of<T, F8, VX>(a.c, table, base + j, head, S::value_at(c, g * 4 + i));
              if (!__builtin_isfinite(x)) o[r][c][i] += to_float<T>(pj) * x;
            }
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    sum[r] += across(sum[r], 16);
    sum[r] += across(sum[r], 32);
  }

  // Waves 2, 3 to 0, 1, then 1 to 0. A value's lane and register are the same in every wave.
  constexpr int NO = R * S::NC * 4;
  __shared__ float part[2][NO + 2 * R][kOpsWave];
#pragma unroll
  for (uint32_t step = 2; step >= 1; step /= 2) {
    if (wave >= step && wave < 2 * step) {
      float(*to)[kOpsWave] = part[wave - step];
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
    if (wave < step) {
      const float(*from)[kOpsWave] = part[wave];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float t = from[NO + 2 * r][lane], u = from[NO + 2 * r + 1][lane];
        const float mx = fmaxf(top[r], t);
        const float x = __builtin_amdgcn_exp2f(top[r] - mx), y = __builtin_amdgcn_exp2f(t - mx);
        top[r] = mx;
        sum[r] = sum[r] * x + u * y;
#pragma unroll
        for (int c = 0; c < S::NC; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[r][c][i] = o[r][c][i] * x + from[(r * S::NC + c) * 4 + i][lane] * y;
      }
    }
    __syncthreads();
  }
  if (wave) return;

  const float v_scale = a.v_scale ? a.v_scale[head] : 1.0f;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (!live[r]) continue;
    const uint32_t row = row0 + r * 16 + m, qh = head * a.group + row % a.group;
    const uint64_t unit = static_cast<uint64_t>(sp.first + token[r]) * a.q_heads + qh;
    if (a.splits > 1) {
      float* to = a.part + (unit * a.splits + split) * DP;
#pragma unroll
      for (int c = 0; c < S::NC; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) to[S::value_at(c, g * 4 + i)] = o[r][c][i] * v_scale;
      if (!g) {
        float* ml = a.part_ml + 2 * (unit * a.splits + split);
        ml[0] = top[r];
        ml[1] = sum[r];
      }
      continue;
    }
    const float by = sum[r] == 0 ? 0.0f : v_scale / sum[r];
    T* to = reinterpret_cast<T*>(a.out.data) + (sp.first + token[r]) * a.out.token + qh * a.out.head;
#pragma unroll
    for (int c = 0; c < S::NC; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t d = S::value_at(c, g * 4 + i);
        if (d < a.c.dim) to[d] = static_cast<T>(o[r][c][i] * by);
      }
    if (!g) {
      const float l2 = sum[r] == 0 ? -INFINITY : top[r] + __builtin_amdgcn_logf(sum[r]);
      if (a.lse) a.lse[unit] = l2 * kLn2;
      if (a.scores_out) a.part_ml[unit] = l2;
    }
  }
}

// ---------------------------------------------------------------- joining the splits
// Splits of one row: out = sum 2^(m_i - M) o_i / sum 2^(m_i - M) l_i. A wave has one row.
template <class T, int DP>
__global__ __launch_bounds__(256) void attention_join_kernel(AttnArgs a) {
  const uint32_t lane = threadIdx.x % kOpsWave;
  const uint32_t row = blockIdx.x * 4 + threadIdx.x / kOpsWave, head = blockIdx.y, seq = blockIdx.z;
  const SeqSpan sp = span_of(a.s, seq);
  if (row >= sp.count * a.group) return;
  const uint32_t token = sp.first + row / a.group, qh = head * a.group + row % a.group;
  const uint64_t unit = static_cast<uint64_t>(token) * a.q_heads + qh;
  uint32_t n = (sp.total + a.split_len - 1) / a.split_len;
  if (!n) n = 1;
  const float* ml = a.part_ml + 2 * unit * a.splits;
  float top = kLowest;
  for (uint32_t i = lane; i < n; i += kOpsWave) top = fmaxf(top, ml[2 * i]);
#pragma unroll
  for (int x = 1; x < kOpsWave; x *= 2) top = fmaxf(top, across(top, x));
  float sum = 0;
  constexpr int V = DP / kOpsWave;
  float o[V] = {};
  const float* part = a.part + unit * a.splits * DP + lane * V;
  for (uint32_t i = 0; i < n; ++i) {
    const float w = __builtin_amdgcn_exp2f(ml[2 * i] - top);
    sum += w * ml[2 * i + 1];
#pragma unroll
    for (int j = 0; j < V; ++j) o[j] += w * part[static_cast<uint64_t>(i) * DP + j];
  }
  const float by = sum == 0 ? 0.0f : 1.0f / sum;
  T* to = reinterpret_cast<T*>(a.out.data) + token * a.out.token + qh * a.out.head;
#pragma unroll
  for (int j = 0; j < V; ++j)
    if (lane * V + j < a.c.dim) to[lane * V + j] = static_cast<T>(o[j] * by);
  if (!lane) {
    const float l2 = sum == 0 ? -INFINITY : top + __builtin_amdgcn_logf(sum);
    if (a.lse) a.lse[unit] = l2 * kLn2;
    if (a.scores_out) a.part_ml[static_cast<uint64_t>(a.s.num_tokens) * a.q_heads * a.splits * 2 + unit] = l2;
  }
}

// ---------------------------------------------------------------- weights of the entries
// scores_out = decay scores_in + sum over the rows of p: with every row's sum known, Q K^T
// once more, this time rows down and keys across, so that a lane adds up its key's rows.
// A wave has 32 keys and goes through the rows; each score has one writer, so that the
// result does not depend on the order of waves.
template <class T, bool F8, int DP>
__global__ __launch_bounds__(256) void attention_scores_kernel(AttnArgs a, const float* lse2) {
  constexpr int KS = DP / 32;
  const uint32_t wave = threadIdx.x / kOpsWave, lane = threadIdx.x % kOpsWave, g = lane / 16, m = lane % 16;
  const uint32_t head = blockIdx.y, seq = blockIdx.z;
  const SeqSpan sp = span_of(a.s, seq);
  const uint32_t base = (blockIdx.x * 4 + wave) * kTile;
  if (base >= sp.total) return;
  const int32_t* table = a.s.table + static_cast<uint64_t>(seq) * a.s.table_stride;
  const uint32_t rows = sp.count * a.group;
  KeyTile<F8, KS> k;
  load_keys<F8, KS>(a.c, table, base, sp.total - 1, head, g, m, k);
  const float to_log2 = a.scale * kLog2e * (a.k_scale ? a.k_scale[head] : 1.0f);
  const bool inner = base + kTile <= sp.before;
  uint32_t key[2];
  bool there[2];
  float sum[2] = {0, 0};
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    uint32_t in_block;
    key[t] = base + (m / 4) * 8 + t * 4 + m % 4;
    there[t] = key[t] < sp.total && block_at(a.c, table, key[t], &in_block) >= 0;
  }
  for (uint32_t row0 = 0; row0 < rows; row0 += 16) {
    if (!a.tree && !inner && sp.before + (row0 + 15 < rows ? row0 + 15 : rows - 1) / a.group < base) continue;
    u32x4 q[KS];
    const uint32_t row = row0 + m;
    const bool live = row < rows;
    load_q<F8, KS>(a, head * a.group + (live ? row % a.group : 0), sp.first + (live ? row / a.group : 0), live, g, q);
    float l2[4];
    uint32_t token[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x = row0 + g * 4 + i;
      token[i] = x / a.group;
      l2[i] = x < rows ? lse2[static_cast<uint64_t>(sp.first + token[i]) * a.q_heads + head * a.group + x % a.group]
                       : INFINITY;
      if (l2[i] == -INFINITY) l2[i] = INFINITY;  // a row that sees nothing
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f32x4 s = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < KS; ++i) s = Type<T>::mfma(q[i], k.template operand<T>(t, i), s);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        bool see = there[t] && row0 + g * 4 + i < rows;
        if (!inner && see && key[t] >= sp.before) {
          const uint32_t d = key[t] - sp.before;
          see = a.tree ? d / 64 < a.tree_words &&
                             (a.tree[static_cast<uint64_t>(sp.first + token[i]) * a.tree_words + d / 64] >> (d % 64) & 1)
                       : d <= token[i];
        }
        const float p = __builtin_amdgcn_exp2f(s[i] * to_log2 - l2[i]);
        sum[t] += see ? p : 0.0f;
      }
    }
  }
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    sum[t] += across(sum[t], 16);
    sum[t] += across(sum[t], 32);
    if (g == t && key[t] < sp.total) {
      const uint64_t at = (static_cast<uint64_t>(seq) * a.c.heads + head) * a.scores_stride + key[t];
      a.scores_out[at] = (a.scores_in && key[t] < sp.before ? a.decay * a.scores_in[at] : 0.0f) + sum[t];
    }
  }
}

template <class T, bool F8, int DP, bool VX>
hipError_t launch_of(const AttnArgs& a, const AttnPlan& p, hipStream_t stream) {
  const dim3 grid(p.splits * p.row_groups, a.c.heads, a.s.num_seqs);
  if (p.tiles_per_wg == 1)
    attention_kernel<T, F8, DP, VX, 1><<<grid, 256, 0, stream>>>(a);
  else
    attention_kernel<T, F8, DP, VX, 2><<<grid, 256, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (p.splits > 1) {
    attention_join_kernel<T, DP><<<dim3((p.rows + 3) / 4, a.c.heads, a.s.num_seqs), 256, 0, stream>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.scores_out) {
    const float* lse2 = a.part_ml + (p.splits > 1 ? static_cast<uint64_t>(a.s.num_tokens) * a.q_heads * p.splits * 2 : 0);
    attention_scores_kernel<T, F8, DP>
        <<<dim3((a.s.max_len + 4 * kTile - 1) / (4 * kTile), a.c.heads, a.s.num_seqs), 256, 0, stream>>>(a, lse2);
    e = hipGetLastError();
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
