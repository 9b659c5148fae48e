// Append, commit and evict on the paged KV cache for gfx950 (MI355X). All three move
// bytes: what bounds them is HBM, or at small sizes a launch and the chain of loads from a
// sequence's length over its block table to the entry.
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
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

template <class T>
struct Pair;
template <>
struct Pair<__bf16> {
  typedef bf16x2 x2;
};
template <>
struct Pair<_Float16> {
  typedef f16x2 x2;
};

template <class T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {  // round to nearest even
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, typename Pair<T>::x2));
}
template <class T>
__device__ __forceinline__ void unpack8(u32x4 w, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t word = w[i];  // a bit cast of the vector's element itself would take its first one
    const f32x2 v = __builtin_convertvector(__builtin_bit_cast(typename Pair<T>::x2, word), f32x2);
    x[2 * i] = v[0];
    x[2 * i + 1] = v[1];
  }
}

// 8 values of a row; elements at any alignment if not wide.
__device__ __forceinline__ u32x4 load8(const uint8_t* p, bool wide) {
  if (wide) return *reinterpret_cast<const u32x4*>(p);
  const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = h[2 * i] | (static_cast<uint32_t>(h[2 * i + 1]) << 16);
  return r;
}
__device__ __forceinline__ void store8(uint8_t* p, u32x4 w, bool wide) {
  if (wide) {
    *reinterpret_cast<u32x4*>(p) = w;
    return;
  }
  uint16_t* h = reinterpret_cast<uint16_t*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    h[2 * i] = static_cast<uint16_t>(w[i]);
    h[2 * i + 1] = static_cast<uint16_t>(w[i] >> 16);
  }
}

// To 8 bits: divided by the scale, held within +-448, rounded to nearest even; NaN stays NaN.
__device__ __forceinline__ u32x2 to_f8(const float* x, float scale) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float v = x[i] / scale;
    y[i] = v != v ? v : fminf(fmaxf(v, -448.0f), 448.0f);
  }
  u32x2 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
    r[i] = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], w, true));
  }
  return r;
}

// ---------------------------------------------------------------- append
// The sequence of a row of the token tensors: the last one that starts at or before it.
// 64 starts at a time, one per lane, so that no load waits for another.
__device__ __forceinline__ uint32_t seq_of(const SeqArgs& s, uint32_t token) {
  if (!s.q_start) return token / s.max_tokens;
  const uint32_t lane = threadIdx.x % kOpsWave;
  uint32_t n = 0;
  for (uint32_t first = 0; first < s.num_seqs; first += kOpsWave) {
    const uint32_t i = first + lane;
    const bool before = i < s.num_seqs && s.q_start[i] <= static_cast<int32_t>(token);
    n += __popcll(__ballot(before));
  }
  return n ? n - 1 : 0;
}

constexpr uint32_t kRun = 16;  // tokens whose x-packed values a workgroup turns

// Where a token's entry lies: its block, or -1, and its place in it.
__device__ __forceinline__ int32_t entry_of(const AppendArgs& a, uint32_t seq, uint32_t token, uint32_t* at) {
  *at = 0;
  if (seq >= a.s.num_seqs) return -1;
  const SeqSpan sp = span_of(a.s, seq);
  const uint32_t i = token - sp.first, entry = sp.before + i;
  if (token < sp.first || i >= sp.count || entry >= sp.total) return -1;
  return block_at(a.c, a.s.table + static_cast<uint64_t>(seq) * a.s.table_stride, entry, at);
}

// x-packed values of kRun tokens and one head: through LDS, so that the tokens of a block, which lie side by
// side for each value, are written by one workgroup, in one store where the run fills an aligned part of it.
template <class T, bool F8>
__device__ __forceinline__ void append_turned(const AppendArgs& a, uint32_t first, uint32_t head, uint16_t* tile, int32_t* ids,
                                              uint32_t* ats) {
  const uint32_t n = a.s.num_tokens - first < kRun ? a.s.num_tokens - first : kRun, D = a.c.dim;
  constexpr uint32_t S = kRun + 2;  // of a value's row in LDS: an odd number of dwords
  if (threadIdx.x < kOpsWave) {  // lane t finds token t's place, all at once
    const uint32_t lane = threadIdx.x;
    uint32_t seq = 0;
    if (!a.s.q_start) {
      seq = (first + lane) / a.s.max_tokens;
    } else {
      for (uint32_t s0 = 0; s0 < a.s.num_seqs; s0 += kOpsWave) {
        const int32_t start = s0 + lane < a.s.num_seqs ? a.s.q_start[s0 + lane] : INT32_MAX;
#pragma unroll
        for (uint32_t t = 0; t < kRun; ++t) {
          const uint32_t before = __popcll(__ballot(start <= static_cast<int32_t>(first + t)));
          if (lane == t) seq += before;
        }
      }
      seq = seq ? seq - 1 : 0;
    }
    if (lane < n) {
      uint32_t at;
      ids[lane] = entry_of(a, seq, first + lane, &at);
      ats[lane] = at;
    }
  }
  const float scale = a.v_scale ? a.v_scale[head] : 1.0f;
  for (uint32_t u = threadIdx.x; u < n * (D / 8); u += 256) {
    const uint32_t t = u / (D / 8), d0 = u % (D / 8) * 8;
    const u32x4 w = load8(a.v.data + 2 * ((first + t) * a.v.token + head * a.v.head + d0), a.wide);
    if constexpr (F8) {
      float x[8];
      unpack8<T>(w, x);
      const u32x2 y = to_f8(x, scale);
#pragma unroll
      for (int j = 0; j < 8; ++j) tile[(d0 + j) * S + t] = y[j / 4] >> (j % 4 * 8) & 0xff;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) tile[(d0 + j) * S + t] = static_cast<uint16_t>(w[j / 2] >> (j % 2 * 16));
    }
  }
  __syncthreads();
  bool whole = n == kRun && ids[0] >= 0 && ats[0] % kRun == 0;  // blocks hold a multiple of 8 (16 of 8 bits)
  for (uint32_t t = 1; t < n; ++t) whole = whole && ids[t] == ids[0] && ats[t] == ats[0] + t;
  for (uint32_t d = threadIdx.x; d < D; d += 256) {
    const uint16_t* row = tile + d * S;
    uint8_t* const base = a.c.v + head * a.c.v_head + static_cast<uint64_t>(d) * a.c.v_chunk;
    if (whole) {
      uint8_t* to = base + static_cast<uint64_t>(ids[0]) * a.c.block_bytes + static_cast<uint64_t>(ats[0]) * a.c.v_token;
      u32x4 w[2];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (F8) {
          if (i < 4) w[0][i] = row[4 * i] | row[4 * i + 1] << 8 | row[4 * i + 2] << 16 | static_cast<uint32_t>(row[4 * i + 3]) << 24;
        } else {
          w[i / 4][i % 4] = row[2 * i] | static_cast<uint32_t>(row[2 * i + 1]) << 16;
        }
      }
      *reinterpret_cast<u32x4*>(to) = w[0];
      if constexpr (!F8) *reinterpret_cast<u32x4*>(to + 16) = w[1];
    } else {
      for (uint32_t t = 0; t < n; ++t) {
        if (ids[t] < 0) continue;
        uint8_t* to = base + static_cast<uint64_t>(ids[t]) * a.c.block_bytes + static_cast<uint64_t>(ats[t]) * a.c.v_token;
        if constexpr (F8)
          *to = static_cast<uint8_t>(row[t]);
        else
          *reinterpret_cast<uint16_t*>(to) = row[t];
      }
    }
  }
}

// L lanes have a row of a token: L * 8 >= head_dim values. Rows of a token are its query heads,
// then its keys, then (but for x-packed values) its values; a workgroup takes `parts`-th parts of
// them. Where there are many tokens it takes all: what the rows share (position, place in the
// cache, cosines and sines) is then read once. The first workgroups, whose chain of loads is longest, turn x-packed
// values. One token: 4.3 us, a launch and that chain; 4095 tokens of 48 rows of 128 f16 values (86 MB): 17.9 us, 4.8
// TB/s, memory; 680 tokens to x-packed 8 bits (12 MB): 9.8 us, the chain and then single bytes, as a draft's run seldom fills
// 16 aligned tokens of a value, from as many threads as a head has values.
template <class T, bool F8, bool VX, int L>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a, uint32_t parts) {
  constexpr uint32_t kRows = 256 / L;
  constexpr uint32_t kTurn = kRows * (L * 8 + 1) * 4, kTile = VX ? L * 8 * (kRun + 2) * 2 : 0;
  __shared__ __attribute__((aligned(16))) uint8_t lds[kTurn > kTile ? kTurn : kTile];
  const uint32_t turns = VX ? (a.s.num_tokens + kRun - 1) / kRun * a.c.heads : 0;
  if constexpr (VX) {
    __shared__ int32_t ids[kRun];
    __shared__ uint32_t ats[kRun];
    if (blockIdx.x < turns) {
      const uint32_t u = blockIdx.x;
      append_turned<T, F8>(a, u / a.c.heads * kRun, u % a.c.heads, reinterpret_cast<uint16_t*>(lds), ids, ats);
      return;
    }
  }
  float(*turn)[L * 8 + 1] = reinterpret_cast<float(*)[L * 8 + 1]>(lds);
  const uint32_t lane = threadIdx.x % L, slot = threadIdx.x / L;
  const uint32_t block_row = blockIdx.x - turns, token = block_row / parts, part = block_row % parts;
  const uint32_t heads = a.c.heads, rows = a.q_heads + (VX ? 1 : 2) * heads;
  const uint32_t d0 = lane * 8, D = a.c.dim, R = a.rot_dim, half = R / 2;
  // Pairs a multiple of 8 apart: a lane's 8 partners are another lane's 8 values, its cosines 32 bytes in a row.
  const bool paired = !a.interleaved && half % 8 == 0;
  const uint32_t seq = seq_of(a.s, token);  // by all lanes of a wave
  float cs[8], sn[8];
  if (R) {
    int32_t p = a.positions[token];
    p = p < 0 ? 0 : p >= static_cast<int64_t>(a.rope_rows) ? static_cast<int32_t>(a.rope_rows - 1) : p;
    const float* t = a.rope + static_cast<uint64_t>(p) * R;
    if (d0 < R) {
      if (paired) {
        const uint32_t j = d0 < half ? d0 : d0 - half;
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
          const f32x4 c = *reinterpret_cast<const f32x4*>(t + j + i), s = *reinterpret_cast<const f32x4*>(t + half + j + i);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            cs[i + k] = c[k];
            sn[i + k] = s[k];
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t d = d0 + i < R ? d0 + i : R - 1, j = a.interleaved ? d / 2 : d < half ? d : d - half;
          cs[i] = t[j];
          sn[i] = t[half + j];
        }
      }
    }
  }
  int32_t id = -1;
  uint32_t at = 0;
  if (part * kRows + 255 / L >= a.q_heads || parts == 1) id = entry_of(a, seq, token, &at);
  const uint64_t block = static_cast<uint64_t>(id < 0 ? 0 : id) * a.c.block_bytes;
  for (uint32_t row0 = part * kRows; row0 < rows; row0 += parts * kRows) {
    const uint32_t row = row0 + slot;
    const uint32_t kind = row < a.q_heads ? 0 : row < a.q_heads + heads ? 1 : 2;
    const uint32_t head = kind == 0 ? row : kind == 1 ? row - a.q_heads : row - a.q_heads - heads;
    const bool on = row < rows && d0 < D;
    float x[8] = {};
    if (on) {
      const RowArgs& src = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
      unpack8<T>(load8(src.data + 2 * (token * src.token + head * src.head + d0), a.wide), x);
    }
    const void* weight = kind == 0 ? a.q_weight : kind == 1 ? a.k_weight : nullptr;
    if (a.q_weight || a.k_weight) {
      float sq = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) sq += x[i] * x[i];
#pragma unroll
      for (int i = 1; i < L; i *= 2) sq += __shfl_xor(sq, i, kOpsWave);
      if (weight && on) {
        const float by = 1.0f / sqrtf(sq / D + a.eps);
        float w[8];
        unpack8<T>(load8(static_cast<const uint8_t*>(weight) + 2 * d0, a.wide), w);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] * by * w[i];
      }
    }
    if (R && row0 < a.q_heads + heads) {
      const bool turns = on && kind < 2 && d0 < R, low = d0 < half;
      if (a.interleaved) {
        if (turns) {
#pragma unroll
          for (int i = 0; i < 8; i += 2)
            if (d0 + i < R) {
              const float u = x[i], v = x[i + 1];
              x[i] = u * cs[i] - v * sn[i];
              x[i + 1] = v * cs[i] + u * sn[i];
            }
        }
      } else if (paired) {
        const uint32_t other = threadIdx.x % kOpsWave / L * L + (low ? lane + half / 8 : lane - half / 8) % L;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float v = __shfl(x[i], other, kOpsWave);
          if (turns) x[i] = low ? x[i] * cs[i] - v * sn[i] : x[i] * cs[i] + v * sn[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) turn[slot][i * L + lane] = x[i];
        __syncthreads();
        if (turns) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const uint32_t d = d0 + i;
            if (d < R) {
              const uint32_t o = d < half ? d + half : d - half;
              const float v = turn[slot][o % 8 * L + o / 8];
              x[i] = d < half ? x[i] * cs[i] - v * sn[i] : x[i] * cs[i] + v * sn[i];
            }
          }
        }
        __syncthreads();
      }
    }
    if (!on) continue;
    const u32x4 w = {pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]), pack2<T>(x[4], x[5]), pack2<T>(x[6], x[7])};
    if (kind == 0) {
      store8(a.out.data + 2 * (token * a.out.token + head * a.out.head + d0), w, a.wide);
      continue;
    }
    if (id < 0) continue;
    uint8_t* to = kind == 1 ? a.c.k + block + head * a.c.k_head + static_cast<uint64_t>(at) * a.c.k_token
                            : a.c.v + block + head * a.c.v_head + static_cast<uint64_t>(at) * a.c.v_token;
    const uint64_t chunk = kind == 1 ? a.c.k_chunk : a.c.v_chunk;
    if constexpr (F8) {
      const float* scale = kind == 1 ? a.k_scale : a.v_scale;
      *reinterpret_cast<u32x2*>(to + d0 / 16 * chunk + d0 % 16) = to_f8(x, scale ? scale[head] : 1.0f);
    } else {
      *reinterpret_cast<u32x4*>(to + d0 / 8 * chunk) = w;
    }
  }
}

// ---------------------------------------------------------------- commit
// A thread has one 16-byte chunk (or x-packed value) of a head and takes the accepted
// entries in order: with ascending indices entry i's place is never the source of a later
// one, so that nothing but a thread's own order matters. What bounds it is the chain of
// loads from a sequence's length over the list and the block table to the entries, so one
// wave walks it once, for all threads, and a thread has 8 entries in flight. 32 layers of one sequence: 6 us; 24 layers
// of 24 sequences, 8 of 32 drafts each, x-packed 8 bits (10 MB): 15 us, as bytes of a value move one by one.
constexpr uint32_t kAhead = 8;    // entries loaded before the first of them is stored
constexpr uint32_t kMoves = 64;   // entries listed at a time, one per lane of the first wave

struct Moves {
  int32_t src[kMoves], dst[kMoves];      // blocks; dst is -1 where nothing moves
  uint32_t src_at[kMoves], dst_at[kMoves];
  int32_t token[kMoves];
  int32_t before;  // entries of the sequence
  int32_t count;  // of this time
  bool last;
};

template <class U>
__device__ __forceinline__ void move_entries(const Moves& l, uint64_t block_bytes, uint8_t* base, uint32_t token_stride) {
  for (int32_t i0 = 0; i0 < l.count; i0 += kAhead) {
    U x[kAhead];
    uint64_t to[kAhead];
    bool on[kAhead];
#pragma unroll
    for (uint32_t j = 0; j < kAhead; ++j) {
      const uint32_t i = i0 + j < kMoves ? i0 + j : kMoves - 1;
      on[j] = static_cast<int32_t>(i0 + j) < l.count && l.dst[i] >= 0;
      if (!on[j]) continue;
      to[j] = static_cast<uint64_t>(l.dst[i]) * block_bytes + static_cast<uint64_t>(l.dst_at[i]) * token_stride;
      x[j] = *reinterpret_cast<const U*>(base + static_cast<uint64_t>(l.src[i]) * block_bytes + static_cast<uint64_t>(l.src_at[i]) * token_stride);
    }
#pragma unroll
    for (uint32_t j = 0; j < kAhead; ++j)
      if (on[j]) *reinterpret_cast<U*>(base + to[j]) = x[j];
  }
}

template <bool F8, bool VX>
__global__ __launch_bounds__(256) void commit_kernel(CommitArgs a) {
  constexpr uint32_t E = F8 ? 1 : 2;
  __shared__ Moves list;
  const uint32_t layer = blockIdx.y, seq = blockIdx.z, lane = threadIdx.x % kOpsWave;
  const int32_t* acc = a.accepted + static_cast<uint64_t>(seq) * a.accepted_stride;
  const int32_t* table = a.s.table + static_cast<uint64_t>(seq) * a.s.table_stride;
  const uint32_t chunks = a.c.dim * E / 16, vs = VX ? a.c.dim : chunks, per = chunks + vs;
  uint8_t* const base = reinterpret_cast<uint8_t*>(a.layer[layer]);
  const uint32_t u = blockIdx.x * 256 + threadIdx.x, head = u / per, i = u % per;
  float* const scores = reinterpret_cast<float*>(a.scores[layer]);
  for (uint32_t first = 0;; first += kMoves) {
    if (threadIdx.x < kOpsWave) {
      const uint32_t at = first + lane;
      const int32_t j = at < a.accepted_stride ? acc[at] : -1, before = at && at < a.accepted_stride ? acc[at - 1] : -1;
      const int32_t c = a.counts[seq];
      SeqSpan sp = span_of(a.s, seq);
      if (!a.s.q_start)  // no token tensors here, whose rows would bound it
        sp.total = sp.before + (a.s.max_tokens < a.s.max_len - sp.before ? a.s.max_tokens : a.s.max_len - sp.before);
      const uint32_t n = c < 0 ? 0 : static_cast<uint32_t>(c) > a.accepted_stride ? a.accepted_stride : static_cast<uint32_t>(c);
      const bool good = at < n && j >= 0 && static_cast<uint32_t>(j) < sp.total - sp.before && j > before;
      const uint64_t bad = ~__ballot(good);
      const uint32_t count = bad ? __builtin_ctzll(bad) : kOpsWave;
      if (lane < count) {
        uint32_t st, dt;
        const int32_t sb = block_at(a.c, table, sp.before + j, &st), db = block_at(a.c, table, sp.before + at, &dt);
        list.src[lane] = sb;
        list.src_at[lane] = st;
        list.dst[lane] = static_cast<uint32_t>(j) == at || sb < 0 ? -1 : db;
        list.dst_at[lane] = dt;
        list.token[lane] = j;
      }
      if (!lane) {
        list.before = static_cast<int32_t>(sp.before);
        list.count = count;
        list.last = bad != 0;
        if (a.lens_out && bad && !layer && !blockIdx.x) a.lens_out[seq] = static_cast<int32_t>(sp.before + first + count);
      }
    }
    __syncthreads();
    if (head < a.c.heads) {
      if (i < chunks) {
        move_entries<u32x4>(list, a.c.block_bytes, base + head * a.c.k_head + static_cast<uint64_t>(i) * a.c.k_chunk, a.c.k_token);
      } else {
        uint8_t* v = base + a.v_offset + head * a.c.v_head + static_cast<uint64_t>(i - chunks) * a.c.v_chunk;
        if constexpr (!VX)
          move_entries<u32x4>(list, a.c.block_bytes, v, a.c.v_token);
        else if constexpr (F8)
          move_entries<uint8_t>(list, a.c.block_bytes, v, a.c.v_token);
        else
          move_entries<uint16_t>(list, a.c.block_bytes, v, a.c.v_token);
      }
    }
    if (scores) {  // a wave has a head's, 4 heads on their way at once
      const uint32_t step = gridDim.x * 4;
      for (uint32_t h0 = blockIdx.x * 4 + threadIdx.x / kOpsWave; h0 < a.c.heads; h0 += 4 * step) {
        float* w = scores + (static_cast<uint64_t>(seq) * a.c.heads + h0) * a.scores_stride + list.before;
        float x[4];
        const bool on = static_cast<int32_t>(lane) < list.count;
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k)
          if (on && h0 + k * step < a.c.heads) x[k] = w[static_cast<uint64_t>(k) * step * a.scores_stride + list.token[lane]];
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k)
          if (on && h0 + k * step < a.c.heads) w[static_cast<uint64_t>(k) * step * a.scores_stride + first + lane] = x[k];
      }
    }
    if (list.last) return;
    __syncthreads();
  }
}

// ---------------------------------------------------------------- evict
// Order of scores as unsigned numbers: NaN below all, the two zeros equal. 0 and kFixed are no score's.
constexpr uint32_t kFixed = 0xffffffffu;
__device__ __forceinline__ uint32_t order_of(float f) {
  uint32_t u = __builtin_bit_cast(uint32_t, f);
  if (f != f) return 1;
  if (u == 0x80000000u) u = 0;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr uint32_t kSelect = 1024;  // threads of a selection
constexpr uint32_t kWaves = kSelect / kOpsWave;
constexpr uint32_t kDigit = 11;     // bits of the threshold found at a time: 11, 11, 10
constexpr uint32_t kBins = 1u << kDigit;
constexpr uint32_t kCopies = 8;     // of the counters, for neighbouring lanes
constexpr uint32_t kCopyBins = kBins + 8;  // a counter's copies lie in different banks
constexpr uint32_t kListed = 16;    // longer rows (in 1024 entries) have their kept entries listed by a launch of its own

// The first and last entries have the highest order there is, places past the end the lowest: with more
// entries than are kept neither needs a condition of its own.
__device__ __forceinline__ uint32_t order_at(const EvictArgs& a, const float* w, uint32_t i, uint32_t n) {
  if (i >= n) return 0;
  return i < a.sinks || i >= n - a.recent ? kFixed : order_of(w[i]);
}

__device__ __forceinline__ uint32_t entries_of(const EvictArgs& a, uint32_t seq) {
  const int32_t len = a.s.lens[seq];
  const uint32_t n = len < 0 ? 0 : static_cast<uint32_t>(len);
  return n > a.s.max_len ? a.s.max_len : n;
}

// What the selection of a row (sequence and KV head) tells the workgroups that list its entries, in the
// workspace: { threshold, how many of those equal to it stay }, then for each 1024 entries { how many
// before them are above the threshold, how many equal to it }.
__device__ __forceinline__ uint32_t* selected(const EvictArgs& a, uint64_t row) {
  return a.chosen + row * 2 * (1 + (a.s.max_len + kSelect - 1) / kSelect);
}

// Sum over the workgroup of values of threads below this one (LDS: a word per wave).
__device__ __forceinline__ uint32_t exclusive_scan(uint32_t v, uint32_t* lds) {
  const uint32_t lane = threadIdx.x % kOpsWave, wave = threadIdx.x / kOpsWave;
  uint32_t x = v;
#pragma unroll
  for (int i = 1; i < kOpsWave; i *= 2) {
    const uint32_t y = __shfl_up(x, i, kOpsWave);
    if (lane >= static_cast<uint32_t>(i)) x += y;
  }
  __syncthreads();
  if (lane == kOpsWave - 1) lds[wave] = x;
  __syncthreads();
  uint32_t before = 0;
#pragma unroll
  for (uint32_t w = 0; w < kWaves; ++w) before += w < wave ? lds[w] : 0;
  return before + x - v;
}

// Which entries of one row stay. First the threshold, the order of the last that stays, found 11 bits at
// a time from the top by counting; where all entries that share the bits found so far stay, the rest need not
// be known. A thread has every 1024th score, N of them at a time in registers: up to 1024 N are read
// once; longer rows are read in each pass. Then counts of those above the threshold and equal to it, from ballots: a
// wave's k-th scores are 64 entries in a row, so (k, wave) is their order. Rows of up to 16 x 1024 are
// listed here; of longer ones, whose 64 scores a thread would go over some more times, the counts go to
// the workgroups of evict_list_kernel.
// What bounds it is one CU's arithmetic: about 10 instructions a score and pass. 8 rows of 64k scores: 33 us; 60 rows of
// 5k 12 us (16 scores a thread instead of 8: 16). Listed by a launch of their own, rows of 16k take 40 us in all, here 25.
template <uint32_t N>
__global__ __launch_bounds__(kSelect) void evict_select_kernel(EvictArgs a) {
  __shared__ __attribute__((aligned(8))) uint32_t bins[kCopyBins * kCopies];
  __shared__ uint32_t scan[kWaves], found[3], counts[N * kWaves];
  const uint32_t head = blockIdx.x, seq = blockIdx.y, lane = threadIdx.x % kOpsWave, wave = threadIdx.x / kOpsWave;
  const uint32_t n = entries_of(a, seq);
  const uint64_t row = static_cast<uint64_t>(seq) * a.c.heads + head;
  const float* w = a.scores + row * a.scores_stride;
  int32_t* out = a.entries + row * a.keep;
  float* ws = a.scores_out ? a.scores_out + row * a.keep : nullptr;
  const uint32_t kept = n < a.keep ? n : a.keep;
  if (!head && !threadIdx.x && a.lens_out) a.lens_out[seq] = static_cast<int32_t>(kept);
  for (uint32_t i = kept + threadIdx.x; i < a.keep; i += kSelect) {
    out[i] = -1;
    if (ws) ws[i] = 0;
  }
  if (n <= a.keep) {  // all stay
    for (uint32_t i = threadIdx.x; i < n; i += kSelect) {
      out[i] = static_cast<int32_t>(i);
      if (ws) ws[i] = w[i];
    }
    return;
  }
  const uint32_t segments = (n + N * kSelect - 1) / (N * kSelect);
  uint32_t order[N];
  const auto load = [&](uint32_t seg) {
    const uint32_t first = seg * N * kSelect + threadIdx.x;
    // Of this thread's: those below `some` exist, those from `lo` below `hi` compete.
    const auto below = [&](uint32_t i) -> uint32_t { return i <= first ? 0 : (i - first + kSelect - 1) / kSelect; };
    const uint32_t some = below(n), lo = below(a.sinks), hi = below(n - a.recent);
#pragma unroll
    for (uint32_t k = 0; k < N; ++k) order[k] = k < some ? __builtin_bit_cast(uint32_t, w[first + k * kSelect]) : 0;
#pragma unroll
    for (uint32_t k = 0; k < N; ++k)
      order[k] = k >= some ? 0 : k < lo || k >= hi ? kFixed : order_of(__builtin_bit_cast(float, order[k]));
  };
  load(0);
  uint32_t want = a.keep, prefix = 0;
  bool ties = true;  // more entries equal the threshold than are wanted
  for (int top = 32; top > 0 && ties; top -= kDigit) {
    const uint32_t shift = top > static_cast<int>(kDigit) ? top - kDigit : 0, digit = (1u << (top - shift)) - 1;
#pragma unroll
    for (uint32_t i = 0; i < kCopies; ++i) *reinterpret_cast<u32x2*>(&bins[i * kCopyBins + threadIdx.x * 2]) = u32x2{0, 0};
    __syncthreads();
    for (uint32_t seg = 0; seg < segments; ++seg) {
      if (segments > 1) load(seg);
      const uint32_t mask = top == 32 ? 0 : ~0u << top;
#pragma unroll
      for (uint32_t k = 0; k < N; ++k)
        if (((order[k] ^ prefix) & mask) == 0) atomicAdd(&bins[lane % kCopies * kCopyBins + (order[k] >> shift & digit)], 1u);
    }
    __syncthreads();
    // A thread has two bins, counted from the top; the one where the sum passes what is wanted is found by a scan.
    uint32_t b[2] = {0, 0};
#pragma unroll
    for (uint32_t c = 0; c < kCopies; ++c) {
      const u32x2 x = *reinterpret_cast<const u32x2*>(&bins[c * kCopyBins + kBins - 2 - threadIdx.x * 2]);
      b[0] += x[1];
      b[1] += x[0];
    }
    uint32_t above = exclusive_scan(b[0] + b[1], scan);
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i) {
      if (above < want && above + b[i] >= want) {  // one thread
        found[0] = kBins - 1 - (threadIdx.x * 2 + i);
        found[1] = want - above;
        found[2] = b[i];
      }
      above += b[i];
    }
    __syncthreads();
    prefix |= found[0] << shift;
    want = found[1];
    ties = found[2] != want;  // else all of the bin stay: those at its lowest order and above
    __syncthreads();
  }
  if (!ties) want = ~0u;
  const auto step = []() { if constexpr (N > kListed) __builtin_amdgcn_sched_barrier(0); };  // keeps one ballot in registers, not all

  if constexpr (N > kListed) {
    uint32_t* to = selected(a, row);
    if (!threadIdx.x) {
      to[0] = prefix;
      to[1] = want;
    }
    uint32_t above = 0, equal = 0;
    for (uint32_t seg = 0; seg < segments; ++seg) {
      if (segments > 1) load(seg);
#pragma unroll
      for (uint32_t k = 0; k < N; ++k) {
        const uint32_t c = __popcll(__ballot(order[k] > prefix)) << 16 | __popcll(__ballot(order[k] == prefix));
        if (!lane) counts[k * kWaves + wave] = c;
        step();
      }
      __syncthreads();
      if (wave == 0) {
        uint32_t c = 0;  // at most 1024 in each half
        if (lane < N)
#pragma unroll
          for (uint32_t i = 0; i < kWaves; ++i) c += counts[lane * kWaves + i];
        uint32_t hi = c >> 16, lo = c & 0xffff;
        const uint32_t my_hi = hi, my_lo = lo;
#pragma unroll
        for (uint32_t i = 1; i < N; i *= 2) {
          const uint32_t x = __shfl_up(hi, i, kOpsWave), y = __shfl_up(lo, i, kOpsWave);
          if (lane >= i) {
            hi += x;
            lo += y;
          }
        }
        const uint32_t chunk = seg * N + lane;
        if (lane < N && chunk * kSelect < n) {
          to[2 + 2 * chunk] = above + hi - my_hi;
          to[3 + 2 * chunk] = equal + lo - my_lo;
        }
        above += __builtin_amdgcn_readlane(hi, N - 1);
        equal += __builtin_amdgcn_readlane(lo, N - 1);
      }
      __syncthreads();
    }
    return;
  }

  // One segment. Both counts of a place in one word: at most 1024 N = 16384 of each.
  const auto sum_up = [&]() {
    __syncthreads();
    const uint32_t c = threadIdx.x < N * kWaves ? counts[threadIdx.x] : 0, at = exclusive_scan(c, scan);
    if (threadIdx.x < N * kWaves) counts[threadIdx.x] = at;
    __syncthreads();
  };
#pragma unroll
  for (uint32_t k = 0; k < N; ++k) {
    const uint32_t c = __popcll(__ballot(order[k] > prefix)) << 16 | __popcll(__ballot(order[k] == prefix));
    if (!lane) counts[k * kWaves + wave] = c;
  }
  sum_up();
  const uint64_t lower = (1ull << lane) - 1;
#pragma unroll
  for (uint32_t k = 0; k < N; ++k) {
    const uint32_t before = counts[k * kWaves + wave];
    const uint64_t gts = __ballot(order[k] > prefix), eqs = __ballot(order[k] == prefix);
    const uint32_t eq = (before & 0xffff) + __popcll(eqs & lower), at = (before >> 16) + __popcll(gts & lower) + (eq < want ? eq : want);
    if ((order[k] > prefix || (order[k] == prefix && eq < want)) && at < a.keep) {
      out[at] = static_cast<int32_t>(k * kSelect + threadIdx.x);
      if (ws) ws[at] = w[k * kSelect + threadIdx.x];
    }
  }
}

// Of 1024 entries of a long row, those that stay, to their place in the list.
__global__ __launch_bounds__(256) void evict_list_kernel(EvictArgs a) {
  constexpr uint32_t kMine = kSelect / 256;
  __shared__ uint32_t counts[kWaves];
  const uint32_t head = blockIdx.y, seq = blockIdx.z, first = blockIdx.x * kSelect, lane = threadIdx.x % kOpsWave, wave = threadIdx.x / kOpsWave;
  const uint32_t n = entries_of(a, seq);
  if (first >= n || n <= a.keep) return;
  const uint64_t row = static_cast<uint64_t>(seq) * a.c.heads + head;
  const float* w = a.scores + row * a.scores_stride;
  const uint32_t* chosen = selected(a, row);
  const uint32_t threshold = chosen[0], want = chosen[1], above = chosen[2 + 2 * blockIdx.x], equal = chosen[3 + 2 * blockIdx.x];
  uint32_t order[kMine];
  float f[kMine];
  uint64_t gts[kMine], eqs[kMine];
#pragma unroll
  for (uint32_t k = 0; k < kMine; ++k) {  // a wave has 256 entries in a row
    const uint32_t i = first + (wave * kMine + k) * kOpsWave + lane;
    f[k] = i < n ? w[i] : 0.0f;
    order[k] = order_at(a, w, i, n);
  }
#pragma unroll
  for (uint32_t k = 0; k < kMine; ++k) {
    gts[k] = __ballot(order[k] > threshold);
    eqs[k] = __ballot(order[k] == threshold);
    if (!lane) counts[wave * kMine + k] = __popcll(gts[k]) << 16 | __popcll(eqs[k]);
  }
  __syncthreads();
  uint32_t before = 0;
#pragma unroll
  for (uint32_t p = 0; p < kWaves; ++p) before += p < wave * kMine ? counts[p] : 0;
  const uint64_t lower = (1ull << lane) - 1;
#pragma unroll
  for (uint32_t k = 0; k < kMine; ++k) {
    const uint32_t eq = equal + (before & 0xffff) + __popcll(eqs[k] & lower);
    const uint32_t at = above + (before >> 16) + __popcll(gts[k] & lower) + (eq < want ? eq : want);
    if ((order[k] > threshold || (order[k] == threshold && eq < want)) && at < a.keep) {
      a.entries[row * a.keep + at] = static_cast<int32_t>(first + (wave * kMine + k) * kOpsWave + lane);
      if (a.scores_out) a.scores_out[row * a.keep + at] = f[k];
    }
    before += __popcll(gts[k]) << 16 | __popcll(eqs[k]);
  }
}

// The kept entries to their new blocks: kMoved of one head in a workgroup. Where they come from and go to is looked up
// once for all their chunks, and a thread has 4 chunks in flight. Reads and writes at the rate of a copy: 16k of 64k
// entries of 8 heads of 128 bf16 values (134 MB) in 33 us, 4.1 TB/s, kept entries being 256 bytes apart and more.
constexpr uint32_t kMoved = 64;

template <bool F8, bool VX>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a) {
  constexpr uint32_t E = F8 ? 1 : 2;
  __shared__ uint64_t from[kMoved], to[kMoved];  // of the blocks
  __shared__ uint32_t from_at[kMoved], to_at[kMoved];
  const uint32_t head = blockIdx.y, seq = blockIdx.z, first = blockIdx.x * kMoved;
  const uint32_t n = entries_of(a, seq), kept = n < a.keep ? n : a.keep;
  if (first >= kept) return;
  const uint32_t count = kept - first < kMoved ? kept - first : kMoved;
  constexpr uint64_t kNone = ~0ull;
  if (threadIdx.x < count) {
    const uint32_t e = first + threadIdx.x;
    uint32_t st, dt;
    const int32_t db = block_at(a.c, a.dst_table + static_cast<uint64_t>(seq) * a.dst_stride, e, &dt);
    const uint32_t src = static_cast<uint32_t>(a.entries[(static_cast<uint64_t>(seq) * a.c.heads + head) * a.keep + e]);
    const int32_t sb = block_at(a.c, a.s.table + static_cast<uint64_t>(seq) * a.s.table_stride, src, &st);
    from[threadIdx.x] = static_cast<uint64_t>(sb < 0 ? 0 : sb) * a.c.block_bytes;
    from_at[threadIdx.x] = st;
    to[threadIdx.x] = sb < 0 || db < 0 ? kNone : static_cast<uint64_t>(db) * a.c.block_bytes;
    to_at[threadIdx.x] = dt;
  }
  __syncthreads();
  const uint32_t chunks = a.c.dim * E / 16, per = VX ? chunks : 2 * chunks, total = count * per;
  constexpr uint32_t kU = 4;
  for (uint32_t u0 = threadIdx.x; u0 < total; u0 += 256 * kU) {
    u32x4 x[kU];
    uint8_t* p[kU];
#pragma unroll
    for (uint32_t j = 0; j < kU; ++j) {
      const uint32_t u = u0 + j * 256, e = u / per, i = u % per;
      p[j] = nullptr;
      if (u >= total || to[e] == kNone) continue;
      const bool key = i < chunks;
      uint8_t* base = key ? a.c.k + head * a.c.k_head + static_cast<uint64_t>(i) * a.c.k_chunk
                          : a.c.v + head * a.c.v_head + static_cast<uint64_t>(i - chunks) * a.c.v_chunk;
      const uint64_t ts = key ? a.c.k_token : a.c.v_token;
      x[j] = *reinterpret_cast<const u32x4*>(base + from[e] + from_at[e] * ts);
      p[j] = base + to[e] + to_at[e] * ts;
    }
#pragma unroll
    for (uint32_t j = 0; j < kU; ++j)
      if (p[j]) *reinterpret_cast<u32x4*>(p[j]) = x[j];
  }
  if constexpr (VX) {
    // A value of consecutive entries lies side by side where they go: consecutive threads write it.
    typedef typename std::conditional<F8, uint8_t, uint16_t>::type U;
    const uint32_t values = count * a.c.dim;
    for (uint32_t u0 = threadIdx.x; u0 < values; u0 += 256 * kU) {
      U x[kU];
      uint8_t* p[kU];
#pragma unroll
      for (uint32_t j = 0; j < kU; ++j) {
        const uint32_t u = u0 + j * 256, d = u / count, e = u % count;
        p[j] = nullptr;
        if (u >= values || to[e] == kNone) continue;
        uint8_t* base = a.c.v + head * a.c.v_head + static_cast<uint64_t>(d) * a.c.v_chunk;
        x[j] = *reinterpret_cast<const U*>(base + from[e] + from_at[e] * E);
        p[j] = base + to[e] + to_at[e] * E;
      }
#pragma unroll
      for (uint32_t j = 0; j < kU; ++j)
        if (p[j]) *reinterpret_cast<U*>(p[j]) = x[j];
    }
  }
}

template <class T, bool F8, bool VX>
hipError_t append_of(const AppendArgs& a, hipStream_t stream) {
  const uint32_t lanes = a.c.dim <= 64 ? 8 : a.c.dim <= 128 ? 16 : 32, per = 256 / lanes, n = a.s.num_tokens;
  const uint32_t all = (a.q_heads + (VX ? 1 : 2) * a.c.heads + per - 1) / per;
  // One workgroup for a token's rows where tokens alone fill the GPU, else one for each part of them (4095 tokens, 48
  // rows: 19 us, in parts 27; 256 to 700 tokens: the same within 0.5 us).
  const uint32_t parts = n >= 512 ? 1 : all;
  const uint32_t grid = n * parts + (VX ? (n + kRun - 1) / kRun * a.c.heads : 0);
  if (lanes == 8) return launch(append_kernel<T, F8, VX, 8>, grid, 256, stream, a, parts);
  if (lanes == 16) return launch(append_kernel<T, F8, VX, 16>, grid, 256, stream, a, parts);
  return launch(append_kernel<T, F8, VX, 32>, grid, 256, stream, a, parts);
}

template <class T>
hipError_t append_by(const AppendArgs& a, const OpsKind& k, hipStream_t stream) {
  const bool f8 = k.cache_type == MMA_TYPE_F8, vx = k.layout == MMA_KV_LAYOUT_XPACKED;
  return f8 ? vx ? append_of<T, true, true>(a, stream) : append_of<T, true, false>(a, stream)
            : vx ? append_of<T, false, true>(a, stream) : append_of<T, false, false>(a, stream);
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, const OpsKind& k, hipStream_t stream) {
  return k.type == MMA_TYPE_BF16 ? append_by<__bf16>(a, k, stream) : append_by<_Float16>(a, k, stream);
}

hipError_t launch_commit(const CommitArgs& a, const OpsKind& k, hipStream_t stream) {
  const bool f8 = k.cache_type == MMA_TYPE_F8, vx = k.layout == MMA_KV_LAYOUT_XPACKED;
  const uint32_t chunks = a.c.dim * (f8 ? 1 : 2) / 16, units = a.c.heads * (chunks + (vx ? a.c.dim : chunks));
  const dim3 grid((units + 255) / 256, a.layers, a.s.num_seqs);
  return f8 ? vx ? launch(commit_kernel<true, true>, grid, 256, stream, a) : launch(commit_kernel<true, false>, grid, 256, stream, a)
            : vx ? launch(commit_kernel<false, true>, grid, 256, stream, a) : launch(commit_kernel<false, false>, grid, 256, stream, a);
}

hipError_t launch_evict(const EvictArgs& a, const OpsKind& k, hipStream_t stream) {
  const bool f8 = k.cache_type == MMA_TYPE_F8, vx = k.layout == MMA_KV_LAYOUT_XPACKED;
  const dim3 pairs(a.c.heads, a.s.num_seqs);
  const bool listed = a.s.max_len <= kListed * kSelect;
  hipError_t e = a.s.max_len <= 8 * kSelect ? launch(evict_select_kernel<8>, pairs, kSelect, stream, a)
                 : listed                   ? launch(evict_select_kernel<kListed>, pairs, kSelect, stream, a)
                                            : launch(evict_select_kernel<64>, pairs, kSelect, stream, a);
  if (e != hipSuccess) return e;
  if (!listed) {
    e = launch(evict_list_kernel, dim3((a.s.max_len + kSelect - 1) / kSelect, a.c.heads, a.s.num_seqs), 256, stream, a);
    if (e != hipSuccess) return e;
  }
  const dim3 grid((std::min(a.keep, a.s.max_len) + kMoved - 1) / kMoved, a.c.heads, a.s.num_seqs);
  return f8 ? vx ? launch(evict_move_kernel<true, true>, grid, 256, stream, a) : launch(evict_move_kernel<true, false>, grid, 256, stream, a)
            : vx ? launch(evict_move_kernel<false, true>, grid, 256, stream, a) : launch(evict_move_kernel<false, false>, grid, 256, stream, a);
}

}  // namespace mma
