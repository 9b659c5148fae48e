// Append, commit and evict on the paged KV cache for gfx950 (MI355X). All three move
// bytes: what bounds them is HBM, or at small sizes a launch and the chain of loads from a
// sequence's length over its block table to the entry.
#include "mma_ops.h"

#include <algorithm>

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

// L lanes have a row of a token: L * 8 >= head_dim values. Rows of a token are its query
// heads, then its keys, then its values.
template <class T, bool F8, bool VX, int L>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
  constexpr uint32_t kRows = 256 / L;
  __shared__ float turn[kRows][L * 8 + 1];
  const uint32_t lane = threadIdx.x % L, slot = threadIdx.x / L;
  const uint32_t token = blockIdx.x;
  const uint32_t row = blockIdx.y * kRows + slot, heads = a.c.heads;
  const uint32_t d0 = lane * 8, D = a.c.dim, R = a.rot_dim;
  const uint32_t seq = seq_of(a.s, token);  // by all lanes of a wave
  const bool in = row < a.q_heads + 2 * heads;
  const uint32_t kind = row < a.q_heads ? 0 : row < a.q_heads + heads ? 1 : 2;
  const uint32_t head = kind == 0 ? row : kind == 1 ? row - a.q_heads : row - a.q_heads - heads;
  const bool on = in && d0 < D;
  float x[8] = {};
  if (on) {
    const RowArgs& src = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
    unpack8<T>(load8(src.data + 2 * (token * src.token + head * src.head + d0), a.wide), x);
  }
  const void* weight = kind == 0 ? a.q_weight : kind == 1 ? a.k_weight : nullptr;
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
  if (R) {
    int32_t p = a.positions[token];
    p = p < 0 ? 0 : p >= static_cast<int64_t>(a.rope_rows) ? static_cast<int32_t>(a.rope_rows - 1) : p;
    const float* cs = a.rope + static_cast<uint64_t>(p) * R;
    const uint32_t half = R / 2;
    if (a.interleaved) {
      if (on && kind < 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t d = d0 + 2 * i;
          if (d < R) {
            const float c = cs[d / 2], s = cs[half + d / 2], u = x[2 * i], v = x[2 * i + 1];
            x[2 * i] = u * c - v * s;
            x[2 * i + 1] = v * c + u * s;
          }
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) turn[slot][i * L + lane] = x[i];
      __syncthreads();
      if (on && kind < 2) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t d = d0 + i;
          if (d < R) {
            const bool low = d < half;
            const uint32_t j = low ? d : d - half, o = low ? d + half : j;
            const float c = cs[j], s = cs[half + j], v = turn[slot][o % 8 * L + o / 8];
            x[i] = low ? x[i] * c - v * s : x[i] * c + v * s;
          }
        }
      }
    }
  }
  if (!on) return;
  const u32x4 w = {pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]), pack2<T>(x[4], x[5]), pack2<T>(x[6], x[7])};
  if (kind == 0) {
    store8(a.out.data + 2 * (token * a.out.token + head * a.out.head + d0), w, a.wide);
    return;
  }
  if (seq >= a.s.num_seqs) return;
  const SeqSpan sp = span_of(a.s, seq);
  const uint32_t i = token - sp.first, entry = sp.before + i;
  if (token < sp.first || i >= sp.count || entry >= sp.total) return;
  uint32_t at;
  const int32_t id = block_at(a.c, a.s.table + static_cast<uint64_t>(seq) * a.s.table_stride, entry, &at);
  if (id < 0) return;
  const uint64_t block = static_cast<uint64_t>(id) * a.c.block_bytes;
  if (kind == 2 && VX) {
    uint8_t* to = a.c.v + block + head * a.c.v_head + static_cast<uint64_t>(at) * a.c.v_token;
    if constexpr (F8) {
      const u32x2 b = to_f8(x, a.v_scale ? a.v_scale[head] : 1.0f);
#pragma unroll
      for (int j = 0; j < 8; ++j) to[static_cast<uint64_t>(d0 + j) * a.c.v_chunk] = static_cast<uint8_t>(b[j / 4] >> (j % 4 * 8));
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        *reinterpret_cast<uint16_t*>(to + static_cast<uint64_t>(d0 + j) * a.c.v_chunk) = static_cast<uint16_t>(w[j / 2] >> (j % 2 * 16));
    }
    return;
  }
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

// ---------------------------------------------------------------- commit
// A thread has one 16-byte chunk (or x-packed value) of a head and takes the accepted
// entries in order: with ascending indices entry i's place is never the source of a later
// one, so that nothing but a thread's own order matters and no barrier is needed.
constexpr uint32_t kAhead = 4;  // entries loaded before the first of them is stored

// How many of a row's accepted tokens are moved: up to the first that is out of order or range.
__device__ __forceinline__ uint32_t accepted_count(const CommitArgs& a, uint32_t seq, uint32_t tokens, uint32_t* first_bad) {
  const int32_t* acc = a.accepted + static_cast<uint64_t>(seq) * a.accepted_stride;
  const int32_t c = a.counts[seq];
  const uint32_t n = c < 0 ? 0 : static_cast<uint32_t>(c) > a.accepted_stride ? a.accepted_stride : static_cast<uint32_t>(c);
  if (threadIdx.x == 0) *first_bad = n;
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < n; i += blockDim.x)
    if (acc[i] < 0 || static_cast<uint32_t>(acc[i]) >= tokens || (i && acc[i] <= acc[i - 1])) atomicMin(first_bad, i);
  __syncthreads();
  return *first_bad;
}

template <class U>
__device__ __forceinline__ void move_entries(const CommitArgs& a, const int32_t* table, const int32_t* acc, uint32_t n,
                                             uint32_t before, uint8_t* base, uint32_t token_stride) {
  for (uint32_t i0 = 0; i0 < n; i0 += kAhead) {
    U x[kAhead];
    uint8_t* to[kAhead];
#pragma unroll
    for (uint32_t j = 0; j < kAhead; ++j) {
      to[j] = nullptr;
      const uint32_t i = i0 + j;
      if (i >= n || acc[i] == static_cast<int32_t>(i)) continue;
      uint32_t st, dt;
      const int32_t sb = block_at(a.c, table, before + acc[i], &st), db = block_at(a.c, table, before + i, &dt);
      if (sb < 0 || db < 0) continue;
      x[j] = *reinterpret_cast<const U*>(base + static_cast<uint64_t>(sb) * a.c.block_bytes + static_cast<uint64_t>(st) * token_stride);
      to[j] = base + static_cast<uint64_t>(db) * a.c.block_bytes + static_cast<uint64_t>(dt) * token_stride;
    }
#pragma unroll
    for (uint32_t j = 0; j < kAhead; ++j)
      if (to[j]) *reinterpret_cast<U*>(to[j]) = x[j];
  }
}

template <bool F8, bool VX>
__global__ __launch_bounds__(256) void commit_kernel(CommitArgs a) {
  constexpr uint32_t E = F8 ? 1 : 2;
  __shared__ uint32_t first_bad;
  const uint32_t layer = blockIdx.x, seq = blockIdx.y;
  const SeqSpan sp = span_of(a.s, seq);
  const uint32_t n = accepted_count(a, seq, sp.total - sp.before, &first_bad);
  if (layer == 0 && threadIdx.x == 0 && a.lens_out) a.lens_out[seq] = static_cast<int32_t>(sp.before + n);
  const int32_t* acc = a.accepted + static_cast<uint64_t>(seq) * a.accepted_stride;
  const int32_t* table = a.s.table + static_cast<uint64_t>(seq) * a.s.table_stride;
  const uint32_t chunks = a.c.dim * E / 16, vs = VX ? a.c.dim : chunks, per = chunks + vs;
  uint8_t* const base = reinterpret_cast<uint8_t*>(a.layer[layer]);
  for (uint32_t u = threadIdx.x; u < a.c.heads * per; u += blockDim.x) {
    const uint32_t head = u / per, i = u % per;
    if (i < chunks) {
      move_entries<u32x4>(a, table, acc, n, sp.before, base + head * a.c.k_head + static_cast<uint64_t>(i) * a.c.k_chunk, a.c.k_token);
    } else {
      uint8_t* v = base + a.v_offset + head * a.c.v_head + static_cast<uint64_t>(i - chunks) * a.c.v_chunk;
      if constexpr (!VX)
        move_entries<u32x4>(a, table, acc, n, sp.before, v, a.c.v_token);
      else if constexpr (F8)
        move_entries<uint8_t>(a, table, acc, n, sp.before, v, a.c.v_token);
      else
        move_entries<uint16_t>(a, table, acc, n, sp.before, v, a.c.v_token);
    }
  }
  if (!a.scores[layer]) return;
  for (uint32_t head = threadIdx.x; head < a.c.heads; head += blockDim.x) {
    float* w = reinterpret_cast<float*>(a.scores[layer]) + (static_cast<uint64_t>(seq) * a.c.heads + head) * a.scores_stride + sp.before;
    for (uint32_t i = 0; i < n; ++i) w[i] = w[acc[i]];
  }
}

// ---------------------------------------------------------------- evict
// Order of scores as unsigned numbers: NaN lowest, the two zeros equal.
__device__ __forceinline__ uint32_t order_of(float f) {
  uint32_t u = __builtin_bit_cast(uint32_t, f);
  if (f != f) return 0;
  if (u == 0x80000000u) u = 0;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr uint32_t kSelect = 1024;  // threads of a selection

// Sum over the workgroup of values below this thread's, and of all (LDS: one word per wave and one more).
__device__ __forceinline__ uint32_t exclusive_scan(uint32_t v, uint32_t* lds, uint32_t* total) {
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
  uint32_t before = 0, all = 0;
  for (uint32_t w = 0; w < kSelect / kOpsWave; ++w) {
    const uint32_t n = lds[w];
    if (w < wave) before += n;
    all += n;
  }
  *total = all;
  return before + x - v;
}

// Which entries of one sequence and KV head stay: the number of scores wanted among those
// that compete gives a threshold, found 8 bits at a time from the top by counting (four
// passes over the scores), then one pass in order writes the entries above it and, of those
// equal to it, the first ones still wanted.
__global__ __launch_bounds__(kSelect) void evict_select_kernel(EvictArgs a) {
  __shared__ uint32_t bins[256], scan[kSelect / kOpsWave + 1], found[2];
  const uint32_t head = blockIdx.x, seq = blockIdx.y;
  const int32_t len = a.s.lens[seq];
  uint32_t n = len < 0 ? 0 : static_cast<uint32_t>(len);
  if (n > a.s.max_len) n = a.s.max_len;
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
  if (n <= a.keep) {
    for (uint32_t i = threadIdx.x; i < n; i += kSelect) {
      out[i] = static_cast<int32_t>(i);
      if (ws) ws[i] = w[i];
    }
    return;
  }
  const uint32_t lo = a.sinks, hi = n - a.recent;  // those that compete
  uint32_t want = a.keep - a.sinks - a.recent;
  uint32_t prefix = 0, equal = 0;  // the threshold's bits so far; how many of those equal to it stay
  if (want) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (uint32_t i = threadIdx.x; i < 256; i += kSelect) bins[i] = 0;
      __syncthreads();
      for (uint32_t i = lo + threadIdx.x; i < hi; i += kSelect) {
        const uint32_t u = order_of(w[i]);
        if (shift == 24 || u >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&bins[u >> shift & 255], 1u);
      }
      __syncthreads();
      if (threadIdx.x == 0) {
        uint32_t left = want, b = 255;
        while (b && bins[b] < left) left -= bins[b--];
        found[0] = b;
        found[1] = left;
      }
      __syncthreads();
      prefix |= found[0] << shift;
      want = found[1];
      __syncthreads();
    }
    equal = want;
  }
  const bool none = a.keep == a.sinks + a.recent;
  uint32_t base = 0, equals = 0;
  for (uint32_t i0 = 0; i0 < n; i0 += kSelect) {
    const uint32_t i = i0 + threadIdx.x;
    const bool live = i < n, fixed = live && (i < lo || i >= hi);
    const float f = live ? w[i] : 0;
    const uint32_t u = order_of(f);
    const bool competes = live && !fixed && !none;
    uint32_t total;
    const bool eq = competes && u == prefix;
    const uint32_t eq_before = equals + exclusive_scan(eq, scan, &total);
    equals += total;
    const bool stay = fixed || (competes && u > prefix) || (eq && eq_before < equal);
    const uint32_t at = base + exclusive_scan(stay, scan, &total);
    base += total;
    if (stay && at < a.keep) {
      out[at] = static_cast<int32_t>(i);
      if (ws) ws[at] = f;
    }
  }
}

// The kept entries to their new blocks: 8 of one head per row of threads.
template <bool F8, bool VX>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a) {
  constexpr uint32_t E = F8 ? 1 : 2;
  const uint32_t head = blockIdx.y, seq = blockIdx.z, first = blockIdx.x * 32;
  const int32_t len = a.s.lens[seq];
  uint32_t n = len < 0 ? 0 : static_cast<uint32_t>(len);
  if (n > a.s.max_len) n = a.s.max_len;
  const uint32_t kept = n < a.keep ? n : a.keep;
  if (first >= kept) return;
  const uint32_t count = kept - first < 32 ? kept - first : 32;
  const int32_t* from = a.entries + (static_cast<uint64_t>(seq) * a.c.heads + head) * a.keep + first;
  const int32_t* src = a.s.table + static_cast<uint64_t>(seq) * a.s.table_stride;
  const int32_t* dst = a.dst_table + static_cast<uint64_t>(seq) * a.dst_stride;
  const uint32_t chunks = a.c.dim * E / 16, per = VX ? chunks : 2 * chunks;
  for (uint32_t u = threadIdx.x; u < count * per; u += blockDim.x) {
    const uint32_t e = u / per, i = u % per;
    uint32_t st, dt;
    const int32_t sb = block_at(a.c, src, static_cast<uint32_t>(from[e]), &st), db = block_at(a.c, dst, first + e, &dt);
    if (sb < 0 || db < 0) continue;
    const bool key = i < chunks;
    uint8_t* base = key ? a.c.k + head * a.c.k_head + static_cast<uint64_t>(i) * a.c.k_chunk
                        : a.c.v + head * a.c.v_head + static_cast<uint64_t>(i - chunks) * a.c.v_chunk;
    const uint64_t ts = key ? a.c.k_token : a.c.v_token;
    *reinterpret_cast<u32x4*>(base + static_cast<uint64_t>(db) * a.c.block_bytes + dt * ts) =
        *reinterpret_cast<const u32x4*>(base + static_cast<uint64_t>(sb) * a.c.block_bytes + st * ts);
  }
  if constexpr (VX) {
    for (uint32_t u = threadIdx.x; u < count * a.c.dim; u += blockDim.x) {
      const uint32_t d = u / count, e = u % count;
      uint32_t st, dt;
      const int32_t sb = block_at(a.c, src, static_cast<uint32_t>(from[e]), &st), db = block_at(a.c, dst, first + e, &dt);
      if (sb < 0 || db < 0) continue;
      uint8_t* base = a.c.v + head * a.c.v_head + static_cast<uint64_t>(d) * a.c.v_chunk;
      const uint8_t* s = base + static_cast<uint64_t>(sb) * a.c.block_bytes + st * E;
      uint8_t* t = base + static_cast<uint64_t>(db) * a.c.block_bytes + dt * E;
      if constexpr (F8)
        *t = *s;
      else
        *reinterpret_cast<uint16_t*>(t) = *reinterpret_cast<const uint16_t*>(s);
    }
  }
}

template <class T, bool F8, bool VX>
hipError_t append_of(const AppendArgs& a, hipStream_t stream) {
  const uint32_t lanes = a.c.dim <= 64 ? 8 : a.c.dim <= 128 ? 16 : 32, rows = 256 / lanes;
  const dim3 grid(a.s.num_tokens, (a.q_heads + 2 * a.c.heads + rows - 1) / rows);
  if (lanes == 8)
    append_kernel<T, F8, VX, 8><<<grid, 256, 0, stream>>>(a);
  else if (lanes == 16)
    append_kernel<T, F8, VX, 16><<<grid, 256, 0, stream>>>(a);
  else
    append_kernel<T, F8, VX, 32><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
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
  const dim3 grid(a.layers, a.s.num_seqs);
  if (f8 && vx)
    commit_kernel<true, true><<<grid, 256, 0, stream>>>(a);
  else if (f8)
    commit_kernel<true, false><<<grid, 256, 0, stream>>>(a);
  else if (vx)
    commit_kernel<false, true><<<grid, 256, 0, stream>>>(a);
  else
    commit_kernel<false, false><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_evict(const EvictArgs& a, const OpsKind& k, hipStream_t stream) {
  const bool f8 = k.cache_type == MMA_TYPE_F8, vx = k.layout == MMA_KV_LAYOUT_XPACKED;
  evict_select_kernel<<<dim3(a.c.heads, a.s.num_seqs), kSelect, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const uint32_t most = std::min(a.keep, a.s.max_len);
  const dim3 grid((most + 31) / 32, a.c.heads, a.s.num_seqs);
  if (f8 && vx)
    evict_move_kernel<true, true><<<grid, 256, 0, stream>>>(a);
  else if (f8)
    evict_move_kernel<true, false><<<grid, 256, 0, stream>>>(a);
  else if (vx)
    evict_move_kernel<false, true><<<grid, 256, 0, stream>>>(a);
  else
    evict_move_kernel<false, false><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace mma
