// Host side of the operators on the paged KV cache: argument checks, the split of an
// attention call and of a beam selection, and the rotary table. The kernels are in mma_attention_kernels.h,
// mma_kv_ops.hip, mma_beam.hip and mma_pages.hip; nothing here allocates or waits.
#include "mma_ops.h"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <initializer_list>

#include "mma_engine.h"
#include "mma_plan.h"

namespace mma {
namespace {

constexpr uint32_t kMaxDim = 256;
constexpr uint32_t kMaxGrid = 65535;  // sequences and heads are grid axes
constexpr uint64_t kMaxRows = 1ull << 26;  // tokens x heads: a launch has below 2^32 threads

// An allocation found by a check of this call. Allocations live as long as the call that is handed
// pointers into them, so what lies inside one already found needs no question to the runtime (0.07 us
// each; a commit of 32 layers and their scores would ask 64 times).
struct Known {
  uint64_t base = 0, size = 0;
};

struct Call {
  int device = 0;
  Known known[4];
  uint32_t next = 0;
  CacheArgs c{};
  SeqArgs s{};
  uint64_t piece = 0, layer_bytes = 0;
};

// Makes the library's device the current one for the launches.
struct Device {
  int prev = -1;
  explicit Device(int dev) {
    if (hipGetDevice(&prev) != hipSuccess) prev = -1;
    if (prev != dev) (void)hipSetDevice(dev);
    now = dev;
  }
  ~Device() {
    if (prev >= 0 && prev != now) (void)hipSetDevice(prev);
  }
  int now;
};

bool aligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// n * m elements of `bytes` each, or UINT64_MAX.
uint64_t extent(uint64_t n, uint64_t m, uint64_t bytes) {
  uint64_t r;
  if (__builtin_mul_overflow(n, m, &r) || __builtin_mul_overflow(r, bytes, &r)) return UINT64_MAX;
  return r;
}

// An output and an input that the kernels read while others of the same launch write: they may not share memory.
mma_status_t apart(const char* out, const void* p, uint64_t n, const char* in, const void* q, uint64_t m) {
  const uint64_t a = reinterpret_cast<uint64_t>(p), b = reinterpret_cast<uint64_t>(q);
  if (!p || !q || !n || !m || (a < b ? b - a >= n : a - b >= m)) return MMA_OK;
  return fail(MMA_ERR_INVALID_ARG, "%s overlaps %s", out, in);
}

mma_status_t device_range(Call* call, const void* p, uint64_t bytes) {
  const uint64_t at = reinterpret_cast<uint64_t>(p);
  for (const Known& k : call->known)
    if (at >= k.base && bytes <= k.size && at - k.base <= k.size - bytes) return MMA_OK;
  Known& k = call->known[call->next++ % 4];
  k = Known{};
  Known got;
  if (mma_status_t s = ops_device_range(p, bytes, &got.base, &got.size)) return s;
  k = got;
  return MMA_OK;
}

// A device array of the call; NULL only where it may be absent.
mma_status_t array(Call* call, const char* what, const void* p, uint64_t bytes, uintptr_t align, bool optional = false) {
  if (!p) {
    if (optional) return MMA_OK;
    return fail(MMA_ERR_INVALID_ARG, "%s is NULL", what);
  }
  if (!aligned(p, align)) return fail(MMA_ERR_INVALID_ARG, "%s has to be %u-byte aligned", what, static_cast<unsigned>(align));
  if (bytes == UINT64_MAX) return fail(MMA_ERR_INVALID_ARG, "%s: its size is beyond 64 bits", what);
  return bytes ? device_range(call, p, bytes) : MMA_OK;
}

// Token rows [tokens][heads][dim] of 2-byte values.
mma_status_t rows(Call* call, const char* what, const mma_rows_t& r, uint32_t tokens, uint32_t heads, uint32_t dim, bool written,
                  RowArgs* out) {
  uint64_t a, b, n;
  if (__builtin_mul_overflow(static_cast<uint64_t>(tokens - 1), r.token_stride, &a) ||
      __builtin_mul_overflow(static_cast<uint64_t>(heads - 1), r.head_stride, &b) || __builtin_add_overflow(a, b, &n) ||
      __builtin_add_overflow(n, static_cast<uint64_t>(dim), &n) || n > UINT64_MAX / 2)
    return fail(MMA_ERR_INVALID_ARG, "%s: its extent is beyond 64 bits", what);
  if (written) {  // no two rows may share a value
    const bool by_token = (heads == 1 || r.head_stride >= dim) && (tokens == 1 || r.token_stride >= b + dim);
    const bool by_head = (tokens == 1 || r.token_stride >= dim) && (heads == 1 || r.head_stride >= a + dim);
    if (!by_token && !by_head) return fail(MMA_ERR_INVALID_ARG, "%s: its rows overlap", what);
  }
  if (mma_status_t s = array(call, what, r.data, 2 * n, 2)) return s;
  out->data = static_cast<uint8_t*>(r.data);
  out->token = r.token_stride;
  out->head = r.head_stride;
  return MMA_OK;
}

// Whether the memory from the first to the last value of two [tokens][heads][dim] rows meets.
bool rows_meet(const RowArgs& x, const RowArgs& y, uint32_t tokens, uint32_t heads, uint32_t dim) {
  const auto end = [&](const RowArgs& r) { return r.data + 2 * ((tokens - 1) * r.token + (heads - 1) * r.head + dim); };
  return x.data < end(y) && y.data < end(x);
}

bool rows_wide(const RowArgs& r) { return aligned(r.data, 16) && r.token % 8 == 0 && r.head % 8 == 0; }

mma_status_t check_types(uint32_t type, uint32_t cache_type, uint32_t elem_bytes) {
  if (type != MMA_TYPE_BF16 && type != MMA_TYPE_F16) return fail(MMA_ERR_INVALID_ARG, "unknown type %u", type);
  if (cache_type != type && cache_type != MMA_TYPE_F8)
    return fail(MMA_ERR_INVALID_ARG, "a cache of type %u does not go with type %u", cache_type, type);
  if (elem_bytes != (cache_type == MMA_TYPE_F8 ? 1u : 2u))
    return fail(MMA_ERR_INVALID_ARG, "elem_bytes %u does not fit cache type %u", elem_bytes, cache_type);
  return MMA_OK;
}

// The layout, as far as no pointer is needed.
mma_status_t check_layout(const mma_kv_layout_t* lay, Call* call) {
  if (!lay) return fail(MMA_ERR_INVALID_ARG, "NULL layout");
  KvSizes sz;
  if (!kv_sizes(lay->num_layers, lay->block_tokens, lay->kv_heads, lay->head_dim, lay->elem_bytes, lay->gpu_num_blocks,
                lay->host_num_slots, kMaxLayers, &sz))
    return fail(MMA_ERR_INVALID_ARG, "invalid KV layout: a field is 0, more than %u layers, a piece above 4 GiB, "
                                     "or a pool or layer size beyond 64 bits", kMaxLayers);
  const uint32_t E = lay->elem_bytes, D = lay->head_dim, B = lay->block_tokens, H = lay->kv_heads;
  if (E != 1 && E != 2) return fail(MMA_ERR_INVALID_ARG, "the operators take elem_bytes 1 and 2");
  if (D % 8 || D > kMaxDim || D * E % 16)
    return fail(MMA_ERR_INVALID_ARG, "head_dim %u: the operators take multiples of 8 up to %u, and of 16 bytes", D, kMaxDim);
  if (H > kMaxGrid) return fail(MMA_ERR_INVALID_ARG, "%u KV heads, at most %u", H, kMaxGrid);
  if (lay->gpu_num_blocks > INT32_MAX) return fail(MMA_ERR_INVALID_ARG, "more than 2^31 - 1 blocks");
  CacheArgs& c = call->c;
  c.block_bytes = sz.piece;
  c.num_blocks = lay->gpu_num_blocks;
  c.tokens = B;
  c.heads = H;
  c.dim = D;
  // entry / B for entries below 2^31: with 2^(s-1) < B <= 2^s, m = 2^(31+s) / B + 1 errs by at most
  // B / 2^(31+s) <= 2^-31 per entry.
  uint32_t s = 0;
  while ((1ull << s) < B) ++s;
  c.div_mul = static_cast<uint32_t>((1ull << (31 + s)) / B + 1);
  c.div_shift = 31 + s;
  const uint64_t row = static_cast<uint64_t>(D) * E;
  uint64_t kh, kt, kc, vh, vt, vc;
  switch (lay->gpu_layout) {
    case MMA_KV_LAYOUT_PIECE:
      kh = vh = row;
      kt = vt = H * row;
      kc = vc = 16;
      break;
    case MMA_KV_LAYOUT_HND:
      kh = vh = B * row;
      kt = vt = row;
      kc = vc = 16;
      break;
    case MMA_KV_LAYOUT_XPACKED:
      if (static_cast<uint64_t>(B) * E % 16)
        return fail(MMA_ERR_INVALID_ARG, "x-packed KV layout needs block_tokens*elem_bytes a multiple of 16");
      kh = vh = B * row;
      kt = 16;
      kc = 16ull * B;
      vt = E;
      vc = static_cast<uint64_t>(B) * E;
      break;
    default:
      return fail(MMA_ERR_INVALID_ARG, "unknown GPU KV layout %u", lay->gpu_layout);
  }
  // Every product of a stride and an index below its bound is an offset within a piece (at most 2^32 - 1);
  // a stride that no index multiplies may be 2^32 itself.
  c.k_head = static_cast<uint32_t>(kh);
  c.k_token = static_cast<uint32_t>(kt);
  c.k_chunk = static_cast<uint32_t>(kc);
  c.v_head = static_cast<uint32_t>(vh);
  c.v_token = static_cast<uint32_t>(vt);
  c.v_chunk = static_cast<uint32_t>(vc);
  call->piece = sz.piece;
  call->layer_bytes = sz.layer;
  return MMA_OK;
}

mma_status_t check_layer(const void* layer, Call* call) {
  if (mma_status_t s = array(call, "the layer tensor", layer, call->layer_bytes, 16)) return s;
  call->c.k = static_cast<uint8_t*>(const_cast<void*>(layer));
  call->c.v = call->c.k + call->piece * call->c.num_blocks;
  return MMA_OK;
}

mma_status_t check_seqs_sizes(const mma_kv_seqs_t* q, uint32_t block_tokens) {
  if (!q) return fail(MMA_ERR_INVALID_ARG, "NULL sequences");
  if (q->num_seqs > kMaxGrid) return fail(MMA_ERR_INVALID_ARG, "%u sequences, at most %u", q->num_seqs, kMaxGrid);
  if (!q->max_len || q->max_len > static_cast<uint32_t>(INT32_MAX) - 4096 ||
      q->max_len > static_cast<uint64_t>(q->table_stride) * block_tokens)
    return fail(MMA_ERR_INVALID_ARG, "max_len %u: from 1 to table_stride * block_tokens (%llu), and below 2^31 - 4096",
                q->max_len, static_cast<unsigned long long>(q->table_stride) * block_tokens);
  return MMA_OK;
}

mma_status_t check_seqs(const mma_kv_seqs_t* q, uint32_t block_tokens, uint32_t num_tokens, Call* call) {
  mma_status_t s;
  if ((s = check_seqs_sizes(q, block_tokens))) return s;
  if ((s = array(call, "block_table", q->block_table, extent(q->num_seqs, q->table_stride, 4), 4))) return s;
  if ((s = array(call, "lens", q->lens, 4ull * q->num_seqs, 4))) return s;
  if ((s = array(call, "q_start", q->q_start, 4ull * q->num_seqs + 4, 4, true))) return s;
  SeqArgs& a = call->s;
  a.table = q->block_table;
  a.lens = q->lens;
  a.q_start = q->q_start;
  a.num_seqs = q->num_seqs;
  a.table_stride = q->table_stride;
  a.max_tokens = std::min(q->max_tokens, num_tokens);
  if (!q->q_start) a.max_tokens = q->max_tokens;  // the rows of a sequence start at its multiple
  a.max_len = q->max_len;
  a.num_tokens = num_tokens;
  return MMA_OK;
}

mma_status_t check_heads(uint32_t q_heads, uint32_t kv_heads, uint32_t num_tokens) {
  if (!q_heads || q_heads % kv_heads)
    return fail(MMA_ERR_INVALID_ARG, "%u query heads are not a multiple of %u KV heads", q_heads, kv_heads);
  if (static_cast<uint64_t>(num_tokens) * q_heads > kMaxRows || num_tokens > kMaxRows / 8)
    return fail(MMA_ERR_INVALID_ARG, "%u tokens of %u query heads in one call, at most 2^26 rows and 2^23 tokens", num_tokens,
                q_heads);
  return MMA_OK;
}

mma_status_t begin(Call* call) { return ops_ready(&call->device); }

mma_status_t launched(hipError_t e, const char* what) {
  return e == hipSuccess ? MMA_OK : fail(MMA_ERR_HIP, "%s launch failed: %s", what, hipGetErrorString(e));
}

uint32_t up(uint64_t n, uint32_t to) { return static_cast<uint32_t>((n + to - 1) / to); }

uint64_t up_to(uint64_t n, uint64_t to) { return (n + to - 1) / to * to; }

// How an attention call is cut. Rows of one sequence and KV head (a token and a head of
// the group each) go in tiles of 16; the entries go in splits, joined afterwards, where
// sequences, heads and rows alone are too few workgroups for 256 CUs.
AttnPlan attention_plan(const CacheArgs& c, const mma_kv_layout_t& layout, const mma_kv_seqs_t& q,
                        const mma_kv_attention_t& a, const mma_kv_shape_t* shape) {
  AttnPlan p{};
  const uint32_t group = a.q_heads / c.heads;
  const uint64_t tokens = std::min(q.max_tokens, a.num_tokens);
  p.rows = static_cast<uint32_t>(tokens * group);
  p.dim_pad = c.dim <= 64 ? 64 : c.dim <= 128 ? 128 : 256;
  // Up to two tiles of rows have their keys in registers (one with heads above 128: the second would not fit
  // them), if a lane's 8 keys share a block. 8 KV heads of 128 unless said. 8-bit and x-packed entries are best there
  // throughout (32 rows, 4 sequences of 3k to 15k, 8-bit x-packed: 32 us, through LDS 56; 4 rows, 32 sequences of 1k to 8k,
  // x-packed bf16: 128 against 153, 8-bit head-major 77 against 154). Of 16-bit entries with heads of 65 to 128 V costs
  // registers to be turned in, and from 17 rows on LDS is better, with fewer from some thousands of entries on, unless
  // their logits are kept (4 rows, bf16: 4 of 3k to 15k, head-major, 38.6 against 34.7, 32 of 1k to 8k 130 against 125, 64k in
  // pieces 59 against 55; but 6 x 900, head-major, 12.7 against 14.4, 64k with weights 70 against 83). Below 65 the two are
  // within 8 % (70 against 76), above 128 the registers win (4 heads of 256: 164 against 215).
  const bool two = stream_two_tiles(p.dim_pad, layout.elem_bytes == 1, layout.gpu_layout == MMA_KV_LAYOUT_XPACKED);
  p.stream = p.rows <= (two ? 32u : 16u) && c.tokens % 8 == 0;
  // Entries that a workgroup's rows walk over: with a window those of the prefix and of its tokens' windows, each to a
  // multiple of 64, and no more than there are.
  const auto walked = [&](uint32_t wg_rows) -> uint32_t {
    if (!shape || !shape->window) return q.max_len;
    const uint64_t prefix = shape->prefix ? std::min(shape->max_prefix, q.max_len) : 0;
    const uint64_t most = up_to(prefix, 64) + std::min<uint64_t>(tokens, wg_rows / group + 2) + shape->window + 64;
    return static_cast<uint32_t>(std::min<uint64_t>(most, q.max_len));
  };
  // Slopes and caps are more work for each entry, which the waves of attention_stream_kernel share and one wave of the other
  // has alone (4 rows, 32 of 1k to 8k, bf16, slopes: head-major 126 us against 150, in pieces 138 against 149). Windows go by
  // the threshold of whole contexts, 4096, though the two do not cross there: with one of 4096 and the first 4, f16, head-major,
  // 4 rows, keys in registers and in LDS take 12.8 and 19.7 us for one sequence, 30.9 and 33.4 for 8, 92.8 and 89.1 for 32.
  const bool shapes = shape && (shape->slopes || shape->softcap != 0);
  if (p.dim_pad == 128 && !two && walked(16) > 4096 && !a.scores_out && !shapes) p.stream = false;
  const uint32_t per_tile = p.stream ? 16 : 64;
  p.tiles_per_wave = p.rows > per_tile ? 2 : 1;
  p.wg_rows = per_tile * p.tiles_per_wave;
  p.row_groups = up(p.rows, p.wg_rows);
  const uint32_t most = walked(p.wg_rows);
  const uint64_t wgs = static_cast<uint64_t>(q.num_seqs) * c.heads * p.row_groups;
  // Workgroups in all: the 512 that run at once, so that all end together; but 2048 where many sequences, likely of
  // different lengths, would leave some of those idle (4 rows, 8 heads of 128, x-packed bf16: 32 of 1k to 8k 126 us against
  // 133, 8 heads of 64 in pieces 78 against 98). Where they are alike, or short, it costs: 32 of 4095 104 against 99, 64 of up
  // to 2k 67 against 59, in 8 bits 42 against 35. Entries of a split: 256 at least (4 rows over 1000 or 4096 entries: 128 the
  // same, 512 14.3 and 15.2 us against 12.0 and 12.5).
  const bool many = p.stream && static_cast<uint64_t>(q.num_seqs) * c.heads >= 64;
  const uint64_t want = many ? 2048 : 512, least = 256;
  uint64_t splits = wgs >= want ? 1 : up(want, std::max<uint64_t>(wgs, 1));
  splits = std::max<uint64_t>(1, std::min<uint64_t>(splits, up(most, least)));
  p.split_len = up(up(most, static_cast<uint32_t>(splits)), 128) * 128;
  p.splits = up(most, p.split_len);
  const uint64_t units = static_cast<uint64_t>(a.num_tokens) * a.q_heads;
  if (p.splits > 1) p.part_bytes = up_to(units * p.splits * p.dim_pad * 4, 256);
  if (a.scores_out) {
    // One tile's logits are kept: 8 bytes a row and entry there and back, against reading the keys again. With the keys
    // read again, 32 sequences of 1k to 8k entries of 8 KV heads, head-major, take this much (kept logits in brackets):
    // 4 rows: heads of 64 in 8 bits 77 us (56), of 128 in bf16 235 (162), of 256 in bf16 474 (300); 8 rows of 64 in 8 bits
    // 79 (73); 16 rows: of 64 in 8 bits 83 (93), in bf16 141 (137), of 128 in 8 bits 163 (143), in bf16 249 (214). So they
    // are kept up to one and a half times a key's bytes; and up to 1 GiB, for the workspace's sake.
    p.logit_stride = static_cast<uint32_t>(up_to(q.max_len, 32));
    const uint64_t kept = extent(static_cast<uint64_t>(q.num_seqs) * c.heads * p.rows, p.logit_stride, 4);
    p.logits = p.stream && p.tiles_per_wave == 1 && 16 * p.rows <= 3 * c.dim * layout.elem_bytes && kept <= 1u << 30;
    // Scores of many rows: keys stay in registers from 257 rows on (8192 rows over 8k entries, with the attention, 588 us
    // against 758), of several sequences from 65 on (192 rows, 4 x 15k: 173 against 190); 128 rows over one sequence
    // of 64k take 147 so and 136 with the rows staying.
    p.keys_stay = p.rows > (q.num_seqs > 1 ? 64u : 256u);
    if (p.logits) {
      p.logit_bytes = up_to(kept, 256);
    } else {
      p.lse_bytes = up_to(units * 4, 256);
      p.q_bytes = up_to(units * c.dim * 2, 256);  // of queries that `out` replaces before the weights are formed
    }
    // Shaped scores of many rows over few keys: the rows in parts, so that 1024 workgroups share them, of 256 rows at least
    // (3 x 1021 tokens x 4 heads, 8 KV heads, 8-bit x-packed: the weights 93 us, in one part 258; 61 with the present kernel).
    p.score_parts = 1;
    if (shape && p.keys_stay && !p.logits) {
      const uint64_t keys = static_cast<uint64_t>(up(q.max_len, 128)) * c.heads * q.num_seqs;
      p.score_parts = static_cast<uint32_t>(std::clamp<uint64_t>(1024 / std::max<uint64_t>(keys, 1), 1, std::max(1u, p.rows / 256)));
      if (p.score_parts > 1)
        p.score_bytes = up_to(extent(static_cast<uint64_t>(p.score_parts) * q.num_seqs * c.heads, q.max_len, 4), 256);
    }
  }
  if (p.splits > 1 || p.logits) p.ml_bytes = up_to(units * p.splits * 8, 256);
  p.bytes = p.part_bytes + p.ml_bytes + p.lse_bytes + p.q_bytes + p.logit_bytes + p.score_bytes;
  return p;
}

uint64_t evict_workspace(const mma_kv_seqs_t* q, uint32_t kv_heads) {
  return static_cast<uint64_t>(q->num_seqs) * kv_heads * 8 * (1 + up(q->max_len, 1024));
}

// What the split goes by, checked where no pointer is needed. A shape that shapes nothing becomes NULL.
mma_status_t check_attention_sizes(const mma_kv_layout_t* layout, const mma_kv_seqs_t* seqs, const mma_kv_attention_t* a,
                                   const mma_kv_shape_t** shape, Call* call) {
  mma_status_t s;
  if (!a) return fail(MMA_ERR_INVALID_ARG, "NULL arguments");
  if (const mma_kv_shape_t* x = *shape) {
    if (x->softcap != 0 && !(x->softcap >= 1e-6f && x->softcap <= 1024.0f))
      return fail(MMA_ERR_INVALID_ARG, "softcap has to be 0, or from 1e-6 to 1024");
    if (a->tree && (x->slopes || x->prefix || x->window))
      return fail(MMA_ERR_INVALID_ARG, "a drafted token's distance is not told by its tree: no slopes, prefix or window with one");
    if (x->softcap == 0 && !x->slopes && !x->prefix && !x->window) *shape = nullptr;
  }
  if ((s = check_layout(layout, call))) return s;
  if ((s = check_types(a->type, a->cache_type, layout->elem_bytes))) return s;
  if ((s = check_heads(a->q_heads, layout->kv_heads, a->num_tokens))) return s;
  return check_seqs_sizes(seqs, layout->block_tokens);
}

mma_status_t attention_workspace(const mma_kv_layout_t* layout, const mma_kv_seqs_t* seqs, const mma_kv_attention_t* a,
                                 const mma_kv_shape_t* shape, uint64_t* bytes) {
  if (!bytes) return fail(MMA_ERR_INVALID_ARG, "NULL argument");
  Call call;
  if (mma_status_t s = check_attention_sizes(layout, seqs, a, &shape, &call)) return s;
  *bytes = a->num_tokens && seqs->num_seqs && seqs->max_tokens ? attention_plan(call.c, *layout, *seqs, *a, shape).bytes : 0;
  return MMA_OK;
}

mma_status_t attention(const mma_kv_layout_t* layout, const void* layer, const mma_kv_seqs_t* seqs,
                       const mma_kv_attention_t* a, const mma_kv_shape_t* shape, void* stream) {
  mma_status_t s;
  Call call;
  if ((s = begin(&call))) return s;
  if ((s = check_attention_sizes(layout, seqs, a, &shape, &call))) return s;
  const uint32_t D = layout->head_dim, H = layout->kv_heads, n = a->num_tokens;
  if (a->tree && !a->tree_words) return fail(MMA_ERR_INVALID_ARG, "a tree needs tree_words");
  if (a->scores_in && !a->scores_out) return fail(MMA_ERR_INVALID_ARG, "scores_in without scores_out");
  if (a->scores_out && a->scores_stride < seqs->max_len)
    return fail(MMA_ERR_INVALID_ARG, "scores_stride %u is below max_len %u", a->scores_stride, seqs->max_len);
  const bool rows_too = n && seqs->max_tokens;  // else the entries' weights fade and no more
  if (!seqs->num_seqs || (!rows_too && !a->scores_out)) return MMA_OK;
  Device dev(call.device);
  if (rows_too && (s = check_layer(layer, &call))) return s;
  if ((s = check_seqs(seqs, layout->block_tokens, n, &call))) return s;
  CappedArgs k{};
  const uint64_t score_bytes = extent(static_cast<uint64_t>(seqs->num_seqs) * H, a->scores_stride, 4);
  if ((s = array(&call, "scores_in", a->scores_in, score_bytes, 4, true))) return s;
  if ((s = array(&call, "scores_out", a->scores_out, score_bytes, 4, true))) return s;
  if (a->scores_in != a->scores_out && (s = apart("scores_out", a->scores_out, score_bytes, "scores_in", a->scores_in, score_bytes)))
    return s;
  k.c = call.c;
  k.s = call.s;
  k.scores_in = a->scores_in;
  k.scores_out = a->scores_out;
  k.scores_stride = a->scores_stride;
  k.decay = a->decay;
  const OpsKind kind{a->type, a->cache_type, layout->gpu_layout};
  if (!rows_too)
    return launched(launch_attention(k, AttnPlan{}, kind, static_cast<hipStream_t>(stream)), "KV attention");
  if ((s = rows(&call, "q", a->q, n, a->q_heads, D, false, &k.q))) return s;
  if ((s = rows(&call, "out", a->out, n, a->q_heads, D, true, &k.out))) return s;
  if ((s = array(&call, "tree", a->tree, extent(n, a->tree_words, 8), 8, true))) return s;
  if ((s = array(&call, "lse", a->lse, extent(n, a->q_heads, 4), 4, true))) return s;
  if ((s = array(&call, "k_scale", a->k_scale, 4ull * H, 4, true))) return s;
  if ((s = array(&call, "v_scale", a->v_scale, 4ull * H, 4, true))) return s;
  const AttnPlan p = attention_plan(call.c, *layout, *seqs, *a, shape);
  if (static_cast<uint64_t>(p.row_groups) * (static_cast<uint64_t>(p.splits) * H * seqs->num_seqs + 7) >= 1ull << 24)
    return fail(MMA_ERR_INVALID_ARG, "%u sequences of up to %u tokens and %u KV heads are more workgroups than a launch takes",
                seqs->num_seqs, seqs->max_tokens, H);
  if (p.bytes) {
    if (a->workspace_bytes < p.bytes)
      return fail(MMA_ERR_BUFFER_TOO_SMALL, "the workspace has %llu bytes, %llu are needed",
                  static_cast<unsigned long long>(a->workspace_bytes), static_cast<unsigned long long>(p.bytes));
    if ((s = array(&call, "workspace", a->workspace, p.bytes, 256))) return s;
  }
  k.tree = a->tree;
  k.lse = a->lse;
  k.k_scale = a->cache_type == MMA_TYPE_F8 ? a->k_scale : nullptr;
  k.v_scale = a->cache_type == MMA_TYPE_F8 ? a->v_scale : nullptr;
  char* ws = static_cast<char*>(a->workspace);
  const auto take = [&](uint64_t bytes) {
    float* at = bytes ? reinterpret_cast<float*>(ws) : nullptr;
    ws += bytes;
    return at;
  };
  k.part = take(p.part_bytes);
  k.part_ml = take(p.ml_bytes);
  k.lse2 = take(p.lse_bytes);
  k.score_q = k.q;
  if (float* copy = take(p.q_bytes); copy && rows_meet(k.q, k.out, n, a->q_heads, D))
    k.score_q = RowArgs{reinterpret_cast<uint8_t*>(copy), static_cast<uint64_t>(a->q_heads) * D, D};
  k.logits = take(p.logit_bytes);
  k.logit_rows = p.rows;
  k.logit_stride = p.logit_stride;
  k.q_heads = a->q_heads;
  k.group = a->q_heads / H;
  k.tree_words = a->tree_words;
  // Entries of a workgroup: 32 for each of its waves where these stay, else 128 to 1024, its start being a few loads one
  // after the other: the 512 workgroups that run at once for one sequence, twice as many for several, whose lengths
  // differ (128 rows over 64k entries 151 us, with 1024 workgroups 172; 96 rows over 4 x 15k: 104 and 88).
  const uint64_t per = static_cast<uint64_t>(seqs->max_len) * seqs->num_seqs * H / (seqs->num_seqs == 1 ? 512 : 1024);
  k.score_len = p.keys_stay ? 128 : static_cast<uint32_t>(std::clamp<uint64_t>(up_to(per, 128), 128, 1024));
  k.splits = p.splits;
  k.split_len = p.split_len;
  k.wide_q = rows_wide(k.q);
  k.wide_out = rows_wide(k.out);
  k.wide_score_q = rows_wide(k.score_q);
  k.scale = a->scale;
  if (!shape) return launched(launch_attention(k, p, kind, static_cast<hipStream_t>(stream)), "KV attention");
  if ((s = array(&call, "slopes", shape->slopes, 4ull * a->q_heads, 4, true))) return s;
  if ((s = array(&call, "prefix", shape->prefix, 4ull * seqs->num_seqs, 4, true))) return s;
  k.slopes = shape->slopes;
  k.prefix = shape->prefix;
  k.max_prefix = shape->max_prefix;
  k.window = std::min<uint32_t>(shape->window, INT32_MAX);
  k.wg_rows = p.wg_rows;
  k.score_parts = std::max(1u, p.score_parts);
  k.score_part = take(p.score_bytes);
  if (shape->softcap == 0) return launched(launch_attention_shaped(k, p, kind, static_cast<hipStream_t>(stream)), "KV attention");
  const double cap2 = shape->softcap * 1.44269504088896340736;
  k.cap2 = static_cast<float>(cap2);
  constexpr double kTerms[5] = {0.9999999676372836, -0.3333279502358464, 0.1331887691419831, -0.052589319781746184, 0.01631544361405081};
  for (int i = 0; i < 5; ++i) k.cap_terms[i] = static_cast<float>(cap2 * kTerms[i]);  // of tanh(u) / u in u^2, u up to 0.55
  return launched(launch_attention_capped(k, p, kind, static_cast<hipStream_t>(stream)), "KV attention");
}

// Memory of a call that its kernels read or write.
struct Part {
  const char* name;
  const void* p;
  uint64_t bytes;
};

// Outputs apart from the inputs and from each other.
mma_status_t all_apart(std::initializer_list<Part> outs, std::initializer_list<Part> ins) {
  for (const Part* o = outs.begin(); o != outs.end(); ++o) {
    for (const Part& i : ins)
      if (mma_status_t s = apart(o->name, o->p, o->bytes, i.name, i.p, i.bytes)) return s;
    for (const Part* q = outs.begin(); q != o; ++q)
      if (mma_status_t s = apart(o->name, o->p, o->bytes, q->name, q->p, q->bytes)) return s;
  }
  return MMA_OK;
}

mma_status_t workspace(Call* call, void* p, uint64_t bytes, uint64_t need, uintptr_t align) {
  if (bytes < need)
    return fail(MMA_ERR_BUFFER_TOO_SMALL, "the workspace has %llu bytes, %llu are needed",
                static_cast<unsigned long long>(bytes), static_cast<unsigned long long>(need));
  return need ? array(call, "workspace", p, need, align) : MMA_OK;
}

struct BeamPlan {
  uint32_t splits, run;
  bool joined;  // each row's parts before the request's
  uint64_t sum_bytes, list_bytes, row_bytes, max_bytes, bytes;
};

mma_status_t check_beam_sizes(const mma_beam_select_t* a, BeamPlan* p) {
  if (!a) return fail(MMA_ERR_INVALID_ARG, "NULL arguments");
  if (a->type != MMA_TYPE_BF16 && a->type != MMA_TYPE_F16 && a->type != MMA_TYPE_F32)
    return fail(MMA_ERR_INVALID_ARG, "unknown type %u of logits", a->type);
  if (!a->beams || a->beams > kBeamMost) return fail(MMA_ERR_INVALID_ARG, "%u beams: from 1 to %u", a->beams, kBeamMost);
  if (!a->keep || a->keep > kBeamKeep) return fail(MMA_ERR_INVALID_ARG, "keep %u: from 1 to %u", a->keep, kBeamKeep);
  if (!a->vocab || a->vocab > INT32_MAX) return fail(MMA_ERR_INVALID_ARG, "a vocabulary of %u: from 1 to 2^31 - 1", a->vocab);
  // A part is as long as lets 1024 workgroups, four on a CU, run at once, or as lets a row's parts fit a merge: to find a
  // part's best costs as much as to sum some thousand logits, and what is found is merged (192 rows of 128001 in 1152
  // workgroups, of which the last 128 run alone: 46.5 us, in 960 40.9, both before the present kernel).
  const uint64_t chunks = up(a->vocab, kBeamChunk), rows = static_cast<uint64_t>(a->batch) * a->beams;
  const uint64_t run = std::max(up(chunks, static_cast<uint32_t>(std::max<uint64_t>(1, 1024 / std::max<uint64_t>(1, rows)))), up(chunks, kBeamMerge / a->keep));
  const uint64_t splits = up(chunks, static_cast<uint32_t>(std::min(run, chunks)));
  if (rows * splits >= 1u << 22)
    return fail(MMA_ERR_INVALID_ARG, "%u requests of %u beams are more workgroups than a launch takes", a->batch, a->beams);
  p->splits = static_cast<uint32_t>(splits);
  p->run = static_cast<uint32_t>(up(chunks, p->splits));
  p->joined = splits * a->keep * a->beams > kBeamMerge;
  p->sum_bytes = rows * splits * 8;
  p->list_bytes = rows * splits * a->keep * 8;
  p->row_bytes = p->joined ? rows * a->keep * 8 : 0;
  p->max_bytes = up_to(rows * splits * 4, 8);
  p->bytes = p->sum_bytes + p->list_bytes + p->row_bytes + p->max_bytes;
  return MMA_OK;
}

// Pages from[k] to to[k] of every layer; of a compaction the table too.
mma_status_t move_pages(const Call& call, const mma_kv_layout_t* layout, void* const* layers, const int32_t* from, const int32_t* to,
                        const uint32_t* moves, uint32_t most, const mma_kv_compact_t* table, hipStream_t stream) {
  static thread_local MoveArgs k;
  k.from = from;
  k.to = to;
  k.moves = moves;
  k.places = 0;
  k.num_blocks = call.c.num_blocks;
  if (table) {
    k.table = table->block_table;
    k.table_out = table->table_out;
    k.moved = table->moved;
    k.places = static_cast<uint64_t>(table->num_seqs) * table->table_stride;
  }
  k.piece = call.piece;
  k.v_offset = call.piece * call.c.num_blocks;
  k.most = most;
  for (uint32_t first = 0; first < layout->num_layers; first += MoveArgs::kMaxLayers) {
    k.layers = std::min(layout->num_layers - first, MoveArgs::kMaxLayers);
    for (uint32_t l = 0; l < k.layers; ++l) k.layer[l] = reinterpret_cast<uint64_t>(layers[first + l]);
    if (mma_status_t s = launched(launch_moves(k, stream), "KV page move")) return s;
    k.places = 0;
  }
  return MMA_OK;
}

uint64_t fork_workspace(uint32_t num_children) { return 12ull * num_children; }

uint64_t compact_workspace(uint32_t num_blocks) { return 8 + 8ull * num_blocks; }

}  // namespace
}  // namespace mma

using namespace mma;

extern "C" {

mma_status_t mma_rope_table(const mma_rope_t* rope, uint64_t rows, float* out) try {
  if (!rope || (rows && !out)) return fail(MMA_ERR_INVALID_ARG, "NULL argument");
  const uint32_t R = rope->rot_dim;
  if (!R || R % 2 || !(rope->base > 0)) return fail(MMA_ERR_INVALID_ARG, "rot_dim has to be even and base positive");
  if (rope->kind > MMA_ROPE_BANDS) return fail(MMA_ERR_INVALID_ARG, "unknown scaling %u", rope->kind);
  if (rope->kind != MMA_ROPE_NONE && !(rope->factor >= 1)) return fail(MMA_ERR_INVALID_ARG, "factor has to be at least 1");
  const bool ends = rope->kind == MMA_ROPE_RAMP || rope->kind == MMA_ROPE_BANDS;
  if (ends && !(rope->original_len > 0 && rope->low > 0 && rope->high > rope->low))
    return fail(MMA_ERR_INVALID_ARG, "original_len > 0 and 0 < low < high are needed");
  const double two_pi = 2 * M_PI;
  double base = rope->base, amp = 1;
  if (rope->kind == MMA_ROPE_BASE) {
    if (R < 4) return fail(MMA_ERR_INVALID_ARG, "MMA_ROPE_BASE needs rot_dim of 4 or more");
    base *= std::pow(rope->factor, static_cast<double>(R) / (R - 2));
  }
  // The index of the pair that turns n times over original_len.
  const auto index = [&](double n) { return R * std::log(rope->original_len / (n * two_pi)) / (2 * std::log(base)); };
  double first = 0, last = 0;
  if (rope->kind == MMA_ROPE_RAMP) {
    if (base == 1) return fail(MMA_ERR_INVALID_ARG, "MMA_ROPE_RAMP needs a base other than 1");
    first = std::max(std::floor(index(rope->high)), 0.0);
    last = std::min(std::ceil(index(rope->low)), R - 1.0);
    if (last <= first) last = first + 0.001;
    amp = 0.1 * std::log(rope->factor) + 1;
  }
  for (uint32_t i = 0; i < R / 2; ++i) {
    double f = std::pow(base, -2.0 * i / R);
    double keep = 1;  // share of the unscaled frequency
    if (rope->kind == MMA_ROPE_LINEAR) keep = 0;
    if (rope->kind == MMA_ROPE_RAMP) keep = 1 - std::min(std::max((i - first) / (last - first), 0.0), 1.0);
    if (rope->kind == MMA_ROPE_BANDS)
      keep = std::min(std::max((rope->original_len * f / two_pi - rope->low) / (rope->high - rope->low), 0.0), 1.0);
    if (keep < 1) f = keep * f + (1 - keep) * f / rope->factor;
    for (uint64_t p = 0; p < rows; ++p) {
      out[p * R + i] = static_cast<float>(amp * std::cos(p * f));
      out[p * R + R / 2 + i] = static_cast<float>(amp * std::sin(p * f));
    }
  }
  return MMA_OK;
} catch (...) {
  return ops_boundary_error("mma_rope_table");
}

mma_status_t mma_kv_append(const mma_kv_layout_t* layout, void* layer, const mma_kv_seqs_t* seqs,
                           const mma_kv_append_t* a, void* stream) try {
  mma_status_t s;
  Call call;
  if ((s = begin(&call))) return s;
  if (!a) return fail(MMA_ERR_INVALID_ARG, "NULL arguments");
  if ((s = check_layout(layout, &call))) return s;
  if ((s = check_types(a->type, a->cache_type, layout->elem_bytes))) return s;
  if ((s = check_heads(a->q_heads, layout->kv_heads, a->num_tokens))) return s;
  const uint32_t D = layout->head_dim, H = layout->kv_heads, n = a->num_tokens;
  if (a->rope && (!a->rot_dim || a->rot_dim % 2 || a->rot_dim > D || !a->rope_rows))
    return fail(MMA_ERR_INVALID_ARG, "rot_dim %u of %u rows: even, from 2 to head_dim, and a row at least", a->rot_dim,
                a->rope_rows);
  if ((a->q_weight || a->k_weight) && !(a->eps >= 0)) return fail(MMA_ERR_INVALID_ARG, "eps has to be 0 or more");
  if ((s = check_seqs_sizes(seqs, layout->block_tokens))) return s;
  if (!n) return MMA_OK;
  Device dev(call.device);
  if (seqs->num_seqs && seqs->max_tokens) {
    if ((s = check_layer(layer, &call))) return s;
    if ((s = check_seqs(seqs, layout->block_tokens, n, &call))) return s;
  } else {  // tokens of no sequence: their queries are wanted all the same
    call.s.max_tokens = 1;
    call.s.num_tokens = n;
  }
  AppendArgs k{};
  if ((s = rows(&call, "q", a->q, n, a->q_heads, D, false, &k.q))) return s;
  if ((s = rows(&call, "k", a->k, n, H, D, false, &k.k))) return s;
  if ((s = rows(&call, "v", a->v, n, H, D, false, &k.v))) return s;
  if ((s = rows(&call, "q_out", a->q_out, n, a->q_heads, D, true, &k.out))) return s;
  if (a->rope) {
    if ((s = array(&call, "rope", a->rope, extent(a->rope_rows, a->rot_dim, 4), 16))) return s;
    if ((s = array(&call, "positions", a->positions, 4ull * n, 4))) return s;
  }
  if ((s = array(&call, "q_weight", a->q_weight, 2ull * D, 2, true))) return s;
  if ((s = array(&call, "k_weight", a->k_weight, 2ull * D, 2, true))) return s;
  if ((s = array(&call, "k_scale", a->k_scale, 4ull * H, 4, true))) return s;
  if ((s = array(&call, "v_scale", a->v_scale, 4ull * H, 4, true))) return s;
  k.c = call.c;
  k.s = call.s;
  k.positions = a->positions;
  k.rope = a->rope;
  k.q_weight = a->q_weight;
  k.k_weight = a->k_weight;
  k.k_scale = a->cache_type == MMA_TYPE_F8 ? a->k_scale : nullptr;
  k.v_scale = a->cache_type == MMA_TYPE_F8 ? a->v_scale : nullptr;
  k.q_heads = a->q_heads;
  k.rot_dim = a->rope ? a->rot_dim : 0;
  k.rope_rows = a->rope_rows;
  k.interleaved = a->interleaved ? 1 : 0;
  k.wide = rows_wide(k.q) && rows_wide(k.k) && rows_wide(k.v) && rows_wide(k.out) && aligned(a->q_weight, 16) &&
           aligned(a->k_weight, 16);
  k.eps = a->eps;
  return launched(launch_append(k, {a->type, a->cache_type, layout->gpu_layout}, static_cast<hipStream_t>(stream)),
                  "KV append");
} catch (...) {
  return ops_boundary_error("mma_kv_append");
}

mma_status_t mma_kv_attention_shaped_workspace(const mma_kv_layout_t* layout, const mma_kv_seqs_t* seqs,
                                               const mma_kv_attention_t* a, const mma_kv_shape_t* shape, uint64_t* bytes) try {
  return attention_workspace(layout, seqs, a, shape, bytes);
} catch (...) {
  return ops_boundary_error("mma_kv_attention_shaped_workspace");
}

mma_status_t mma_kv_attention_workspace(const mma_kv_layout_t* layout, const mma_kv_seqs_t* seqs,
                                        const mma_kv_attention_t* a, uint64_t* bytes) try {
  return attention_workspace(layout, seqs, a, nullptr, bytes);
} catch (...) {
  return ops_boundary_error("mma_kv_attention_workspace");
}

mma_status_t mma_kv_attention_shaped(const mma_kv_layout_t* layout, const void* layer, const mma_kv_seqs_t* seqs,
                                     const mma_kv_attention_t* a, const mma_kv_shape_t* shape, void* stream) try {
  return attention(layout, layer, seqs, a, shape, stream);
} catch (...) {
  return ops_boundary_error("mma_kv_attention_shaped");
}

mma_status_t mma_kv_attention(const mma_kv_layout_t* layout, const void* layer, const mma_kv_seqs_t* seqs,
                              const mma_kv_attention_t* a, void* stream) try {
  return attention(layout, layer, seqs, a, nullptr, stream);
} catch (...) {
  return ops_boundary_error("mma_kv_attention");
}

mma_status_t mma_kv_commit(const mma_kv_layout_t* layout, void* const* gpu_layers, const mma_kv_seqs_t* seqs,
                           const mma_kv_commit_t* a, void* stream) try {
  mma_status_t s;
  Call call;
  if ((s = begin(&call))) return s;
  if (!a || !gpu_layers) return fail(MMA_ERR_INVALID_ARG, "NULL argument");
  if ((s = check_layout(layout, &call))) return s;
  if ((s = check_seqs_sizes(seqs, layout->block_tokens))) return s;
  if (a->scores && a->scores_stride < seqs->max_len)
    return fail(MMA_ERR_INVALID_ARG, "scores_stride %u is below max_len %u", a->scores_stride, seqs->max_len);
  const uint64_t each = 4ull * seqs->num_seqs;
  if ((s = apart("lens_out", a->lens_out, each, "seqs->lens", seqs->lens, each))) return s;
  if ((s = apart("lens_out", a->lens_out, each, "counts", a->counts, each))) return s;
  if ((s = apart("lens_out", a->lens_out, each, "accepted", a->accepted, extent(seqs->num_seqs, a->accepted_stride, 4)))) return s;
  if (!seqs->num_seqs || (!a->accepted_stride && !a->lens_out)) return MMA_OK;  // lists of no places still give lens_out
  Device dev(call.device);
  if ((s = check_seqs(seqs, layout->block_tokens, INT32_MAX, &call))) return s;
  if ((s = array(&call, "accepted", a->accepted, extent(seqs->num_seqs, a->accepted_stride, 4), 4, !a->accepted_stride))) return s;
  if ((s = array(&call, "counts", a->counts, each, 4))) return s;
  if ((s = array(&call, "lens_out", a->lens_out, each, 4, true))) return s;
  const uint64_t score_bytes = extent(static_cast<uint64_t>(seqs->num_seqs) * layout->kv_heads, a->scores_stride, 4);
  for (uint32_t l = 0; l < layout->num_layers; ++l) {
    if ((s = array(&call, "a layer tensor", gpu_layers[l], call.layer_bytes, 16))) return s;
    if (a->scores && (s = array(&call, "a layer's scores", a->scores[l], score_bytes, 4))) return s;
  }
  static thread_local CommitArgs k;
  k.c = call.c;
  k.s = call.s;
  k.accepted = a->accepted;
  k.counts = a->counts;
  k.v_offset = call.piece * call.c.num_blocks;
  k.accepted_stride = a->accepted_stride;
  k.scores_stride = a->scores_stride;
  for (uint32_t first = 0; first < layout->num_layers; first += CommitArgs::kMaxLayers) {
    k.layers = std::min(layout->num_layers - first, CommitArgs::kMaxLayers);
    k.lens_out = first ? nullptr : a->lens_out;
    for (uint32_t l = 0; l < k.layers; ++l) {
      k.layer[l] = reinterpret_cast<uint64_t>(gpu_layers[first + l]);
      k.scores[l] = a->scores ? reinterpret_cast<uint64_t>(a->scores[first + l]) : 0;
    }
    const OpsKind kind{MMA_TYPE_BF16, layout->elem_bytes == 1 ? MMA_TYPE_F8 : MMA_TYPE_BF16, layout->gpu_layout};
    if ((s = launched(launch_commit(k, kind, static_cast<hipStream_t>(stream)), "KV commit"))) return s;
  }
  return MMA_OK;
} catch (...) {
  return ops_boundary_error("mma_kv_commit");
}

mma_status_t mma_kv_evict_workspace(const mma_kv_layout_t* layout, const mma_kv_seqs_t* seqs, uint64_t* bytes) try {
  if (!bytes) return fail(MMA_ERR_INVALID_ARG, "NULL argument");
  Call call;
  mma_status_t s;
  if ((s = check_layout(layout, &call))) return s;
  if ((s = check_seqs_sizes(seqs, layout->block_tokens))) return s;
  *bytes = evict_workspace(seqs, layout->kv_heads);
  return MMA_OK;
} catch (...) {
  return ops_boundary_error("mma_kv_evict_workspace");
}

mma_status_t mma_kv_evict(const mma_kv_layout_t* layout, void* layer, const mma_kv_seqs_t* seqs,
                          const mma_kv_evict_t* a, void* stream) try {
  mma_status_t s;
  Call call;
  if ((s = begin(&call))) return s;
  if (!a) return fail(MMA_ERR_INVALID_ARG, "NULL arguments");
  if ((s = check_layout(layout, &call))) return s;
  if ((s = check_seqs_sizes(seqs, layout->block_tokens))) return s;
  if (!a->keep || a->keep > static_cast<uint32_t>(INT32_MAX) - 4096 ||
      static_cast<uint64_t>(a->sinks) + a->recent > a->keep)
    return fail(MMA_ERR_INVALID_ARG, "keep %u: at least 1 and sinks + recent, below 2^31 - 4096", a->keep);
  if (a->keep > static_cast<uint64_t>(a->dst_stride) * layout->block_tokens)
    return fail(MMA_ERR_INVALID_ARG, "dst_stride %u blocks do not hold %u entries", a->dst_stride, a->keep);
  if (a->scores_stride < seqs->max_len)
    return fail(MMA_ERR_INVALID_ARG, "scores_stride %u is below max_len %u", a->scores_stride, seqs->max_len);
  const uint64_t each = 4ull * seqs->num_seqs, heads = static_cast<uint64_t>(seqs->num_seqs) * layout->kv_heads;
  const uint64_t score_bytes = extent(heads, a->scores_stride, 4), kept_bytes = extent(heads, a->keep, 4);
  if ((s = apart("lens_out", a->lens_out, each, "seqs->lens", seqs->lens, each))) return s;
  if ((s = apart("scores_out", a->scores_out, kept_bytes, "scores", a->scores, score_bytes))) return s;
  if ((s = apart("entries", a->entries, kept_bytes, "scores", a->scores, score_bytes))) return s;
  if (!seqs->num_seqs) return MMA_OK;
  Device dev(call.device);
  if ((s = check_layer(layer, &call))) return s;
  if ((s = check_seqs(seqs, layout->block_tokens, 0, &call))) return s;
  if ((s = array(&call, "dst_table", a->dst_table, extent(seqs->num_seqs, a->dst_stride, 4), 4))) return s;
  if ((s = array(&call, "scores", a->scores, score_bytes, 4))) return s;
  if ((s = array(&call, "entries", a->entries, kept_bytes, 4))) return s;
  if ((s = array(&call, "scores_out", a->scores_out, kept_bytes, 4, true))) return s;
  if ((s = array(&call, "lens_out", a->lens_out, each, 4, true))) return s;
  const uint64_t need = evict_workspace(seqs, layout->kv_heads);
  if (a->workspace_bytes < need)
    return fail(MMA_ERR_BUFFER_TOO_SMALL, "the workspace has %llu bytes, %llu are needed",
                static_cast<unsigned long long>(a->workspace_bytes), static_cast<unsigned long long>(need));
  if ((s = array(&call, "workspace", a->workspace, need, 8))) return s;
  EvictArgs k{};
  k.chosen = static_cast<uint32_t*>(a->workspace);
  k.c = call.c;
  k.s = call.s;
  k.dst_table = a->dst_table;
  k.scores = a->scores;
  k.entries = a->entries;
  k.scores_out = a->scores_out;
  k.lens_out = a->lens_out;
  k.dst_stride = a->dst_stride;
  k.scores_stride = a->scores_stride;
  k.keep = a->keep;
  k.sinks = a->sinks;
  k.recent = a->recent;
  const OpsKind kind{MMA_TYPE_BF16, layout->elem_bytes == 1 ? MMA_TYPE_F8 : MMA_TYPE_BF16, layout->gpu_layout};
  return launched(launch_evict(k, kind, static_cast<hipStream_t>(stream)), "KV evict");
} catch (...) {
  return ops_boundary_error("mma_kv_evict");
}

mma_status_t mma_beam_select_workspace(const mma_beam_select_t* a, uint64_t* bytes) try {
  if (!bytes) return fail(MMA_ERR_INVALID_ARG, "NULL argument");
  BeamPlan p{};
  if (mma_status_t s = check_beam_sizes(a, &p)) return s;
  *bytes = p.bytes;
  return MMA_OK;
} catch (...) {
  return ops_boundary_error("mma_beam_select_workspace");
}

mma_status_t mma_beam_select(const mma_beam_select_t* a, void* stream) try {
  mma_status_t s;
  Call call;
  BeamPlan p{};
  if ((s = begin(&call))) return s;
  if ((s = check_beam_sizes(a, &p))) return s;
  if (a->done && (a->done_token < 0 || static_cast<uint32_t>(a->done_token) >= a->vocab))
    return fail(MMA_ERR_INVALID_ARG, "done_token %d is not in a vocabulary of %u", a->done_token, a->vocab);
  if (!a->batch) return MMA_OK;
  const uint64_t rows = static_cast<uint64_t>(a->batch) * a->beams, size = a->type == MMA_TYPE_F32 ? 4 : 2;
  const uint64_t kept = 4ull * a->batch * a->keep;
  uint64_t reach;
  if (__builtin_mul_overflow(rows - 1, a->row_stride, &reach) || reach > UINT64_MAX / 8)
    return fail(MMA_ERR_INVALID_ARG, "logits: their extent is beyond 64 bits");
  reach = (reach + a->vocab) * size;
  if ((s = all_apart({{"tokens", a->tokens, kept}, {"parents", a->parents, kept}, {"scores_out", a->scores_out, kept}},
                     {{"logits", a->logits, reach}, {"scores", a->scores, 4 * rows}, {"done", a->done, rows}})))
    return s;
  Device dev(call.device);
  if ((s = array(&call, "logits", a->logits, reach, size))) return s;
  if ((s = array(&call, "scores", a->scores, 4 * rows, 4))) return s;
  if ((s = array(&call, "done", a->done, rows, 1, true))) return s;
  if ((s = array(&call, "tokens", a->tokens, kept, 4))) return s;
  if ((s = array(&call, "parents", a->parents, kept, 4))) return s;
  if ((s = array(&call, "scores_out", a->scores_out, kept, 4))) return s;
  if ((s = workspace(&call, a->workspace, a->workspace_bytes, p.bytes, 8))) return s;
  BeamArgs k{};
  k.logits = static_cast<const uint8_t*>(a->logits);
  k.row_bytes = a->row_stride * size;
  k.scores = a->scores;
  k.done = a->done;
  k.tokens = a->tokens;
  k.parents = a->parents;
  k.scores_out = a->scores_out;
  char* ws = static_cast<char*>(a->workspace);
  k.part_sum = reinterpret_cast<double*>(ws);
  k.lists = reinterpret_cast<uint64_t*>(ws + p.sum_bytes);
  k.rows = p.joined ? k.lists + p.list_bytes / 8 : nullptr;
  k.part_max = reinterpret_cast<float*>(ws + p.sum_bytes + p.list_bytes + p.row_bytes);
  k.batch = a->batch;
  k.beams = a->beams;
  k.vocab = a->vocab;
  k.keep = a->keep;
  k.splits = p.splits;
  k.run = p.run;
  k.done_token = a->done_token;
  return launched(launch_beam(k, a->type, static_cast<hipStream_t>(stream)), "beam selection");
} catch (...) {
  return ops_boundary_error("mma_beam_select");
}

mma_status_t mma_kv_fork_workspace(const mma_kv_fork_t* a, uint64_t* bytes) try {
  if (!a || !bytes) return fail(MMA_ERR_INVALID_ARG, "NULL argument");
  *bytes = fork_workspace(a->num_children);
  return MMA_OK;
} catch (...) {
  return ops_boundary_error("mma_kv_fork_workspace");
}

mma_status_t mma_kv_fork(const mma_kv_layout_t* layout, void* const* gpu_layers, const mma_kv_seqs_t* seqs,
                         const mma_kv_fork_t* a, void* stream) try {
  mma_status_t s;
  Call call;
  if ((s = begin(&call))) return s;
  if (!a || !gpu_layers) return fail(MMA_ERR_INVALID_ARG, "NULL argument");
  if ((s = check_layout(layout, &call))) return s;
  if ((s = check_seqs_sizes(seqs, layout->block_tokens))) return s;
  if (a->num_children > kMaxGrid) return fail(MMA_ERR_INVALID_ARG, "%u children, at most %u", a->num_children, kMaxGrid);
  if (static_cast<uint64_t>(a->out_stride) * layout->block_tokens < seqs->max_len)
    return fail(MMA_ERR_INVALID_ARG, "out_stride %u blocks do not hold %u entries", a->out_stride, seqs->max_len);
  const uint64_t places = static_cast<uint64_t>(a->num_children) * a->out_stride;
  if (places > 1u << 30) return fail(MMA_ERR_INVALID_ARG, "more than 2^30 places in table_out");
  const uint64_t counts = 4ull * layout->gpu_num_blocks, each = 4ull * a->num_children, lens = 4ull * seqs->num_seqs;
  const uint64_t table = extent(seqs->num_seqs, seqs->table_stride, 4);
  if ((s = all_apart({{"refs_out", a->refs_out, counts}, {"table_out", a->table_out, 4 * places}, {"lens_out", a->lens_out, each},
                      {"free_out", a->free_out, 4}},
                     {{"block_table", seqs->block_table, table}, {"lens", seqs->lens, lens}, {"parents", a->parents, each},
                      {"grow", a->grow, each}})))
    return s;
  for (const Part& o : {Part{"table_out", a->table_out, 4 * places}, Part{"lens_out", a->lens_out, each}, Part{"free_out", a->free_out, 4}})
    if ((s = apart(o.name, o.p, o.bytes, "refs", a->refs, counts))) return s;
  if (a->refs_out != a->refs && (s = apart("refs_out", a->refs_out, counts, "refs", a->refs, counts))) return s;
  Device dev(call.device);
  if (seqs->num_seqs) {
    if ((s = check_seqs(seqs, layout->block_tokens, 0, &call))) return s;
  }
  if (a->num_children) {
    if ((s = array(&call, "parents", a->parents, each, 4))) return s;
    if ((s = array(&call, "grow", a->grow, each, 4, true))) return s;
    if ((s = array(&call, "table_out", a->table_out, 4 * places, 4))) return s;
    if ((s = array(&call, "lens_out", a->lens_out, each, 4))) return s;
  }
  if ((s = array(&call, "refs", a->refs, counts, 4))) return s;
  if ((s = array(&call, "refs_out", a->refs_out, counts, 4))) return s;
  if ((s = array(&call, "free_out", a->free_out, 4, 4))) return s;
  if ((s = workspace(&call, a->workspace, a->workspace_bytes, fork_workspace(a->num_children), 4))) return s;
  for (uint32_t l = 0; l < layout->num_layers; ++l)
    if ((s = array(&call, "a layer tensor", gpu_layers[l], call.layer_bytes, 16))) return s;
  ForkArgs k{};
  k.table = seqs->block_table;
  k.lens = seqs->lens;
  k.parents = a->parents;
  k.grow = a->grow;
  k.refs = a->refs;
  k.refs_out = a->refs_out;
  k.table_out = a->table_out;
  k.lens_out = a->lens_out;
  k.free_out = a->free_out;
  k.from = static_cast<int32_t*>(a->workspace);
  k.to = k.from + a->num_children;
  k.wants = reinterpret_cast<uint32_t*>(k.to + a->num_children);
  k.num_seqs = seqs->num_seqs;
  k.table_stride = seqs->table_stride;
  k.num_children = a->num_children;
  k.out_stride = a->out_stride;
  k.num_blocks = layout->gpu_num_blocks;
  k.tokens = layout->block_tokens;
  k.max_len = seqs->max_len;
  const hipStream_t on = static_cast<hipStream_t>(stream);
  if ((s = launched(launch_fork(k, on), "KV fork"))) return s;
  return move_pages(call, layout, gpu_layers, k.from, k.to, nullptr, a->num_children, nullptr, on);
} catch (...) {
  return ops_boundary_error("mma_kv_fork");
}

mma_status_t mma_kv_compact_workspace(const mma_kv_layout_t* layout, uint64_t* bytes) try {
  if (!bytes) return fail(MMA_ERR_INVALID_ARG, "NULL argument");
  Call call;
  if (mma_status_t s = check_layout(layout, &call)) return s;
  *bytes = compact_workspace(layout->gpu_num_blocks);
  return MMA_OK;
} catch (...) {
  return ops_boundary_error("mma_kv_compact_workspace");
}

mma_status_t mma_kv_compact(const mma_kv_layout_t* layout, void* const* gpu_layers, const mma_kv_compact_t* a, void* stream) try {
  mma_status_t s;
  Call call;
  if ((s = begin(&call))) return s;
  if (!a || !gpu_layers) return fail(MMA_ERR_INVALID_ARG, "NULL argument");
  if ((s = check_layout(layout, &call))) return s;
  const uint64_t places = static_cast<uint64_t>(a->num_seqs) * a->table_stride, counts = 4ull * layout->gpu_num_blocks;
  if (places > 1u << 30) return fail(MMA_ERR_INVALID_ARG, "more than 2^30 places in the table");
  if ((s = all_apart({{"table_out", a->table_out, 4 * places}, {"refs_out", a->refs_out, counts}, {"moved", a->moved, counts},
                      {"held_out", a->held_out, 4}}, {})))
    return s;
  for (const Part& o : {Part{"refs_out", a->refs_out, counts}, Part{"moved", a->moved, counts}, Part{"held_out", a->held_out, 4}})
    if ((s = apart(o.name, o.p, o.bytes, "block_table", a->block_table, 4 * places))) return s;
  for (const Part& o : {Part{"table_out", a->table_out, 4 * places}, Part{"moved", a->moved, counts}, Part{"held_out", a->held_out, 4}})
    if ((s = apart(o.name, o.p, o.bytes, "refs", a->refs, counts))) return s;
  if (a->refs_out != a->refs && (s = apart("refs_out", a->refs_out, counts, "refs", a->refs, counts))) return s;
  if (a->table_out != a->block_table && (s = apart("table_out", a->table_out, 4 * places, "block_table", a->block_table, 4 * places))) return s;
  Device dev(call.device);
  if (places) {
    if ((s = array(&call, "block_table", a->block_table, 4 * places, 4))) return s;
    if ((s = array(&call, "table_out", a->table_out, 4 * places, 4))) return s;
  }
  if ((s = array(&call, "refs", a->refs, counts, 4))) return s;
  if ((s = array(&call, "refs_out", a->refs_out, counts, 4))) return s;
  if ((s = array(&call, "moved", a->moved, counts, 4))) return s;
  if ((s = array(&call, "held_out", a->held_out, 4, 4))) return s;
  if ((s = workspace(&call, a->workspace, a->workspace_bytes, compact_workspace(layout->gpu_num_blocks), 8))) return s;
  for (uint32_t l = 0; l < layout->num_layers; ++l)
    if ((s = array(&call, "a layer tensor", gpu_layers[l], call.layer_bytes, 16))) return s;
  CompactArgs k{};
  k.refs = a->refs;
  k.refs_out = a->refs_out;
  k.moved = a->moved;
  k.held_out = a->held_out;
  k.moves = static_cast<uint32_t*>(a->workspace);
  k.from = reinterpret_cast<int32_t*>(k.moves + 2);
  k.to = k.from + layout->gpu_num_blocks;
  k.num_blocks = layout->gpu_num_blocks;
  const hipStream_t on = static_cast<hipStream_t>(stream);
  if ((s = launched(launch_compact(k, on), "KV compaction"))) return s;
  return move_pages(call, layout, gpu_layers, k.from, k.to, k.moves, layout->gpu_num_blocks / 2, a, on);
} catch (...) {
  return ops_boundary_error("mma_kv_compact");
}

}  // extern "C"
