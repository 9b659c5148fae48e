// The operators on the paged KV cache: what their host side (mma_ops.cpp) hands to
// their kernels, and what it needs of the runtime (mma_runtime.cpp).
#ifndef MMA_OPS_H_
#define MMA_OPS_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/mma.h"

namespace mma {

// ------------------------------------------------------------ of the runtime
mma_status_t ops_ready(int* device);  // after mma_init, no sticky failure
// Checks that [p, p + bytes) lies in one allocation of the device; *base and *size get that allocation (or the
// range itself), so that a caller need not ask again for what it knows to be inside.
mma_status_t ops_device_range(const void* p, uint64_t bytes, uint64_t* base, uint64_t* size);
mma_status_t ops_boundary_error(const char* func);  // in a catch (...) block

// ------------------------------------------------------------ kernel arguments
// A cache layer. Entry j of a head: block j / tokens by multiplication (div_mul,
// div_shift: exact below 2^31), then byte offsets within the block. A 16-byte chunk
// of an entry's key or (rows layouts) value is contiguous in every layout.
struct CacheArgs {
  uint8_t* k;  // K of block 0; V follows K of every block
  uint8_t* v;
  uint64_t block_bytes;
  uint32_t num_blocks;
  uint32_t tokens;
  uint32_t div_mul, div_shift;
  uint32_t heads, dim;
  uint32_t k_head, k_token, k_chunk;  // bytes
  uint32_t v_head, v_token, v_chunk;  // v_chunk: of 16 bytes of a row, or x-packed of one value of the head
};

struct SeqArgs {
  const int32_t* table;
  const int32_t* lens;
  const int32_t* q_start;
  uint32_t num_seqs, table_stride, max_tokens, max_len, num_tokens;
};

struct RowArgs {
  uint8_t* data;
  uint64_t token, head;  // strides in elements
};

struct AppendArgs {
  CacheArgs c;
  SeqArgs s;
  RowArgs q, k, v, out;
  const int32_t* positions;
  const float* rope;
  const void* q_weight;
  const void* k_weight;
  const float* k_scale;
  const float* v_scale;
  uint32_t q_heads, rot_dim, rope_rows, interleaved;
  uint32_t wide;  // every row starts at 16 bytes
  float eps;
};

struct AttnArgs {
  CacheArgs c;
  SeqArgs s;
  RowArgs q, out;
  RowArgs score_q;  // the queries as the weights kernel reads them: q, or its copy where `out` takes q's place
  const uint64_t* tree;
  float* lse;
  const float* scores_in;
  float* scores_out;
  const float* k_scale;
  const float* v_scale;
  float* part;      // of each row and split: the sum of p V
  float* part_ml;   // and the maximum (in powers of 2) and sum of p; NULL where neither is read
  float* lse2;      // of each row, base 2: for the scores kernel, else NULL
  float* logits;    // [sequence][KV head][logit_rows][logit_stride], base 2, or NULL
  uint32_t logit_rows, logit_stride;
  uint32_t q_heads, group, tree_words, scores_stride;
  uint32_t score_len;          // entries of a workgroup of the scores kernel: a multiple of 32, at most 1024
  uint32_t splits, split_len;  // entries of a split: a multiple of the tile
  uint32_t wide_q, wide_out, wide_score_q;  // rows start at 16 bytes
  float scale, decay;
};

struct CommitArgs {
  CacheArgs c;  // k, v unused
  SeqArgs s;
  const int32_t* accepted;
  const int32_t* counts;
  int32_t* lens_out;
  uint64_t v_offset;  // of V of block 0 from the layer's start
  uint32_t accepted_stride, scores_stride, layers;
  static constexpr uint32_t kMaxLayers = 192;  // of one launch: the arguments stay below 4 KiB
  uint64_t layer[kMaxLayers];
  uint64_t scores[kMaxLayers];
};

struct EvictArgs {
  CacheArgs c;
  SeqArgs s;
  const int32_t* dst_table;
  const float* scores;
  int32_t* entries;
  float* scores_out;
  int32_t* lens_out;
  uint32_t* chosen;  // workspace: 2 (1 + max_len / 1024, rounded up) words a row
  uint32_t dst_stride, scores_stride, keep, sinks, recent;
};

// What a kernel is compiled for.
struct OpsKind {
  uint32_t type, cache_type, layout;
};

// Split of an attention call (mma_ops.cpp: attention_plan).
struct AttnPlan {
  bool stream;              // attention_stream_kernel, else attention_rows_kernel
  uint32_t rows;            // most rows (token, head of a group) of one sequence and KV head
  uint32_t tiles_per_wave;  // of 16 rows
  uint32_t row_groups;      // workgroups that the rows take
  uint32_t splits, split_len;
  uint32_t dim_pad;
  bool logits;              // scores from logits that the main kernel keeps
  bool keys_stay;           // else: attention_scores_kernel keeps a wave's keys, or the rows
  uint32_t logit_stride;
  uint64_t part_bytes, ml_bytes, lse_bytes, q_bytes, logit_bytes, bytes;
};

// Whether attention_stream_kernel is there for two tiles of rows, with their keys and values in registers: not with heads
// above 128, and of 65 to 128 not where V is turned in registers.
constexpr bool stream_two_tiles(uint32_t dim_pad, bool f8, bool xpacked) {
  return dim_pad == 64 || (dim_pad == 128 && (f8 || xpacked));
}

hipError_t launch_append(const AppendArgs& a, const OpsKind& k, hipStream_t stream);
hipError_t launch_attention(const AttnArgs& a, const AttnPlan& p, const OpsKind& k, hipStream_t stream);
hipError_t launch_commit(const CommitArgs& a, const OpsKind& k, hipStream_t stream);
hipError_t launch_evict(const EvictArgs& a, const OpsKind& k, hipStream_t stream);

// ------------------------------------------------------------ device helpers
#ifdef __HIPCC__
constexpr int kOpsWave = 64;

// A launch and its own status: an error that an earlier call left in the runtime is neither taken for this launch's nor
// taken away.
template <class T>
struct AsIs {
  typedef T type;
};
template <class... P>
hipError_t launch(void (*kernel)(P...), dim3 grid, uint32_t block, hipStream_t stream, const typename AsIs<P>::type&... args) {
  void* params[] = {const_cast<P*>(&args)...};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(block), params, 0, stream);
}

__device__ __forceinline__ uint32_t block_of(const CacheArgs& c, uint32_t entry) {
  return static_cast<uint32_t>((static_cast<uint64_t>(entry) * c.div_mul) >> c.div_shift);
}

// Block of entry `entry` of a sequence's table row, or -1. The caller keeps entry / tokens inside the row.
__device__ __forceinline__ int32_t block_at(const CacheArgs& c, const int32_t* row, uint32_t entry, uint32_t* token) {
  const uint32_t b = block_of(c, entry);
  *token = entry - b * c.tokens;
  const int32_t id = row[b];
  return static_cast<uint32_t>(id) < c.num_blocks ? id : -1;
}

struct SeqSpan {
  uint32_t first;  // row of its first token
  uint32_t count;  // tokens
  uint32_t before; // entries before them
  uint32_t total;  // entries with them, within max_len
};

__device__ __forceinline__ SeqSpan span_of(const SeqArgs& s, uint32_t seq) {
  SeqSpan r;
  const int64_t n = s.num_tokens;
  int64_t a, b;
  if (s.q_start) {
    a = s.q_start[seq];
    b = s.q_start[seq + 1];
  } else {
    a = static_cast<int64_t>(seq) * s.max_tokens;
    b = a + s.max_tokens;
  }
  a = a < 0 ? 0 : a > n ? n : a;
  b = b < a ? a : b > n ? n : b;
  const int64_t t = b - a;
  r.first = static_cast<uint32_t>(a);
  r.count = static_cast<uint32_t>(t > s.max_tokens ? s.max_tokens : t);
  const int32_t len = s.lens[seq];
  r.before = len < 0 ? 0u : static_cast<uint32_t>(len);
  if (r.before > s.max_len) r.before = s.max_len;
  const uint32_t room = s.max_len - r.before;
  r.total = r.before + (r.count < room ? r.count : room);
  return r;
}
#endif  // __HIPCC__

}  // namespace mma

#endif  // MMA_OPS_H_
