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
  static constexpr bool kShaped = false, kCapped = false;
};

// Attention whose scores have a shape (mma_kv_shape_t).
struct ShapedArgs : AttnArgs {
  const float* slopes;    // [q_heads] or NULL
  const int32_t* prefix;  // [num_seqs] or NULL
  uint32_t max_prefix;
  uint32_t window;        // entries up to a token's own, at most 2^31 - 1; 0: all
  uint32_t wg_rows;       // rows of a workgroup
  float* score_part;      // weights of parts of the rows, [score_parts][num_seqs][heads][max_len], where there are several
  uint32_t score_parts;
  static constexpr bool kShaped = true;
};

// And a cap.
struct CappedArgs : ShapedArgs {
  float cap2;          // base 2
  float cap_terms[5];  // of small scores (capped)
  static constexpr bool kCapped = true;
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

// Beam search's selection. Parts of rows: [row][split], lists of `keep` keys each (mma_beam.hip).
constexpr uint32_t kBeamChunk = 4096;   // logits that a workgroup takes at once
constexpr uint32_t kBeamMerge = 16384;  // keys that a merge takes
constexpr uint32_t kBeamMost = 64;      // beams of a request
constexpr uint32_t kBeamKeep = 128;

struct BeamArgs {
  const uint8_t* logits;
  uint64_t row_bytes;
  const float* scores;
  const uint8_t* done;
  int32_t* tokens;
  int32_t* parents;
  float* scores_out;
  double* part_sum;
  uint64_t* lists;
  uint64_t* rows;  // each row's parts joined, or NULL where a request's parts are few enough
  float* part_max;
  uint32_t batch, beams, vocab, keep;
  uint32_t splits, run;  // parts of a row, and how many times kBeamChunk logits each is
  int32_t done_token;
};

struct ForkArgs {
  const int32_t* table;
  const int32_t* lens;
  const int32_t* parents;
  const int32_t* grow;
  const int32_t* refs;
  int32_t* refs_out;
  int32_t* table_out;
  int32_t* lens_out;
  int32_t* free_out;
  int32_t* from;    // of each child: the block that is copied for it, or -1
  int32_t* to;      // and where, or -1
  uint32_t* wants;  // new blocks of the children before it
  uint32_t num_seqs, table_stride, num_children, out_stride, num_blocks, tokens, max_len;
};

struct CompactArgs {
  const int32_t* refs;
  int32_t* refs_out;
  int32_t* moved;
  int32_t* held_out;
  int32_t* from;  // the moves
  int32_t* to;
  uint32_t* moves;  // how many
  uint32_t num_blocks;
};

struct MoveArgs {
  const int32_t* from;
  const int32_t* to;
  const uint32_t* moves;  // how many, or NULL: `most`
  uint64_t piece;         // bytes of a block's K or V
  uint64_t v_offset;      // of V of block 0 from the layer's start
  const int32_t* table;   // of a compaction: its places, and where blocks have moved
  int32_t* table_out;
  const int32_t* moved;
  uint64_t places;
  uint32_t num_blocks;
  uint32_t most, layers;
  static constexpr uint32_t kMaxLayers = 192;
  uint64_t layer[kMaxLayers];
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
  uint32_t wg_rows;         // rows of a workgroup
  uint32_t row_groups;      // workgroups that the rows take
  uint32_t splits, split_len;
  uint32_t dim_pad;
  bool logits;              // scores from logits that the main kernel keeps
  bool keys_stay;           // else: attention_scores_kernel keeps a wave's keys, or the rows
  uint32_t logit_stride;
  uint32_t score_parts;     // with a shape: parts of the rows whose weights are added up at the end
  uint64_t part_bytes, ml_bytes, lse_bytes, q_bytes, logit_bytes, score_bytes, bytes;
};

// Whether attention_stream_kernel is there for two tiles of rows, with their keys and values in registers: not with heads
// above 128, and of 65 to 128 not where V is turned in registers.
constexpr bool stream_two_tiles(uint32_t dim_pad, bool f8, bool xpacked) {
  return dim_pad == 64 || (dim_pad == 128 && (f8 || xpacked));
}

hipError_t launch_append(const AppendArgs& a, const OpsKind& k, hipStream_t stream);
hipError_t launch_attention(const AttnArgs& a, const AttnPlan& p, const OpsKind& k, hipStream_t stream);
hipError_t launch_attention_shaped(const ShapedArgs& a, const AttnPlan& p, const OpsKind& k, hipStream_t stream);
hipError_t launch_attention_capped(const CappedArgs& a, const AttnPlan& p, const OpsKind& k, hipStream_t stream);
hipError_t launch_commit(const CommitArgs& a, const OpsKind& k, hipStream_t stream);
hipError_t launch_beam(const BeamArgs& a, uint32_t type, hipStream_t stream);
hipError_t launch_fork(const ForkArgs& a, hipStream_t stream);
hipError_t launch_compact(const CompactArgs& a, hipStream_t stream);
hipError_t launch_moves(const MoveArgs& a, hipStream_t stream);
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
