// What the translation units of the attention operators share: geometry, arguments, and the
// device helpers that read a sequence's segments and block handles.
#pragma once
#include "kvtier_internal.cuh"

namespace kvt {

// A pool as the attention operators see it (kvtier_host.cu fills it in).
struct PoolView {
  const kv_pool_desc* desc;
  const PartGeom* geom;
  int n_parts;
  EntryState st;
  uint32_t* status;
  int32_t variant[4];
};
PoolView pool_view(kv_pool* p);
// Enqueues what deferred packing holds back and lets the stream wait for promotions in flight.
int32_t pool_settle(kv_pool* p, kv_stream_t stream);
int32_t pool_cuda_error(kv_pool* p, cudaError_t e);

// The blocks of one partition and layer through a table of handles.
struct TableView {
  const uint32_t* table;   // [n_rows][layers][heads]
  uint64_t n_rows;
  const uint32_t* loc;
  uint64_t n_tags;
  uint8_t* slab;
  uint64_t base, n;        // the partition's global ids
  uint32_t heads, layers, layer;
  uint32_t n_chunks;       // 2: K and V, 1: MLA
  uint32_t chunk_bytes;
  uint32_t block_tokens;
  Divisor by_tokens, by_heads;
  uint32_t* status;

  __device__ __forceinline__ void flag(uint32_t bit) const { atomicOr(status, bit); }

  // Index of the chunk that holds the K (or MLA) rows of table row `row`, head h, in units of
  // chunk_bytes from the slab; ~0u if the block is not in HBM.  The V chunk lies `heads` chunks behind.
  __device__ __forceinline__ uint32_t chunk(uint64_t row, uint32_t h) const {
    const uint32_t handle = table[(row * layers + layer) * heads + h];
    if (handle >= n_tags) return ~0u;
    const uint32_t id = loc[handle];
    if (id & KV_LOC_HOST) return ~0u;          // in the host tier, or (KV_NONE) nowhere
    if (id < base || id - base >= n) {
      flag(KV_DEV_BAD_INDEX);
      return ~0u;
    }
    const uint32_t e = (uint32_t)(id - base);
    const uint32_t b = by_heads(e);
    return b * (n_chunks - 1u) * heads + e;    // b * n_chunks * heads + e % heads
  }
};

// A run of table rows: `tokens` tokens from the first token of row `row` on.
struct Segment {
  uint32_t row, tokens;
};

enum : int { kKindPrefix = 0, kKindSuffix = 1 };

struct AttendArgs {
  TableView tv;
  const void* q;
  void* out;
  float* lse;
  int64_t q_seq, q_head, out_seq, out_head;   // strides in elements
  float scale2;                               // scale * log2(e)
  uint32_t n_seqs, n_groups, q_heads, group;  // group: query heads of a KV head
  Divisor by_group;
  uint32_t dk, dv;                            // elements of a key row and of a value row
  const uint32_t* suffix;                     // [n_seqs][2]
  const uint32_t* prefix;                     // [n_groups][2]
  const uint32_t* group_start;                // [n_groups + 1]
  uint32_t max_suffix, max_prefix, max_members;
  uint32_t tiles[2];                          // by kv_attend_tiles.cu ...
  uint32_t stream[2];                         // ... or by kv_attend_stream.cu
  // The tokens of a segment are worked on in chunks of chunk_tokens[kind], whose results are parts:
  // part c of (sequence s, query head j) is at (s * q_heads + j) * n_parts + c, prefix chunks first; a chunk has
  // per_chunk parts.
  uint32_t chunk_tokens[2], chunks[2], per_chunk[2], n_parts;
  float* part_o;                              // [..][dv], normalised
  float* part_lse;                            // log2 of the part's sum of exponentials
  float* total;                               // the same of each row, where weights are asked for
  uint32_t direct;                            // one part: written to out and lse straight away
  // Attention weight of each `grain` tokens (log2 of the sum of exponentials), for every row:
  // prefix [group][head][grain][max_members * group], suffix [seq][head][grain][group].
  float* grain[2];
  uint32_t grain_tokens, grains[2];           // grains of a segment of the longest length
  unsigned long long* weight;                 // [n_tags], or nullptr

  __device__ __forceinline__ Segment checked(const uint32_t* seg, uint32_t i, uint32_t most, bool tell) const {
    Segment s{seg[2ull * i], seg[2ull * i + 1]};
    const uint64_t rows = s.tokens ? (uint64_t)tv.by_tokens(s.tokens - 1u) + 1u : 0u;
    if (s.tokens > most || s.row + rows > tv.n_rows) {
      if (tell) tv.flag(KV_DEV_BAD_INDEX);
      s.tokens = 0;
    }
    return s;
  }
  // Sequences [lo, hi) of group g; none if the group's bounds are no such range.
  __device__ __forceinline__ void members(uint32_t g, uint32_t& lo, uint32_t& hi, bool tell) const {
    lo = group_start[g];
    hi = group_start[g + 1u];
    if (lo > hi || hi > n_seqs || hi - lo > max_members) {
      if (tell) tv.flag(KV_DEV_BAD_INDEX);
      hi = lo = 0;
    }
  }
  // The group of sequence s, or ~0u.
  __device__ __forceinline__ uint32_t group_of(uint32_t s) const {
    uint32_t lo = 0, hi = n_groups;   // the last group that starts at or before s
    while (lo < hi) {
      const uint32_t mid = (lo + hi) / 2u;
      if (group_start[mid] <= s) lo = mid + 1u; else hi = mid;
    }
    if (!lo) return ~0u;
    uint32_t a, b;
    members(lo - 1u, a, b, false);
    return s >= a && s < b ? lo - 1u : ~0u;
  }
};

constexpr uint32_t kMaxRowDim = 576;          // widest row of keys (MLA)
constexpr uint32_t kStreamUnit = 16, kStreamTokens = 1024;   // a warp's of kv_attend_stream.cu
constexpr int kFinishThreads = 256;           // of a CTA that joins parts or adds weights up
constexpr uint32_t kWeightRows = 256;         // rows of a block that one item of the weights takes
constexpr uint64_t kMaxGrid = 0x7fffffffull, kMaxWeightItems = 0xf0000000ull;   // of a launch: a call beyond them is refused (split)
constexpr uint32_t kMaxChunkTokens = 4096, kMaxChunkBlocks = 256;   // most a CTA takes of a segment

// log2 of the threads that add up a block's weight of so many rows
inline uint32_t weight_shift(uint32_t rows) {
  uint32_t shift = 0;
  while (shift < 5u && (1u << shift) < rows) ++shift;
  return shift;
}

// kv_attend.cu
cudaError_t launch_attend(const AttendArgs& a, int dtype, bool mla, cudaStream_t s);

// kv_attend_tiles.cu: whether it takes a geometry, and its part of launch_attend
bool tiles_take(uint32_t dk, uint32_t dv, bool mla, uint32_t block_tokens, uint64_t slab_rows);
cudaError_t launch_attend_tiles(const AttendArgs& a, int dtype, bool mla, bool prefix, bool suffix, cudaStream_t s);

// kv_attend_stream.cu: the same for up to 32 rows (two row tiles of 16, each a stream of its own).  behind_tiles: launch_attend_tiles went ahead in this call, and the two
// may run side by side.
bool stream_takes(uint32_t dk, uint32_t dv, bool mla, uint32_t block_tokens, uint64_t slab_rows);
uint32_t stream_warps(uint32_t dk);   // of an SM
cudaError_t launch_attend_stream(const AttendArgs& a, int dtype, bool prefix, bool suffix, bool behind_tiles,
                                 cudaStream_t s);

// kv_append.cu
struct AppendArgs {
  TableView tv;
  const void *k, *v, *q;
  void* q_out;
  int64_t k_tok, k_head, v_tok, v_head, q_tok, q_head, o_tok, o_head;   // strides in elements
  const int64_t* slot;         // [n]
  const int32_t* pos;          // [n_axes][n]
  const float* inv_freq;       // [rot_dim / 2]
  uint64_t n;
  uint32_t q_heads, dk, dv;
  uint32_t rot_first, rot_dim, interleaved, n_axes;
  uint8_t axis[128];
};
cudaError_t launch_append(const AppendArgs& a, int dtype, bool wide, cudaStream_t s);

// kv_attention.cu
cudaError_t launch_attention_score(const EntryState& st, const uint32_t* loc, uint64_t n_tags, uint32_t epoch, float decay, uint32_t protect,
                                   unsigned long long* weight, float* acc, cudaStream_t s);

}  // namespace kvt
