// C ABI of the attention operators (kv_append, kv_attend, kv_attention_score): argument checks, the split of
// the work, launches.
#include <cmath>

#include "kv_attend.cuh"

using namespace kvt;

namespace {

inline cudaStream_t S(kv_stream_t s) { return static_cast<cudaStream_t>(s); }
inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Elements of a query or key head and of a value head; a negative status if the operators do not take them.
int32_t dims(const PoolView& v, int32_t q, uint32_t* dk, uint32_t* dv) {
  const kv_model_desc& m = v.desc->part[q].model;
  if (m.dtype_bits != 16 || m.n_q_heads <= 0) return KV_ERR_UNSUPPORTED_VARIANT;
  const bool mla = v.variant[q] == KV_MLA;
  *dk = (uint32_t)(mla ? m.d_latent + m.d_rope : m.head_dim);
  *dv = (uint32_t)(mla ? m.d_latent : m.head_dim);
  if (v.geom[q].heads > 4096u || (uint32_t)m.n_q_heads % v.geom[q].heads != 0) return KV_ERR_UNSUPPORTED_VARIANT;
  return KV_OK;
}

TableView table_view(const PoolView& v, int32_t q, int32_t layer, const uint32_t* d_table, uint64_t n_rows) {
  const PartGeom& g = v.geom[q];
  TableView t;
  t.table = d_table;
  t.n_rows = n_rows;
  t.loc = v.desc->d_loc;
  t.n_tags = v.desc->n_tags < KV_NONE ? v.desc->n_tags : KV_NONE;
  t.slab = g.slab;
  t.base = g.base;
  t.n = g.n;
  t.heads = g.heads;
  t.layers = (uint32_t)v.desc->part[q].model.n_layers;
  t.layer = (uint32_t)layer;
  t.n_chunks = g.n_chunks;
  t.chunk_bytes = g.chunk_bytes;
  t.block_tokens = (uint32_t)v.desc->part[q].block_tokens;
  t.by_tokens = Divisor(t.block_tokens);
  t.by_heads = Divisor(t.heads);
  t.status = v.status;
  return t;
}

// How a call's work is split: tokens of a chunk and chunks, for prefixes and suffixes.
constexpr uint32_t kSms = 148;
// Rows from which on a segment goes to the tensor cores' 128-row tiles.
constexpr uint32_t kTileRows = 33;
struct Split {
  bool tiles[2], stream[2];
  uint32_t chunk_tokens[2], chunks[2], per_chunk[2], n_parts, grain_tokens, grains[2];
  uint64_t lse_at, total_at, grain_at[2], bytes;
};

// How segments of `tiles` tiles (at most) are cut when `ctas` row tiles are split alike: `per` tiles a chunk.
struct Cut {
  uint64_t ctas, tiles, most_per, per;
  uint64_t chunks() const { return ctas ? (tiles + per - 1) / per : 0; }
};
// The cuts of prefixes and suffixes that one launch runs through, `slots` CTAs at a time, prefixes first: those for which the
// longer of the longest CTA and an even share of all of them is shortest.  A CTA costs `extra` tiles beside its own; runs
// are taken to be as long as their bounds; a part more than one in all costs another launch.
void cut(Cut& p, Cut& s, uint64_t slots, uint64_t extra, bool alone) {
  uint64_t best = ~0ull, best_p = 1, best_s = 1;
  auto first = [](const Cut& c) { return c.ctas ? (c.tiles + c.most_per - 1) / c.most_per : 1; };
  auto last = [slots](const Cut& c) { return c.ctas ? 2 * slots / c.ctas + 1 : 0; };
  // (few of the many cuts of few row tiles: a step of an eighth, of a third where there are two to choose)
  const uint64_t step = p.ctas && s.ctas ? 3 : 8;
  for (uint64_t np = first(p); np <= first(p) + last(p); np += np < step ? 1 : np / step) {
    p.per = p.ctas ? (p.tiles + np - 1) / np : 1;
    for (uint64_t ns = first(s); ns <= first(s) + last(s); ns += ns < step ? 1 : ns / step) {
      s.per = s.ctas ? (s.tiles + ns - 1) / ns : 1;
      const uint64_t n_p = p.ctas * p.chunks(), n_s = s.ctas * s.chunks(), longest = (n_p && p.per > s.per) || !n_s ? p.per : s.per;
      uint64_t cost;
      if (!n_p || !n_s) {
        cost = (n_p + n_s + slots - 1) / slots * (longest + extra);
      } else {
        const uint64_t all = n_p * (p.per + extra) + s.ctas * s.tiles + n_s * extra;
        cost = all / slots + (n_p + n_s > slots ? ((p.per < s.per ? p.per : s.per) + extra) / 2 : 0);
        if (cost < longest + extra) cost = longest + extra;
      }
      if (alone && n_p + n_s > p.ctas + s.ctas) cost += 2 * extra;
      if (cost < best) {
        best = cost;
        best_p = p.per;
        best_s = s.per;
      }
      if (s.per == 1) break;
    }
    if (p.per == 1) break;
  }
  p.per = best_p;
  s.per = best_s;
}

bool split(const PoolView& v, int32_t q, uint32_t dk, uint32_t dv, uint32_t n_seqs, uint32_t n_groups, uint32_t max_suffix,
           uint32_t max_prefix, uint32_t max_members, bool weights, Split* out) {
  const uint32_t bt = (uint32_t)v.desc->part[q].block_tokens, heads = v.geom[q].heads;
  const uint32_t q_heads = (uint32_t)v.desc->part[q].model.n_q_heads, group = q_heads / heads;
  const bool mla = v.variant[q] == KV_MLA;
  const bool shared = n_groups && max_prefix && max_members;
  // (per token of the longest run nothing may leave 31 bits)
  if (max_suffix >= 0x40000000u || max_prefix >= 0x40000000u || n_seqs >= 0x1000000u || n_groups >= 0x1000000u) return false;
  if (max_members > n_seqs) max_members = n_seqs;
  if ((uint64_t)max_members * group >= 0x10000000u || (uint64_t)n_seqs * q_heads >= 0x40000000u) return false;
  out->tiles[0] = out->tiles[1] = out->stream[0] = out->stream[1] = false;
  out->chunk_tokens[0] = out->chunk_tokens[1] = 64;
  out->chunks[0] = out->chunks[1] = 0;
  out->per_chunk[0] = out->per_chunk[1] = 1;
  const uint64_t prefix_rows = (uint64_t)max_members * group;
  const uint64_t slab_rows = v.geom[q].n * v.geom[q].n_chunks * bt;
  const bool streams = stream_takes(dk, dv, mla, bt, slab_rows);
  const bool fits = tiles_take(dk, dv, mla, bt, slab_rows);
  uint64_t limit = (uint64_t)kMaxChunkBlocks * bt / 64 * 64;   // most tokens of a chunk
  if (limit < 64) limit = 64;
  if (limit > kMaxChunkTokens) limit = kMaxChunkTokens;
  // prefix and suffix, by the kernels that take them: tiles, streams, the rest
  Cut tiles[2] = {}, rest[2] = {};
  uint64_t rest_slots = 2 * kSms;
  for (int k = 0; k < 2; ++k) {
    if (k == 0 && !shared) continue;
    const uint64_t rows = k == 0 ? prefix_rows : group, segs = (uint64_t)(k == 0 ? n_groups : n_seqs) * heads;
    const uint32_t most = k == 0 ? max_prefix : max_suffix ? max_suffix : 1;
    out->tiles[k] = fits && rows >= kTileRows;
    out->stream[k] = !out->tiles[k] && streams && rows <= 32;
    if (out->tiles[k]) {
      const uint64_t tile = mla ? 128 : 256;
      out->per_chunk[k] = !mla && rows <= 128 ? 2 : 1;
      tiles[k] = Cut{(rows + tile - 1) / tile * segs * (mla ? 2 : 1), ((uint64_t)most + 63) / 64, limit / 64, 1};
    } else if (out->stream[k]) {
      // a warp's chunk, 8 to 32 units: chunks for five warps in six where all runs are as long as their bound.  (0.6 as many: MQA of ragged
      // runs 36 -> 42 us, of one long run among short ones 29 -> 33, of equal runs 42 -> 41; MHA with one long run 55 -> 43, else even.)
      const uint64_t units = ((uint64_t)most + kStreamUnit - 1) / kStreamUnit;
      uint64_t per = (rows + 15) / 16 * segs * units * 12 / 10 / (kSms * stream_warps(dk));
      per = per < 8 ? 8 : per > 32 ? 32 : per;
      per = (units + (units + per - 1) / per - 1) / ((units + per - 1) / per);    // the same number of chunks, evenly
      out->chunk_tokens[k] = (uint32_t)(per * kStreamUnit);
      out->chunks[k] = (uint32_t)((units + per - 1) / per);
    } else {
      const uint64_t tile = mla ? 64 : rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
      rest[k] = Cut{(rows + tile - 1) / tile * segs, ((uint64_t)most + 63) / 64, limit / 64, 1};
      if (mla) rest_slots = kSms;
    }
  }
  for (Cut* c : {tiles, rest}) {
    if (!c[0].ctas && !c[1].ctas) continue;
    cut(c[0], c[1], c == tiles ? kSms : rest_slots, c == tiles ? 8 : 4, !shared);
    for (int k = 0; k < 2; ++k) {
      if (!c[k].ctas) continue;
      out->chunk_tokens[k] = (uint32_t)(c[k].per * 64);
      out->chunks[k] = (uint32_t)c[k].chunks();
    }
  }
  // what the launches will be: nothing is enqueued of a call that one of them could not take
  typedef unsigned __int128 Count;
  Count by_tiles = 0, by_streams = 0, by_rest = 0, weight_ctas = 0;
  for (int k = shared ? 0 : 1; k < 2; ++k) {
    const uint64_t segs = (uint64_t)(k == 0 ? n_groups : n_seqs) * heads, kind_rows = k == 0 ? prefix_rows : group;
    if (out->tiles[k]) by_tiles += (Count)tiles[k].ctas * out->chunks[k];
    else if (out->stream[k]) by_streams += (Count)((kind_rows + 15) / 16) * segs * out->chunks[k];
    else by_rest += (Count)rest[k].ctas * out->chunks[k];
    if (!weights) continue;
    const Count items = (Count)segs * (((uint64_t)(k == 0 ? max_prefix : max_suffix) + bt - 1) / bt) * ((kind_rows + kWeightRows - 1) / kWeightRows);
    if (items > kMaxWeightItems) return false;
    weight_ctas += (items << weight_shift((uint32_t)kind_rows)) / kFinishThreads + 1;
  }
  if (by_tiles > kMaxGrid || by_streams > kMaxGrid || by_rest > kMaxGrid || weight_ctas > kMaxGrid) return false;
  out->n_parts = out->chunks[0] * out->per_chunk[0] + out->chunks[1] * out->per_chunk[1];
  out->grain_tokens = bt % 16 == 0 ? 16 : 1;
  const unsigned __int128 rows = (unsigned __int128)n_seqs * q_heads;
  unsigned __int128 at = 0;
  auto take = [&at](unsigned __int128 bytes) { const uint64_t o = (uint64_t)at; at = (at + bytes + 255) / 256 * 256; return o; };
  if (out->n_parts > 1) take(rows * out->n_parts * dv * 4);
  out->lse_at = take(rows * out->n_parts * 4);
  out->total_at = take(weights ? rows * 4 : 0);
  for (int k = 0; k < 2; ++k) {
    const uint32_t most = k == 0 ? (shared ? max_prefix : 0) : max_suffix;
    out->grains[k] = (uint32_t)(((uint64_t)most + out->grain_tokens - 1) / out->grain_tokens);
    out->grain_at[k] = take(weights ? (unsigned __int128)(k == 0 ? n_groups : n_seqs) * heads * out->grains[k] *
                                          (k == 0 ? prefix_rows : group) * 4
                                    : 0);
  }
  if (at > ((unsigned __int128)1 << 46)) return false;
  out->bytes = (uint64_t)at;
  return true;
}

bool attend_dims(const PoolView& v, int32_t q, uint32_t dk, uint32_t dv) {
  if (v.variant[q] == KV_MLA) return dv <= 512 && dk <= kMaxRowDim && dk % 8 == 0 && dv % 8 == 0;
  return dk <= 256 && dk % 8 == 0;
}

}  // namespace

extern "C" {

uint64_t kv_attend_scratch_bytes(kv_pool* p, int32_t q, uint32_t n_seqs, uint32_t n_groups, uint32_t max_suffix,
                                 uint32_t max_prefix, uint32_t max_members, int32_t weights) {
  if (!p) return 0;
  const PoolView v = pool_view(p);
  uint32_t dk, dv;
  if (q < 0 || q >= v.n_parts || dims(v, q, &dk, &dv) != KV_OK || !attend_dims(v, q, dk, dv)) return 0;
  Split s;
  return split(v, q, dk, dv, n_seqs, n_groups, max_suffix, max_prefix, max_members, weights != 0, &s) ? (s.bytes ? s.bytes : 256) : 0;
}

int32_t kv_attend(kv_pool* p, const kv_attend_desc* d, kv_stream_t stream) {
  if (!p || !d) return KV_ERR_INVALID_ARG;
  const PoolView v = pool_view(p);
  const int32_t q = d->partition;
  if (q < 0 || q >= v.n_parts || d->layer < 0 || d->layer >= v.desc->part[q].model.n_layers) return KV_ERR_INVALID_ARG;
  if (d->dtype != KV_DTYPE_BF16 && d->dtype != KV_DTYPE_F16) return KV_ERR_INVALID_ARG;
  uint32_t dk, dv;
  const int32_t rc = dims(v, q, &dk, &dv);
  if (rc != KV_OK) return rc;
  if (!attend_dims(v, q, dk, dv)) return KV_ERR_UNSUPPORTED_VARIANT;
  const float scale2 = d->scale * 1.44269504088896340736f;   // exponentials are of base 2
  if (!std::isfinite(scale2)) return KV_ERR_INVALID_ARG;
  if (d->n_seqs == 0) return KV_OK;
  if (!d->d_q || !d->d_out || !aligned(d->d_q, 2) || !aligned(d->d_out, 2) || !d->d_suffix || !aligned(d->d_suffix, 4)) return KV_ERR_INVALID_ARG;
  if (d->n_groups && (!d->d_prefix || !d->d_group || !aligned(d->d_prefix, 4) || !aligned(d->d_group, 4))) return KV_ERR_INVALID_ARG;
  if (d->n_rows && (!d->d_table || !aligned(d->d_table, 4))) return KV_ERR_INVALID_ARG;
  if (d->n_rows >= 0x100000000ull || !aligned(d->d_lse, 4) || !aligned(d->d_weight, 8)) return KV_ERR_INVALID_ARG;
  Split sp;
  if (!split(v, q, dk, dv, d->n_seqs, d->n_groups, d->max_suffix, d->max_prefix, d->max_members, d->d_weight != nullptr, &sp)) return KV_ERR_INVALID_ARG;
  if (!d->d_scratch || !aligned(d->d_scratch, 16) || d->scratch_bytes < sp.bytes) return KV_ERR_INVALID_ARG;
  const int32_t rs = pool_settle(p, stream);
  if (rs != KV_OK) return rs;
  AttendArgs a{};
  a.tv = table_view(v, q, d->layer, d->d_table, d->n_rows);
  a.q = d->d_q;
  a.out = d->d_out;
  a.lse = d->d_lse;
  a.q_seq = d->q_stride[0];
  a.q_head = d->q_stride[1];
  a.out_seq = d->out_stride[0];
  a.out_head = d->out_stride[1];
  a.scale2 = scale2;
  a.n_seqs = d->n_seqs;
  a.n_groups = sp.chunks[0] ? d->n_groups : 0u;
  a.q_heads = (uint32_t)v.desc->part[q].model.n_q_heads;
  a.group = a.q_heads / a.tv.heads;
  a.by_group = Divisor(a.group);
  a.dk = dk;
  a.dv = dv;
  a.suffix = d->d_suffix;
  a.prefix = d->d_prefix;
  a.group_start = d->d_group;
  a.max_suffix = d->max_suffix;
  a.max_prefix = d->max_prefix;
  a.max_members = d->max_members < d->n_seqs ? d->max_members : d->n_seqs;
  uint8_t* const scratch = static_cast<uint8_t*>(d->d_scratch);
  for (int k = 0; k < 2; ++k) {
    a.tiles[k] = sp.tiles[k];
    a.stream[k] = sp.stream[k];
    a.chunk_tokens[k] = sp.chunk_tokens[k];
    a.chunks[k] = sp.chunks[k];
    a.per_chunk[k] = sp.per_chunk[k];
    a.grains[k] = sp.grains[k];
    a.grain[k] = reinterpret_cast<float*>(scratch + sp.grain_at[k]);
  }
  a.n_parts = sp.n_parts;
  a.direct = sp.n_parts == 1;
  a.part_o = reinterpret_cast<float*>(scratch);
  a.part_lse = reinterpret_cast<float*>(scratch + sp.lse_at);
  a.total = reinterpret_cast<float*>(scratch + sp.total_at);
  a.grain_tokens = sp.grain_tokens;
  a.weight = reinterpret_cast<unsigned long long*>(d->d_weight);
  return pool_cuda_error(p, launch_attend(a, d->dtype, v.variant[q] == KV_MLA, S(stream)));
}

int32_t kv_append(kv_pool* p, const kv_append_desc* d, kv_stream_t stream) {
  if (!p || !d) return KV_ERR_INVALID_ARG;
  const PoolView v = pool_view(p);
  const int32_t q = d->partition;
  if (q < 0 || q >= v.n_parts || d->layer < 0 || d->layer >= v.desc->part[q].model.n_layers) return KV_ERR_INVALID_ARG;
  if (d->dtype != KV_DTYPE_BF16 && d->dtype != KV_DTYPE_F16) return KV_ERR_INVALID_ARG;
  uint32_t dk, dv;
  const int32_t rc = dims(v, q, &dk, &dv);
  if (rc != KV_OK) return rc;
  const bool mla = v.variant[q] == KV_MLA;
  const kv_rope_desc& r = d->rope;
  if (r.rot_dim < 0 || r.rot_dim > 256 || r.rot_dim % 2 != 0 || r.rot_first < 0 ||
      (int64_t)r.rot_first + r.rot_dim > (int64_t)dk)
    return KV_ERR_INVALID_ARG;
  if (r.rot_dim > 0) {
    if (r.n_axes < 1 || r.n_axes > 4) return KV_ERR_INVALID_ARG;
    for (int i = 0; i < r.rot_dim / 2; ++i)
      if (r.axis[i] >= r.n_axes) return KV_ERR_INVALID_ARG;
  }
  if (d->n_tokens == 0) return KV_OK;
  if (r.rot_dim > 0 && (!r.d_inv_freq || !aligned(r.d_inv_freq, 4) || !d->d_pos || !aligned(d->d_pos, 4))) return KV_ERR_INVALID_ARG;
  if (d->n_tokens > 0x7fffffffull || d->n_rows >= 0x100000000ull) return KV_ERR_INVALID_ARG;
  if (!d->d_k || !aligned(d->d_k, 2) || (mla ? d->d_v != nullptr : !d->d_v) || !aligned(d->d_v, 2)) return KV_ERR_INVALID_ARG;
  if ((d->d_q != nullptr) != (d->d_q_out != nullptr) || !aligned(d->d_q, 2) || !aligned(d->d_q_out, 2)) return KV_ERR_INVALID_ARG;
  // (a token's elements are counted in 31 bits)
  const uint64_t heads = v.geom[q].heads, q_heads = d->d_q ? (uint64_t)v.desc->part[q].model.n_q_heads : 0u;
  if ((heads + q_heads) * dk + (mla ? 0u : heads * dv) >= 0x80000000ull) return KV_ERR_UNSUPPORTED_VARIANT;
  if (!d->d_slot || !aligned(d->d_slot, 8) || (d->n_rows && (!d->d_table || !aligned(d->d_table, 4)))) return KV_ERR_INVALID_ARG;
  const int32_t rs = pool_settle(p, stream);
  if (rs != KV_OK) return rs;
  AppendArgs a{};
  a.tv = table_view(v, q, d->layer, d->d_table, d->n_rows);
  a.k = d->d_k;
  a.v = d->d_v;
  a.q = d->d_q;
  a.q_out = d->d_q_out;
  a.k_tok = d->k_stride[0]; a.k_head = d->k_stride[1];
  a.v_tok = d->v_stride[0]; a.v_head = d->v_stride[1];
  a.q_tok = d->q_stride[0]; a.q_head = d->q_stride[1];
  a.o_tok = d->q_out_stride[0]; a.o_head = d->q_out_stride[1];
  a.slot = d->d_slot;
  a.pos = d->d_pos;
  a.inv_freq = r.d_inv_freq;
  a.n = d->n_tokens;
  a.q_heads = d->d_q ? (uint32_t)v.desc->part[q].model.n_q_heads : 0u;
  a.dk = dk;
  a.dv = mla ? 0u : dv;
  a.rot_first = (uint32_t)r.rot_first;
  a.rot_dim = (uint32_t)r.rot_dim;
  a.interleaved = r.interleaved != 0;
  a.n_axes = (uint32_t)r.n_axes;
  for (int i = 0; i < 128; ++i) a.axis[i] = r.axis[i];
  // 16-byte vectors where every one of them is aligned; blocks always are, if their rows are
  auto strides = [](const int64_t (&s)[2]) { return s[0] % 8 == 0 && s[1] % 8 == 0; };
  const bool wide = dk % 8 == 0 && a.dv % 8 == 0 && a.rot_first % 8 == 0 && a.rot_dim % (a.interleaved ? 8 : 16) == 0 &&
                    aligned(d->d_k, 16) && strides(d->k_stride) && (mla || (aligned(d->d_v, 16) && strides(d->v_stride))) &&
                    (!d->d_q || (aligned(d->d_q, 16) && strides(d->q_stride) && aligned(d->d_q_out, 16) && strides(d->q_out_stride)));
  return pool_cuda_error(p, launch_append(a, d->dtype, wide, S(stream)));
}

int32_t kv_attention_score(kv_pool* p, uint32_t epoch, float decay, uint32_t protect, uint64_t* d_weight, float* d_acc,
                           kv_stream_t stream) {
  if (!p || !(decay >= 0.0f && decay <= 1.0f) || protect >= 0x80000000u) return KV_ERR_INVALID_ARG;
  const PoolView v = pool_view(p);
  if (v.desc->n_tags && (!d_weight || !d_acc)) return KV_ERR_INVALID_ARG;
  if (!aligned(d_weight, 16) || !aligned(d_acc, 16)) return KV_ERR_INVALID_ARG;
  const int32_t rs = pool_settle(p, stream);
  if (rs != KV_OK) return rs;
  return pool_cuda_error(p, launch_attention_score(v.st, v.desc->d_loc, v.desc->n_tags, epoch, decay, protect,
                                                   reinterpret_cast<unsigned long long*>(d_weight), d_acc, S(stream)));
}

}  // extern "C"
