// Bounds of kv_attend whose work does not fit its launches, without a GPU: they are refused before anything is enqueued and have no scratch,
// and what is taken fits.  The runtime and the other kernels are the stand-ins of enqueued_order.cu.
#define main order_main
#include "enqueued_order.cu"
#undef main

#include "kv_attend.cuh"

static bool g_tiles = true, g_streams = true;
static int g_attend = 0;
static kvt::AttendArgs g_last;

namespace kvt {
cudaError_t launch_attend(const AttendArgs& a, int, bool, cudaStream_t) { ++g_attend; g_last = a; return cudaSuccess; }
cudaError_t launch_append(const AppendArgs&, int, bool, cudaStream_t) { return cudaSuccess; }
cudaError_t launch_attention_score(const EntryState&, const uint32_t*, uint64_t, uint32_t, float, uint32_t, unsigned long long*, float*, cudaStream_t) { return cudaSuccess; }
bool tiles_take(uint32_t, uint32_t, bool, uint32_t, uint64_t) { return g_tiles; }
bool stream_takes(uint32_t, uint32_t, bool mla, uint32_t, uint64_t) { return g_streams && !mla; }
uint32_t stream_warps(uint32_t) { return 12; }
}  // namespace kvt

static std::vector<std::vector<uint64_t>> g_arrays;
static void* memory(uint64_t bytes) {
  g_arrays.emplace_back(bytes / 8 + 4);
  return (void*)(((uintptr_t)g_arrays.back().data() + 15) & ~15ull);
}

static kv_pool* make(const kv_model_desc& m, int block_tokens) {
  kv_pool_desc d{};
  d.n_partitions = 1;
  const uint64_t heads = m.variant == KV_MLA || m.variant == KV_MQA ? 1 : m.variant == KV_MHA ? m.n_q_heads : m.n_kv_heads, n = 2 * 10 * heads;
  d.part[0].model = m;
  d.part[0].block_tokens = block_tokens;
  d.part[0].blocks_per_layer = 10;
  d.part[0].d_slab = (void*)kSlab;
  d.part[0].h_ring = (void*)kPinned;
  d.part[0].ring_slots = 4;
  d.n_tags = 64;
  d.d_ema = (float*)memory(n * 4); d.d_decay = (float*)memory(n * 4); d.d_touch = (uint32_t*)memory(n * 4);
  d.d_last_epoch = (uint32_t*)memory(n * 4); d.d_pair = (uint8_t*)memory(n); d.d_state = (uint8_t*)memory(n);
  d.d_tag = (uint32_t*)memory(n * 4); d.d_score = (float*)memory(n * 4); d.d_hits = (uint64_t*)memory(128);
  d.d_misses = (uint64_t*)memory(128); d.d_P = (float*)memory(64); d.d_loc = (uint32_t*)memory(d.n_tags * 4);
  d.alpha0 = d.beta0 = 1.0f;
  d.staging_bytes = 1 << 20;
  for (int b = 0; b < 4; ++b) d.d_staging[b] = (void*)(kStage + ((uint64_t)b << 32));
  d.max_promote = 16;
  uint64_t dev = 0, host = 0;
  if (kv_workspace_bytes(&d, &dev, &host) != KV_OK) return nullptr;
  d.d_workspace = memory(dev); d.workspace_bytes = dev;
  d.h_workspace = memory(host); d.h_workspace_bytes = host;
  g_state.assign(n, KV_STATE_FREE);
  kv_pool* p = nullptr;
  return kv_pool_create(&d, (void*)1, &p) == KV_OK ? p : nullptr;
}

struct Bounds { uint32_t seqs, groups, suffix, prefix, members; int weights; };
static void* g_mem;
static int32_t call(kv_pool* p, const Bounds& b, uint64_t scratch, float scale = 0.125f) {
  kv_attend_desc a{};
  a.dtype = KV_DTYPE_BF16;
  a.scale = scale;
  a.n_seqs = b.seqs;
  a.n_groups = b.groups;
  a.max_suffix = b.suffix;
  a.max_prefix = b.prefix;
  a.max_members = b.members;
  a.d_q = a.d_out = g_mem;
  a.d_table = a.d_suffix = a.d_prefix = a.d_group = (const uint32_t*)g_mem;
  a.n_rows = 20;
  a.d_weight = b.weights ? (uint64_t*)g_mem : nullptr;
  a.d_scratch = g_mem;
  a.scratch_bytes = scratch;
  return kv_attend(p, &a, (void*)1);
}
static uint64_t scratch(kv_pool* p, const Bounds& b) {
  return kv_attend_scratch_bytes(p, 0, b.seqs, b.groups, b.suffix, b.prefix, b.members, b.weights);
}
static int g_failed = 0;
static void expect(bool ok, const char* what) {
  if (!ok) { std::printf("%s\n", what); g_failed = 1; }
}
static void refused(kv_pool* p, const Bounds& b, const char* what) {
  const int before = g_attend;
  expect(scratch(p, b) == 0 && call(p, b, ~0ull) == KV_ERR_INVALID_ARG && g_attend == before, what);
}

// what the launches make of g_last (threads of a weight's item: up to 32)
static bool fits(const Bounds& b, bool mla) {
  typedef unsigned __int128 N;
  const kvt::AttendArgs& a = g_last;
  N tiles = 0, streams = 0, rest = 0, weights = 0;
  for (int k = a.chunks[0] ? 0 : 1; k < 2; ++k) {
    const N rows = k ? a.group : (N)a.max_members * a.group, segs = (N)(k ? a.n_seqs : a.n_groups) * a.tv.heads;
    if (a.tiles[k]) tiles += (mla ? (rows + 127) / 128 * 2 : (rows + 255) / 256) * segs * a.chunks[k];
    else if (a.stream[k]) streams += (rows + 15) / 16 * segs * a.chunks[k];
    else rest += (rows + 63) / 64 * segs * a.chunks[k];
    const N items = segs * (((N)(k ? a.max_suffix : a.max_prefix) + a.tv.block_tokens - 1) / a.tv.block_tokens) * ((rows + 255) / 256);
    if (b.weights && items >= ((N)1 << 32) - 256) return false;
    weights += items * (rows < 32 ? 1 : 32) / 256;
  }
  const N most = 0x7fffffff;
  return tiles <= most && streams <= most && rest <= most && (!b.weights || weights <= most);
}

int main() {
  g_mem = memory(1 << 16);
  kv_pool* const mha = make(kv_model_desc{KV_MHA, 2, 32, 32, 64, 0, 0, 16}, 16);
  kv_pool* const mqa = make(kv_model_desc{KV_MQA, 2, 33, 1, 64, 0, 0, 16}, 16);
  kv_pool* const mla = make(kv_model_desc{KV_MLA, 2, 128, 128, 128, 512, 64, 16}, 64);
  if (!mha || !mqa || !mla) return fail("pool");
  // 2,000 sequences of 2^20 tokens: attention fits, the weights of 4.2 billion blocks do not
  const Bounds many{2000, 0, 1u << 20, 0, 0, 0};
  expect(scratch(mha, many) > 0 && call(mha, many, ~0ull) == KV_OK && g_attend == 1, "long sequences");
  refused(mha, {2000, 0, 1u << 20, 0, 0, 1}, "weights of too many blocks");
  refused(mha, {1u << 20, 0, 1u << 20, 0, 0, 0}, "streams of too many chunks");
  refused(mha, {1, 1u << 23, 16, 1u << 20, 1, 0}, "prefixes of too many groups");
  refused(mqa, {1u << 15, 0, 1u << 28, 0, 0, 0}, "tiles of too many chunks");
  g_tiles = g_streams = false;
  refused(mha, {1, 1u << 23, 16, 1u << 20, 1, 0}, "the same, by rows");
  refused(mla, {1, 1u << 23, 16, 1u << 28, 1, 0}, "the same, latent rows");
  // a scale that is finite, but not by 1 / log 2
  const Bounds one{1, 0, 16, 0, 0, 0};
  expect(call(mha, one, ~0ull, 2e38f) == KV_OK && call(mha, one, ~0ull, -2e38f) == KV_OK, "a large scale");
  const int before_scale = g_attend;
  expect(call(mha, one, ~0ull, 3e38f) == KV_ERR_INVALID_ARG && call(mha, one, ~0ull, -3e38f) == KV_ERR_INVALID_ARG && g_attend == before_scale, "too large a scale");
  // tokens of 2^31 elements and more: queries of 2^22 latent heads
  kv_pool* const broad = make(kv_model_desc{KV_MLA, 2, 1 << 22, 1 << 22, 128, 512, 64, 16}, 64);
  if (!broad) return fail("pool of many heads");
  kv_append_desc t{};
  t.dtype = KV_DTYPE_BF16;
  t.n_tokens = 3;
  t.d_k = t.d_q = t.d_q_out = g_mem;
  t.d_table = (const uint32_t*)g_mem;
  t.n_rows = 20;
  t.d_slot = (const int64_t*)g_mem;
  expect(kv_append(broad, &t, (void*)1) == KV_ERR_UNSUPPORTED_VARIANT, "tokens of 2^31 elements");
  t.d_q = t.d_q_out = nullptr;
  expect(kv_append(broad, &t, (void*)1) == KV_OK, "their keys alone");
  t.d_q = t.d_q_out = g_mem;
  expect(kv_append(mla, &t, (void*)1) == KV_OK, "tokens of ordinary heads");
  kv_pool_destroy(broad);
  // whatever is taken fits
  std::mt19937_64 rng(5);
  int took = 0, not_taken = 0;
  for (int i = 0; i < 8000; ++i) {
    auto up_to = [&](int bits) { return (uint32_t)(rng() >> (64 - 1 - rng() % bits)); };
    g_tiles = rng() % 2;
    g_streams = rng() % 2;
    kv_pool* const p = rng() % 3 == 0 ? mla : rng() % 2 ? mqa : mha;
    const Bounds b{1 + up_to(24) % ((1u << 24) - 1), up_to(24) % (1u << 24), up_to(30) % (1u << 30), up_to(30) % (1u << 30), up_to(20), (int)(rng() % 2)};
    const uint64_t bytes = scratch(p, b);
    const int before = g_attend;
    const int32_t rc = call(p, b, bytes ? bytes : ~0ull);
    expect(rc == (bytes ? KV_OK : KV_ERR_INVALID_ARG) && g_attend == before + (bytes ? 1 : 0), "scratch and call disagree");
    if (bytes) expect(fits(b, p == mla), "a call that does not fit its launches was taken");
    (bytes ? took : not_taken) += 1;
  }
  expect(took > 500 && not_taken > 500, "both kinds of bounds");
  kv_pool_destroy(mha);
  kv_pool_destroy(mqa);
  kv_pool_destroy(mla);
  return g_failed;
}
