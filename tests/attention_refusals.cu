// Which calls of kv_append, kv_attend and kv_attention_score the library's host side refuses, and what a call that it takes
// would launch, without a GPU: the runtime and the other kernels are the stand-ins of enqueued_order.cu, the
// operators' launches note what they are given.  Prints a line for each failure; exit status 1 if there is one.
#define main order_main
#include "enqueued_order.cu"
#undef main

#include <cmath>
#include <functional>

#include "kv_attend.cuh"

namespace kvt {
int g_attend, g_append, g_score;
AttendArgs g_last;
cudaError_t launch_attend(const AttendArgs& a, int, bool, cudaStream_t) { ++g_attend; g_last = a; return cudaSuccess; }
cudaError_t launch_append(const AppendArgs&, int, bool, cudaStream_t) { ++g_append; return cudaSuccess; }
cudaError_t launch_attention_score(const EntryState&, const uint32_t*, uint64_t, uint32_t, float, uint32_t, unsigned long long*, float*, cudaStream_t) {
  ++g_score;
  return cudaSuccess;
}
bool tiles_take(uint32_t, uint32_t, bool, uint32_t block_tokens, uint64_t) { return block_tokens % 16 == 0; }
bool stream_takes(uint32_t dk, uint32_t, bool mla, uint32_t, uint64_t) { return !mla && (dk == 64 || dk == 128); }
uint32_t stream_warps(uint32_t) { return 12; }
}  // namespace kvt

static int g_failed = 0;
static void expect(bool ok, const char* what) {
  if (!ok) {
    std::printf("%s\n", what);
    g_failed = 1;
  }
}

static std::vector<std::vector<uint64_t>> g_arrays;
static void* memory(uint64_t bytes) {
  g_arrays.emplace_back(bytes / 8 + 4);
  return (void*)(((uintptr_t)g_arrays.back().data() + 15) & ~15ull);
}

static kv_pool* make(const kv_model_desc& m, int block_tokens) {
  static kv_pool_desc d;
  d = kv_pool_desc{};
  d.n_partitions = 1;
  const uint64_t heads = m.variant == KV_MLA ? 1 : m.variant == KV_MHA ? m.n_q_heads : m.n_kv_heads, n = 2 * 10 * heads;
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

int main() {
  using kvt::g_append;
  using kvt::g_attend;
  using kvt::g_score;
  const kv_stream_t s = (void*)1;
  void* const mem = memory(1 << 16);
  kv_pool* const p = make(kv_model_desc{KV_GQA, 2, 8, 2, 64, 0, 0, 16}, 16);
  if (!p) return fail("pool");

  // ---- kv_attend ----
  kv_attend_desc a{};
  a.dtype = KV_DTYPE_BF16;
  a.layer = 1;
  a.scale = 0.125f;
  a.n_seqs = 3;
  a.n_groups = 1;
  a.max_suffix = 500;
  a.max_prefix = 2000;
  a.max_members = 3;
  a.d_q = a.d_out = mem;
  a.d_lse = (float*)mem;
  a.d_table = a.d_suffix = a.d_prefix = a.d_group = (const uint32_t*)mem;
  a.n_rows = 20;
  a.d_scratch = mem;
  a.scratch_bytes = kv_attend_scratch_bytes(p, 0, 3, 1, 500, 2000, 3, 0);
  expect(a.scratch_bytes > 0, "scratch bytes");
  expect(kv_attend(p, &a, s) == KV_OK && g_attend == 1, "a good kv_attend");
  expect(kvt::g_last.n_groups == 1 && kvt::g_last.group == 4 && !kvt::g_last.direct && kvt::g_last.n_parts == kvt::g_last.chunks[0] * kvt::g_last.per_chunk[0] +
             kvt::g_last.chunks[1] * kvt::g_last.per_chunk[1], "its parts");
  for (int k = 0; k < 2; ++k) {
    const uint32_t most = k ? 500 : 2000, c = kvt::g_last.chunk_tokens[k];
    expect(c > 0 && c % 16 == 0 && (uint64_t)c * kvt::g_last.chunks[k] >= most && (uint64_t)c * (kvt::g_last.chunks[k] - 1) < most, "chunks cover a run");
  }
  auto refused = [&](const char* what, int32_t want, const std::function<void(kv_attend_desc&)>& change) {
    kv_attend_desc b = a;
    change(b);
    const int before = g_attend;
    expect(kv_attend(p, &b, s) == want && g_attend == before, what);
  };
  const int32_t bad = KV_ERR_INVALID_ARG;
  expect(kv_attend(nullptr, &a, s) == bad && kv_attend(p, nullptr, s) == bad, "no pool, no description");
  refused("partition", bad, [](kv_attend_desc& b) { b.partition = 1; });
  refused("partition below", bad, [](kv_attend_desc& b) { b.partition = -1; });
  refused("layer", bad, [](kv_attend_desc& b) { b.layer = 2; });
  refused("layer below", bad, [](kv_attend_desc& b) { b.layer = -1; });
  refused("type", bad, [](kv_attend_desc& b) { b.dtype = 2; });
  refused("scale", bad, [](kv_attend_desc& b) { b.scale = NAN; });
  refused("infinite scale", bad, [](kv_attend_desc& b) { b.scale = INFINITY; });
  refused("q", bad, [](kv_attend_desc& b) { b.d_q = nullptr; });
  refused("out", bad, [](kv_attend_desc& b) { b.d_out = nullptr; });
  refused("odd q", bad, [](kv_attend_desc& b) { b.d_q = (const char*)b.d_q + 1; });
  refused("suffix", bad, [](kv_attend_desc& b) { b.d_suffix = nullptr; });
  refused("prefix", bad, [](kv_attend_desc& b) { b.d_prefix = nullptr; });
  refused("groups", bad, [](kv_attend_desc& b) { b.d_group = nullptr; });
  refused("table", bad, [](kv_attend_desc& b) { b.d_table = nullptr; });
  refused("rows", bad, [](kv_attend_desc& b) { b.n_rows = 1ull << 32; });
  refused("scratch", bad, [](kv_attend_desc& b) { b.d_scratch = nullptr; });
  refused("unaligned scratch", bad, [](kv_attend_desc& b) { b.d_scratch = (char*)b.d_scratch + 8; });
  refused("little scratch", bad, [](kv_attend_desc& b) { b.scratch_bytes -= 1; });
  refused("long suffix", bad, [](kv_attend_desc& b) { b.max_suffix = 1u << 30; });
  refused("long prefix", bad, [](kv_attend_desc& b) { b.max_prefix = 1u << 30; });
  refused("many sequences", bad, [](kv_attend_desc& b) { b.n_seqs = 1u << 24; });
  refused("unaligned weights", bad, [](kv_attend_desc& b) { b.d_weight = (uint64_t*)((char*)b.d_scratch + 4); });
  refused("no sequences", KV_OK, [](kv_attend_desc& b) { b.n_seqs = 0; b.d_q = nullptr; });
  expect(kv_attend_scratch_bytes(nullptr, 0, 1, 0, 1, 0, 0, 0) == 0 && kv_attend_scratch_bytes(p, 1, 1, 0, 1, 0, 0, 0) == 0 &&
             kv_attend_scratch_bytes(p, 0, 1u << 24, 0, 1, 0, 0, 0) == 0, "scratch of refused bounds");
  // every bound has a scratch that the call takes, and chunks that cover it
  for (uint32_t seqs : {1u, 7u, 300u})
    for (uint32_t most : {0u, 1u, 15u, 16u, 17u, 500u, 4096u, 100000u, 3000000u})
      for (uint32_t prefix : {0u, 1u, 70000u})
        for (int weights = 0; weights < 2; ++weights) {
          kv_attend_desc b = a;
          b.n_seqs = seqs;
          b.max_suffix = most;
          b.max_prefix = prefix;
          b.max_members = seqs;
          b.d_weight = weights ? (uint64_t*)mem : nullptr;
          b.scratch_bytes = kv_attend_scratch_bytes(p, 0, seqs, 1, most, prefix, seqs, weights);
          const bool took = b.scratch_bytes && kv_attend(p, &b, s) == KV_OK;
          expect(took, "a bound");
          if (!took) continue;
          const kvt::AttendArgs& l = kvt::g_last;
          for (int k = 0; k < 2; ++k) {
            const uint64_t n = k ? most : prefix;
            expect((uint64_t)l.chunk_tokens[k] * l.chunks[k] >= n && l.chunk_tokens[k] <= (l.stream[k] ? kvt::kStreamTokens : kvt::kMaxChunkTokens), "a bound's chunks");
          }
          expect(l.chunks[1] >= 1 && l.n_parts >= 1 && (l.direct == (l.n_parts == 1)) && !(l.direct && l.per_chunk[1] == 2), "a bound's parts");
          const uint64_t rows = (uint64_t)seqs * 8, floats = l.direct ? 0 : rows * l.n_parts * 64;
          expect((uint64_t)((char*)l.part_lse - (char*)l.part_o) >= floats * 4 &&
                     (uint64_t)((char*)l.part_lse - (char*)b.d_scratch) + rows * l.n_parts * 4 <= b.scratch_bytes, "a bound's scratch");
        }

  // ---- kv_append ----
  kv_append_desc d{};
  d.dtype = KV_DTYPE_F16;
  d.n_tokens = 5;
  d.d_k = d.d_v = d.d_q = d.d_q_out = mem;
  d.d_table = (const uint32_t*)mem;
  d.n_rows = 20;
  d.d_slot = (const int64_t*)mem;
  d.d_pos = (const int32_t*)mem;
  d.rope.rot_dim = 64;
  d.rope.n_axes = 3;
  d.rope.d_inv_freq = (const float*)mem;
  expect(kv_append(p, &d, s) == KV_OK && g_append == 1, "a good kv_append");
  auto no_append = [&](const char* what, int32_t want, const std::function<void(kv_append_desc&)>& change) {
    kv_append_desc b = d;
    change(b);
    const int before = g_append;
    expect(kv_append(p, &b, s) == want && g_append == before, what);
  };
  expect(kv_append(nullptr, &d, s) == bad && kv_append(p, nullptr, s) == bad, "no pool, no description");
  no_append("partition", bad, [](kv_append_desc& b) { b.partition = 4; });
  no_append("layer", bad, [](kv_append_desc& b) { b.layer = 2; });
  no_append("type", bad, [](kv_append_desc& b) { b.dtype = -1; });
  no_append("odd rotation", bad, [](kv_append_desc& b) { b.rope.rot_dim = 63; });
  no_append("rotation beyond the head", bad, [](kv_append_desc& b) { b.rope.rot_first = 2; });
  no_append("long rotation", bad, [](kv_append_desc& b) { b.rope.rot_dim = 258; });
  no_append("axes", bad, [](kv_append_desc& b) { b.rope.n_axes = 0; });
  no_append("many axes", bad, [](kv_append_desc& b) { b.rope.n_axes = 5; });
  no_append("an axis beyond", bad, [](kv_append_desc& b) { b.rope.axis[31] = 3; });
  no_append("frequencies", bad, [](kv_append_desc& b) { b.rope.d_inv_freq = nullptr; });
  no_append("positions", bad, [](kv_append_desc& b) { b.d_pos = nullptr; });
  no_append("keys", bad, [](kv_append_desc& b) { b.d_k = nullptr; });
  no_append("values", bad, [](kv_append_desc& b) { b.d_v = nullptr; });
  no_append("queries without a place", bad, [](kv_append_desc& b) { b.d_q_out = nullptr; });
  no_append("a place without queries", bad, [](kv_append_desc& b) { b.d_q = nullptr; });
  no_append("slots", bad, [](kv_append_desc& b) { b.d_slot = nullptr; });
  no_append("table", bad, [](kv_append_desc& b) { b.d_table = nullptr; });
  no_append("many tokens", bad, [](kv_append_desc& b) { b.n_tokens = 1ull << 31; });
  no_append("no tokens", KV_OK, [](kv_append_desc& b) { b.n_tokens = 0; });
  d.d_q = d.d_q_out = nullptr;
  d.rope.rot_dim = 0;
  d.d_pos = nullptr;
  expect(kv_append(p, &d, s) == KV_OK && g_append == 2, "keys and values alone, nothing turned");

  // ---- kv_attention_score ----
  uint64_t* const w = (uint64_t*)mem;
  float* const acc = (float*)mem;
  expect(kv_attention_score(p, 1, 0.5f, 2, w, acc, s) == KV_OK && g_score == 1, "a good kv_attention_score");
  expect(kv_attention_score(nullptr, 1, 0.5f, 2, w, acc, s) == bad && kv_attention_score(p, 1, -0.1f, 2, w, acc, s) == bad &&
             kv_attention_score(p, 1, 1.1f, 2, w, acc, s) == bad && kv_attention_score(p, 1, NAN, 2, w, acc, s) == bad &&
             kv_attention_score(p, 1, 0.5f, 1u << 31, w, acc, s) == bad && kv_attention_score(p, 1, 0.5f, 2, nullptr, acc, s) == bad &&
             kv_attention_score(p, 1, 0.5f, 2, w, nullptr, s) == bad && kv_attention_score(p, 1, 0.5f, 2, w + 1, acc, s) == bad && g_score == 1,
         "refused kv_attention_score");
  kv_pool_destroy(p);

  // ---- models that the operators do not take ----
  struct { kv_model_desc m; int block; int32_t attend, append; } const models[] = {
      {{KV_GQA, 2, 8, 2, 64, 0, 0, 8}, 16, KV_ERR_UNSUPPORTED_VARIANT, KV_ERR_UNSUPPORTED_VARIANT},      // INT8
      {{KV_GQA, 2, 8, 2, 12, 0, 0, 16}, 16, KV_ERR_UNSUPPORTED_VARIANT, KV_OK},                          // rows of 24 bytes
      {{KV_GQA, 2, 8, 2, 264, 0, 0, 16}, 16, KV_ERR_UNSUPPORTED_VARIANT, KV_OK},
      {{KV_MLA, 2, 16, 16, 128, 512, 64, 16}, 64, KV_OK, KV_OK},
      {{KV_MLA, 2, 16, 16, 128, 576, 0, 16}, 64, KV_ERR_UNSUPPORTED_VARIANT, KV_OK},
      {{KV_MLA, 2, 16, 16, 128, 512, 128, 16}, 64, KV_ERR_UNSUPPORTED_VARIANT, KV_OK}};
  for (const auto& x : models) {
    kv_pool* const m = make(x.m, x.block);
    if (!m) return fail("pool of a model");
    kv_attend_desc b = a;
    b.n_groups = 0;
    b.scratch_bytes = 1ull << 40;
    expect(kv_attend(m, &b, s) == x.attend, "attention over a model");
    expect((kv_attend_scratch_bytes(m, 0, 3, 0, 500, 0, 0, 0) != 0) == (x.attend == KV_OK), "its scratch");
    kv_append_desc e = d;
    if (x.m.variant == KV_MLA) e.d_v = nullptr;
    expect(kv_append(m, &e, s) == x.append, "a model's cache");
    if (x.m.variant == KV_MLA) {
      e.d_v = mem;
      expect(kv_append(m, &e, s) == bad, "values of an MLA model");
    }
    kv_pool_destroy(m);
  }
  return g_failed;
}
