// The order of what kv_append, kv_attend and kv_attention_score enqueue beside demotions and promotions, without a GPU: the
// runtime and the other kernels are the stand-ins of enqueued_order.cu (vector clocks); the operators' launches read the state and the slab of
// every resident entry, kv_append writes some.  kv_attend and kv_append come on the pool's compute stream or on another one (0), which the caller
// orders behind kv_admit and kv_demote, and the compute stream behind it before what changes entries -- and behind kv_promote not at all: the calls
// join promotions themselves.
// usage: attention_order <seed> <deferred 0|1> <gather threshold>   or   attention_order capture
#define main order_main
#include "enqueued_order.cu"
#undef main

#include <functional>

#include "kv_attend.cuh"

static int g_launches = 0;
static cudaStream_t g_captured = (cudaStream_t)99;
static uint64_t g_entries = 0;
static std::vector<uint32_t> g_written;

namespace kvt {
bool stream_captured(cudaStream_t s) { return s == g_captured; }
static void read_all(int s) {
  for (uint64_t i = 0; i < g_entries; ++i) {
    touch(s, "entry state", i, false);
    if (g_state[i] == KV_STATE_RESIDENT) touch(s, "slab entry", i, false);
  }
}
cudaError_t launch_attend(const AttendArgs&, int, bool, cudaStream_t s) { ++g_launches; read_all(op(s, "attend")); return cudaSuccess; }
cudaError_t launch_append(const AppendArgs&, int, bool, cudaStream_t s_) {
  ++g_launches;
  const int s = op(s_, "append");
  for (uint64_t i = 0; i < g_entries; ++i) touch(s, "entry state", i, false);
  for (uint32_t i : g_written) touch(s, "slab entry", i, true);
  return cudaSuccess;
}
cudaError_t launch_attention_score(const EntryState& st, const uint32_t*, uint64_t, uint32_t, float, uint32_t, unsigned long long*, float*, cudaStream_t s_) {
  ++g_launches;
  const int s = op(s_, "attention score");
  for (uint64_t i = 0; i < st.n; ++i) { touch(s, "entry state", i, false); touch(s, "score", i, true); }
  return cudaSuccess;
}
bool tiles_take(uint32_t, uint32_t, bool, uint32_t, uint64_t) { return true; }
bool stream_takes(uint32_t, uint32_t, bool, uint32_t, uint64_t) { return true; }
uint32_t stream_warps(uint32_t) { return 12; }
}  // namespace kvt

static std::vector<std::vector<uint64_t>> g_arrays;
static void* real(uint64_t bytes) {
  g_arrays.emplace_back(bytes / 8 + 4);
  return (void*)(((uintptr_t)g_arrays.back().data() + 15) & ~15ull);
}

int main(int argc, char** argv) {
  const bool capture = argc > 1 && std::string(argv[1]) == "capture";
  if (!capture && argc < 4) return fail("arguments");
  std::mt19937_64 rng(capture ? 1 : std::atoi(argv[1]));
  kv_pool_desc d{};
  d.n_partitions = 2;
  const uint64_t n_part[2] = {2 * 2 * 60, 2 * 2 * 40}, n = n_part[0] + n_part[1], ring = 150;
  for (int q = 0; q < 2; ++q) {
    kv_partition_desc& p = d.part[q];
    p.model = kv_model_desc{KV_AUTO, 2, 4, 2, 128, 0, 0, 16};
    p.block_tokens = 128;   // 64 KB entries
    p.blocks_per_layer = q == 0 ? 60 : 40;
    p.d_slab = (void*)(kSlab + ((uint64_t)q << 40));
    p.h_ring = (void*)(kPinned + ((uint64_t)q << 40));
    p.ring_slots = ring;
  }
  d.n_tags = 1 << 16;
  d.d_ema = (float*)real(n * 4); d.d_decay = (float*)real(n * 4); d.d_touch = (uint32_t*)real(n * 4);
  d.d_last_epoch = (uint32_t*)real(n * 4); d.d_pair = (uint8_t*)real(n); d.d_state = (uint8_t*)real(n);
  d.d_tag = (uint32_t*)real(n * 4); d.d_score = (float*)real(n * 4); d.d_hits = (uint64_t*)real(128);
  d.d_misses = (uint64_t*)real(128); d.d_P = (float*)real(64); d.d_loc = (uint32_t*)real(d.n_tags * 4);
  d.alpha0 = d.beta0 = 1.0f;
  const uint64_t batch = 1u << 20;
  d.staging_bytes = batch + 4096;
  for (int b = 0; b < 4; ++b) d.d_staging[b] = (void*)(kStage + ((uint64_t)b << 32));
  d.max_promote = 1024;
  uint64_t dev = 0, host = 0;
  if (kv_workspace_bytes(&d, &dev, &host) != KV_OK) return fail("kv_workspace_bytes");
  d.d_workspace = real(dev); d.workspace_bytes = dev;
  d.h_workspace = real(host); d.h_workspace_bytes = host;
  g_state.assign(n, KV_STATE_FREE);
  g_entries = n;
  const kv_stream_t compute = (void*)1, d2h = (void*)2, h2d = (void*)3, other = (void*)0;
  kv_pool* p = nullptr;
  if (kv_pool_create(&d, compute, &p) != KV_OK) return fail("kv_pool_create");
  if (kv_set_deferred_packing(p, capture ? 1 : std::atoi(argv[2])) != KV_OK) return fail("deferred");
  if (kv_set_gather_threshold(p, capture ? 0 : std::strtoull(argv[3], nullptr, 10)) != KV_OK) return fail("gather threshold");
  std::vector<uint8_t> pairs(n + 16);
  std::vector<std::vector<uint32_t>> keep;
  auto ids = [&](int q, bool resident) {
    std::vector<uint32_t> v;
    for (uint64_t i = q ? n_part[0] : 0; i < (q ? n : n_part[0]); ++i)
      if ((g_state[i] == KV_STATE_RESIDENT) == resident) v.push_back((uint32_t)i);
    return v;
  };
  auto demote = [&](uint64_t a, uint64_t b) -> int32_t {
    std::vector<uint32_t> v;
    uint64_t counts[4] = {0, 0, 0, 0}, want[2] = {a, b};
    for (int q = 0; q < 2; ++q) {
      std::vector<uint32_t> have = ids(q, true);
      std::shuffle(have.begin(), have.end(), rng);
      have.resize(std::min<uint64_t>({have.size(), want[q], ring}));
      counts[q] = have.size();
      v.insert(v.end(), have.begin(), have.end());
    }
    std::sort(v.begin(), v.end());
    const uint64_t m = v.size();
    v.resize(m + 8);
    keep.push_back(std::move(v));
    uint32_t* at = (uint32_t*)(((uintptr_t)keep.back().data() + 15) & ~15ull);
    std::memmove(at, keep.back().data(), m * 4);
    return m ? kv_demote_counted(p, at, m, counts, batch, compute, d2h) : KV_OK;
  };
  auto promote = [&](int q, uint64_t most) -> int32_t {
    std::vector<uint8_t> l(ring);
    kv_ring_query(p, q, nullptr, nullptr, l.data());
    std::vector<uint64_t> v;
    for (uint64_t i = 0; i < ring; ++i) if (l[i]) v.push_back(i);
    std::shuffle(v.begin(), v.end(), rng);
    v.resize(std::min<uint64_t>({v.size(), most, ids(q, false).size()}));
    return v.empty() ? KV_OK : kv_promote(p, q, v.data(), v.size(), batch, compute, h2d);
  };
  auto check = [&](int32_t rc, const char* what) {
    if (rc != KV_OK && g_bad.empty()) g_bad = std::string(what) + " returned " + std::to_string(rc);
  };
  void* const mem = real(1 << 16);
  kv_attend_desc a{};
  a.dtype = KV_DTYPE_BF16;
  a.scale = 0.125f;
  a.n_seqs = 3;
  a.max_suffix = 100;
  a.d_q = a.d_out = mem;
  a.d_table = a.d_suffix = (const uint32_t*)mem;
  a.n_rows = 20;
  a.d_scratch = real(1 << 20);
  a.scratch_bytes = 1 << 20;
  auto attend = [&](kv_stream_t s) { return kv_attend(p, &a, s); };
  auto append = [&](kv_stream_t s) {
    g_written.clear();
    for (int q = 0; q < 2; ++q) {
      std::vector<uint32_t> v = ids(q, true);
      std::shuffle(v.begin(), v.end(), rng);
      v.resize(std::min<size_t>(v.size(), 5));
      g_written.insert(g_written.end(), v.begin(), v.end());
    }
    kv_append_desc b{};
    b.dtype = KV_DTYPE_BF16;
    b.n_tokens = 5;
    b.d_k = b.d_v = mem;
    b.d_table = (const uint32_t*)mem;
    b.n_rows = 20;
    b.d_slot = (const int64_t*)mem;
    return kv_append(p, &b, s);
  };
  auto score = [&](kv_stream_t s) { return kv_attention_score(p, 1, 0.5f, 0, (uint64_t*)mem, (float*)mem, s); };
  // `to` waits for all that has been enqueued on `from`
  auto order = [&](int from, int to) {
    for (int r = 0; r < kStreams; ++r) g_clock[to][r] = std::max(g_clock[to][r], g_clock[from][r]);
  };
  uint32_t epoch = 0;
  check(kv_admit(p, 0, 0.9f, pairs.data(), pairs.size(), 0, nullptr, compute), "kv_admit");
  order(1, 0);

  if (capture) {
    auto stands = [&](kv_stream_t s, const char* what, const std::function<int32_t(kv_stream_t)>& call) {
      Clock before[kStreams];
      std::memcpy(before, g_clock, sizeof(before));
      const int launches = g_launches;
      g_captured = (cudaStream_t)s;
      const int32_t rc = call(s);
      g_captured = (cudaStream_t)99;
      if ((rc != KV_ERR_CUDA || launches != g_launches || std::memcmp(before, g_clock, sizeof(before))) && g_bad.empty())
        g_bad = std::string(what) + ": not refused, or something was enqueued";
    };
    auto taken = [&](kv_stream_t s, const char* what, const std::function<int32_t(kv_stream_t)>& call) {
      uint64_t seen[kStreams];
      std::memcpy(seen, g_clock[sid((cudaStream_t)s)], sizeof(seen));
      g_captured = (cudaStream_t)s;
      check(call(s), what);
      g_captured = (cudaStream_t)99;
      for (int r = 0; r < kStreams; ++r)      // (a captured stream waits for nothing outside)
        if (r != sid((cudaStream_t)s) && seen[r] != g_clock[sid((cudaStream_t)s)][r] && g_bad.empty()) g_bad = std::string(what) + " waits inside a capture";
      order(1, 0); order(0, 1);               // (the stand-ins do at once what a replay would)
    };
    for (kv_stream_t s : {compute, other}) {
      taken(s, "before any promotion", attend);
      taken(s, "before any promotion", append);
      taken(s, "before any promotion", score);
    }
    check(demote(60, 40), "kv_demote"); order(1, 0);   // (packing is deferred: some of it is held back)
    for (kv_stream_t s : {compute, other}) {
      stands(s, "packing held back", attend);
      stands(s, "packing held back", append);
      stands(s, "packing held back", score);
    }
    check(kv_flush(p), "kv_flush"); order(1, 0);
    for (kv_stream_t s : {compute, other}) taken(s, "behind kv_flush", attend);
    check(promote(0, 20), "kv_promote");
    for (kv_stream_t s : {compute, other}) {
      stands(s, "promotion open", attend);
      stands(s, "promotion open", append);
      stands(s, "promotion open", score);
      stands(s, "promotion open", [&](kv_stream_t x) { return kv_join_promotions(p, x); });
    }
    check(attend(other), "another stream's wait is its own affair");
    stands(compute, "still open", attend);
    order(0, 1);
    check(kv_join_promotions(p, compute), "kv_join_promotions");
    order(1, 0);
    for (kv_stream_t s : {compute, other}) {
      taken(s, "joined", attend);
      taken(s, "joined", append);
      taken(s, "joined", score);
    }
    if (kv_join_promotions(nullptr, compute) != KV_ERR_INVALID_ARG && g_bad.empty()) g_bad = "no pool";
  } else {
    for (int step = 0; step < 150 && g_bad.empty(); ++step) {
      switch (rng() % 10) {
        case 0: case 1:
          order(0, 1);
          check(demote(rng() % 80, rng() % 60), "kv_demote");
          order(1, 0);
          break;
        case 2: case 3: case 4:
          order(0, 1);
          check(promote((int)(rng() % 2), 1 + rng() % 60), "kv_promote");
          break;
        case 5: check(attend(other), "kv_attend"); break;
        case 6: check(attend(compute), "kv_attend"); break;
        case 7:
          if (rng() % 2) { order(0, 1); check(append(compute), "kv_append"); order(1, 0); }
          else { order(1, 0); check(append(other), "kv_append"); order(0, 1); }
          break;
        case 8:
          check(score(compute), "kv_attention_score");
          if (ids(0, true).size() + ids(1, true).size()) check(kv_select_victims(p, 1, (uint32_t*)d.d_score, compute), "kv_select_victims");
          break;
        default:
          order(0, 1);
          if (rng() % 2) check(kv_admit(p, ++epoch, 0.9f, pairs.data(), pairs.size(), 0, nullptr, compute), "kv_admit");
          else check(kv_epoch_score(p, ++epoch, nullptr, nullptr, 0, compute), "kv_epoch_score");
          order(1, 0);
      }
    }
  }
  check(kv_flush(p), "kv_flush");
  kv_pool_destroy(p);
  if (!g_bad.empty()) { std::printf("%s\n", g_bad.c_str()); return 1; }
  return 0;
}
