// kv_attend where a block is read by many rows: tiles on the fifth-generation tensor cores.
//
// A row tile is 128 rows (query heads of the members of a group, or of a sequence): its scores
// S = Q K^T and its output O = P V are accumulators in tensor memory, 128 lanes x a column for each token or
// output element.  Blocks come by TMA, a box of one block x 64 elements (128 bytes, swizzled), so that a tile
// of tokens lies in shared memory as the matrix instructions want it whatever blocks it is made of; a block
// that is not there is a box outside the tensor, which reads as zeros.
//
// Roles: warps 0 and 3 look blocks up and issue the copies of keys and of values, warps 1 and 2 issue the matrix instructions of
// a team each, and each further group of four warps is a team's softmax, a thread per row: it reads its row
// of S, keeps maximum and sum, and writes the probabilities over S, from where P V takes them as the operand
// in tensor memory.  A team has a row tile, or, where one is all there can be, every other tile of its tokens.  S has two
// places a team, so that the scores of the next tokens are formed while these become probabilities.
// The output is rescaled only when a row's maximum has grown by more than 2^8 since the last time (its sum is kept to the same
// base, so that results are what they were).
//
// MLA: a row of 576 elements is key (all of them) and value (the first 512).  128 x 512 outputs would
// fill the tensor memory, so a CTA takes 256 of the columns, and both CTAs form the scores.  The first 256 elements
// of Q lie in tensor memory, which leaves room for two tiles of 64 tokens in shared memory.
//
// Measured: 64 tokens by two row tiles of 128-element heads take about 2,000 cycles of an SM: exponentials 1,024 at the
// least, products about 1,200, the softmax of either team 1,500 to 1,800 (half of it latencies: waits, reads of tensor memory,
// the maximum), so the chain of a team from scores to probabilities to output bounds it.  64 tokens by 128 MLA rows and half the
// columns: 1,830 cycles on a few SMs, 2,800 on all of them (the L2 is a seventh busy then, the tensor pipe 41 %; what makes
// the difference is not established).  Of the measured matrix rate whole calls reach 0.38 and 0.28.
//
// Every wait is bounded: one that gives up sets KV_DEV_WAIT_EXPIRED and a flag that ends the other
// waits; copies and matrix instructions in flight are then waited for (bounded) before the CTA leaves.
#include "kv_attend_device.cuh"
#include "kv_attend_tma.cuh"

namespace kvt {
namespace {

__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// An operand's descriptor: the lower half moves with the address, the upper half is the same for all (see operand()).
constexpr uint32_t kOperandHigh = (1024u >> 4) | 1u << 14 | 2u << 29;
// D (+)= A B, A and B from shared memory
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\tsetp.ne.u32 p, %4, 0;\n\tmov.b64 x, {%1, %5};\n\tmov.b64 y, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(add), "r"(kOperandHigh)
      : "memory");
}
// A from tensor memory
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 y;\n\tsetp.ne.u32 p, %4, 0;\n\tmov.b64 y, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(add), "r"(kOperandHigh)
      : "memory");
}
// One thread of the warp.
__device__ __forceinline__ bool elected() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}
#define KVT_R8(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]), "=r"(r[i + 4]), "=r"(r[i + 5]), "=r"(r[i + 6]), "=r"(r[i + 7])
#define KVT_W8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])
// 32 columns of the thread's lane
__device__ __forceinline__ void tmem_load(uint32_t* r, uint32_t at) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
      "%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : KVT_R8(r, 0), KVT_R8(r, 8), KVT_R8(r, 16), KVT_R8(r, 24)
      : "r"(at));
}
__device__ __forceinline__ void tmem_store(uint32_t at, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,"
      "%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::KVT_W8(r, 0),
      KVT_W8(r, 8), KVT_W8(r, 16), KVT_W8(r, 24), "r"(at)
      : "memory");
}
#define KVT_U8(r, i) "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7])
// The loads are complete; what uses r comes behind.
__device__ __forceinline__ void tmem_loaded(uint32_t* r) {
  asm volatile("" : KVT_U8(r, 0), KVT_U8(r, 8));
  asm volatile("" : KVT_U8(r, 16), KVT_U8(r, 24));
}
__device__ __forceinline__ void tmem_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Two 32-bit operations in one instruction.
struct Pair {
  unsigned long long v;
  __device__ __forceinline__ Pair(float lo, float hi) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi)); }
  __device__ __forceinline__ void get(float& lo, float& hi) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
};
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(a.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return a;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(a.v) : "l"(a.v), "l"(b.v));
  return a;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Operand in shared memory, 128-byte rows with the 128-byte swizzle: groups of eight rows 1,024 bytes apart
// (the upper half); `panels`: distance of the 64-element panels of an operand whose rows run along the
// product's sum (V: a row is a token).
__device__ __forceinline__ uint32_t operand(uint32_t at, uint32_t panels) { return (at >> 4) | (panels >> 4) << 16; }
// 32-bit accumulators, operands of T, M = 128; tr: B's rows run along the sum
template <typename T>
__device__ __forceinline__ constexpr uint32_t instruction(uint32_t n, bool tr) {
  const uint32_t type = sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
  return 1u << 4 | type << 7 | type << 10 | (tr ? 1u : 0u) << 16 | (n >> 3) << 17 | (128u >> 4) << 24;
}

// Shapes.  kDk, kDv: elements of a key and of a value row; kCols: output columns of a CTA; kTok: tokens of a tile.
template <int kDk_, int kDv_, int kCols_, int kTiles_, int kTok_, int kStages_>
struct Shape {
  static constexpr int kDk = kDk_, kDv = kDv_, kCols = kCols_, kTiles = kTiles_, kTok = kTok_, kStages = kStages_;
  static constexpr bool kLatent = kDk != kDv;               // value rows lie in the key rows
  static constexpr int kQTmem = kLatent ? 256 : 0;          // elements of Q in tensor memory
  static constexpr int kQPanels = (kDk - kQTmem) / 64;
  static constexpr int kPanelBytes = kTok * 128;            // a tile's tokens x 64 elements
  // A stage has two parts that are filled and given back on their own: keys and values, or (MLA) the panels that only
  // the scores read and the CTA's columns of the values, which the scores read too.
  static constexpr int kAPanels = kLatent ? (kDk - kCols) / 64 : kDk / 64, kBPanels = kCols / 64;
  static constexpr int kKBytes = kAPanels * kPanelBytes, kVBytes = kBPanels * kPanelBytes;
  static constexpr int kQBytes = kTiles * kQPanels * 128 * 128;
  static constexpr int kMasks = 8;                          // see the softmax
  static constexpr int kFirst = 4;                          // first warp of the softmax
  static constexpr int kThreads = (kFirst + 4 * kTiles) * 32;
  // tensor memory columns: outputs, then scores, then Q
  static constexpr int kSlots = 2 * kTiles;                 // of scores: two for each row tile, in turn
  static constexpr int kSAt = kTiles * kCols, kQAt = kSAt + kSlots * kTok;
  static constexpr int kTmem = 512;
  static_assert(kQAt + kQTmem / 2 <= kTmem, "tensor memory");
  static_assert(kTok == 64, "four grains of weight");
  static constexpr int kControl = 1024;
  static constexpr int kOutBytes = kTiles == 2 ? 32768 : 0;    // 4 KB a warp, where its results change places (MLA: in the queries' place)
  static constexpr size_t kSmem = (size_t)kQBytes + kStages * (kKBytes + kVBytes) + kOutBytes + kControl + 1024;
  static_assert(kSmem <= 232448, "shared memory of a CTA");
};

struct Control {   // in shared memory
  unsigned long long k_full[4], k_empty[4], v_full[4], v_empty[4];
  unsigned long long s_full[4], p_ready[4], pv_done[2], o_done[2], q_ready[2];
  uint32_t mask[8][4];
  uint32_t tmem, gave_up;
};
static_assert(sizeof(Control) <= 1024, "control block");

// First element of panel p of a stage's part.
template <typename S>
__host__ __device__ constexpr int panel_at(int part, int p, int col0) {
  return !S::kLatent ? p * 64 : part ? col0 + p * 64 : p * 64 + (p * 64 >= col0 ? S::kCols : 0);
}

// The products of team r.  While the probabilities of tile t are formed, the scores of tile t + 1 are.
template <typename T, typename S, int kCol0>
__device__ __forceinline__ void issue(Control* ctl, uint32_t tmem_, uint32_t q_at, uint32_t ring_at, int r_, uint32_t n_tiles_, bool shared_, uint32_t box_rows_, uint32_t* status) {
  constexpr uint32_t kStage = S::kKBytes + S::kVBytes;
  constexpr uint32_t kScores = instruction<T>(S::kTok, false), kOutput = instruction<T>(S::kCols, true);
  volatile uint32_t* const gave_up = &ctl->gave_up;
  // (the same for the whole warp, so that addresses and descriptors stay in uniform registers)
  const uint32_t tmem = __shfl_sync(~0u, tmem_, 0), n_tiles = __shfl_sync(~0u, n_tiles_, 0);
  const int r = __shfl_sync(~0u, r_, 0);
  const bool shared = __shfl_sync(~0u, (int)shared_, 0) != 0;
  const int q_tile = shared ? 0 : r;
  const uint32_t q_op = operand(q_at + q_tile * (S::kQPanels * 16384), 0), o_at = tmem + r * S::kCols;
  // (tiles counted by themselves: i; in the ring: t)
  auto place = [&](uint32_t i) { return shared ? 2u * i + (uint32_t)r : i; };
  // S_r[i & 1] (+)= Q_r K_t^T over the elements of a stage's part
  auto scores = [&](uint32_t i, uint32_t t, int part) {
    const uint32_t k_op = operand(ring_at + (t % S::kStages) * kStage + (part ? S::kKBytes : 0), 0);
    const uint32_t d = tmem + S::kSAt + (2 * r + (i & 1)) * S::kTok;
#pragma unroll
    for (int p = 0; p < (part ? S::kBPanels : S::kAPanels); ++p) {
      const int at = panel_at<S>(part, p, kCol0);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t b = k_op + (p * S::kPanelBytes + k * 32) / 16, add = part || p || k;
        if (at < S::kQTmem) mma_ts(d, tmem + S::kQAt + at / 2 + k * 8, b, kScores, add);
        else mma_ss(d, q_op + ((at - S::kQTmem) / 64 * 16384 + k * 32) / 16, b, kScores, add);
      }
    }
  };
  // values: (MLA) panels of a tile, else panels of a block, blocks one after the other
  const uint32_t box_rows = __shfl_sync(~0u, box_rows_, 0), v_panel = S::kLatent ? S::kPanelBytes : box_rows * 128u;
  uint32_t v_step[S::kTok / 16];
#pragma unroll
  for (int k = 0; k < S::kTok / 16; ++k)
    v_step[k] = S::kLatent ? k * 128u : (k * 16u / box_rows * (S::kBPanels * v_panel) + k * 16u % box_rows * 128u) / 16u;
  auto output = [&](uint32_t i, uint32_t t) {   // O_r += P_r[i & 1] V_t
    const uint32_t v_op = operand(ring_at + (t % S::kStages) * kStage + S::kKBytes, v_panel);
    const uint32_t p_at = tmem + S::kSAt + (2 * r + (i & 1)) * S::kTok;
#pragma unroll
    for (int k = 0; k < S::kTok / 16; ++k) mma_ts(o_at, p_at + k * 8, v_op + v_step[k], kOutput, k ? 1u : i);
  };
  auto wait = [&](unsigned long long* bar, uint32_t parity) {
    return __all_sync(~0u, bar_wait(smem_address(bar), parity, gave_up, status));
  };
  // both: asked at once, as an answer takes a while even where it is yes
  auto wait2 = [&](unsigned long long* bar, uint32_t parity, unsigned long long* bar2, uint32_t parity2) {
    const bool a = bar_test(smem_address(bar), parity), b = bar_test(smem_address(bar2), parity2);
    if (__all_sync(~0u, a && b)) return true;
    return wait(bar, parity) && wait(bar2, parity2);
  };
  auto next_scores = [&](uint32_t i) {
    const uint32_t t = place(i), st = t % S::kStages, parity = (t / S::kStages) & 1;
    // these scores take the place of probabilities that an output of two tiles ago is formed from: products of
    // different accumulators may overlap, so it has to be complete
    if (i < 2 ? !wait(&ctl->k_full[st], parity) : !wait2(&ctl->k_full[st], parity, &ctl->pv_done[r], i & 1)) return false;
    fence_after();
    if (elected()) {
      scores(i, t, 0);
      if (!S::kLatent) commit(smem_address(&ctl->s_full[2 * r + (i & 1)]));
      commit(smem_address(&ctl->k_empty[st]));
    }
    __syncwarp();
    if (S::kLatent) {
      if (!wait(&ctl->v_full[st], parity)) return false;
      if (elected()) {
        scores(i, t, 1);
        commit(smem_address(&ctl->s_full[i & 1]));
      }
      __syncwarp();
    }
    return true;
  };
  if (!wait(&ctl->q_ready[q_tile], 0)) return;
  fence_after();
  if (!next_scores(0)) return;
  for (uint32_t i = 0; i < n_tiles; ++i) {
    if (i + 1 < n_tiles && !next_scores(i + 1)) return;
    const uint32_t t = place(i), st = t % S::kStages;
    if (!wait2(&ctl->v_full[st], (t / S::kStages) & 1, &ctl->p_ready[2 * r + (i & 1)], (i >> 1) & 1)) return;
    fence_after();
    if (elected()) {
      output(i, t);
      commit(smem_address(&ctl->pv_done[r]));
      commit(smem_address(&ctl->v_empty[st]));
      if (i + 1 == n_tiles) commit(smem_address(&ctl->o_done[r]));
    }
    __syncwarp();
  }
}

// A row tile's queries, a thread for each row: the first elements (MLA) into tensor memory, the others into shared memory as
// the copies would lay them.  (Short loops: this runs once, and its instructions come from memory.  Written out for all
// of a row's vectors it took 15,000 cycles.)
template <typename T, typename S>
__device__ __forceinline__ void load_queries(const AttendArgs& a, const Item& w, uint8_t* q_s, uint32_t tmem, int r, uint32_t in_tile, uint32_t lane_at,
                                             uint32_t q_sign, uint32_t q_bits) {
  const uint32_t row = r * 128u + in_tile;
  const bool there = row < w.rows;
  uint32_t seq = 0, head = 0;
  if (there) row_of(a, w, row, seq, head);
  const T* const src = static_cast<const T*>(a.q) + (int64_t)seq * a.q_seq + (int64_t)head * a.q_head;
  const bool wide = (reinterpret_cast<uintptr_t>(a.q) & 15u) == 0 && a.q_seq % 8 == 0 && a.q_head % 8 == 0;
  constexpr int kVecs = S::kDk / 8, kInTmem = S::kQTmem / 8;    // 16-byte vectors of a row
#pragma unroll 1
  for (int c0 = 0; c0 < kVecs; c0 += 8) {                       // a panel at a time
    uint4 v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = make_uint4(0, 0, 0, 0);
    if (there && wide) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = reinterpret_cast<const uint4*>(src)[c0 + e];
    } else if (there) {
#pragma unroll 1
      for (int e = 0; e < 64; ++e) {
        const uint32_t x = (uint32_t)reinterpret_cast<const uint16_t*>(src)[c0 * 8 + e] << (e % 2 * 16);
#pragma unroll
        for (int k = 0; k < 32; ++k)
          if (k == e / 2) (&v[k / 4].x)[k % 4] |= x;
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = make_uint4((v[e].x & q_bits) ^ q_sign, (v[e].y & q_bits) ^ q_sign, (v[e].z & q_bits) ^ q_sign, (v[e].w & q_bits) ^ q_sign);
    if (c0 < kInTmem) {
      uint32_t x[32];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[4 * e] = v[e].x;
        x[4 * e + 1] = v[e].y;
        x[4 * e + 2] = v[e].z;
        x[4 * e + 3] = v[e].w;
      }
      tmem_store(tmem + (lane_at << 16) + S::kQAt + c0 * 4, x);
    } else {
      uint8_t* const to = q_s + (r * S::kQPanels + (c0 - kInTmem) / 8) * 16384u + in_tile * 128u;
#pragma unroll
      for (int e = 0; e < 8; ++e) *reinterpret_cast<uint4*>(to + ((e ^ (in_tile & 7u)) * 16u)) = v[e];
    }
  }
  if (S::kQTmem) tmem_wait_store();
  proxy_fence();
  fence_before();
}

template <typename T, typename S, bool kWeights>
__global__ void __launch_bounds__(S::kThreads, 1) tiles_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap map,
                                                               const __grid_constant__ CUtensorMap map_wide,
                                                               uint32_t first_kind_items, uint32_t box_rows, uint32_t outside,
                                                               uint32_t q_sign, uint32_t q_bits) {
  constexpr int kHalves = S::kDv / S::kCols;   // CTAs that share out a row tile's columns
  extern __shared__ uint8_t raw[];
  uint8_t* const smem = raw + ((1024u - (smem_address(raw) & 1023u)) & 1023u);
  uint8_t* const q_s = smem;
  uint8_t* const ring = smem + S::kQBytes;
  uint8_t* const outs = S::kOutBytes ? ring + S::kStages * (S::kKBytes + S::kVBytes) : q_s;
  Control* const ctl = reinterpret_cast<Control*>(ring + S::kStages * (S::kKBytes + S::kVBytes) + S::kOutBytes);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  wait_for_kernel_ahead();

  Item w;
  uint32_t i = blockIdx.x / kHalves;
  const uint32_t col0 = blockIdx.x % kHalves * S::kCols;
  const bool second = i >= first_kind_items;
  if (!item_of(a, second ? kKindSuffix : kKindPrefix, second ? i - first_kind_items : i, S::kTiles * 128, w, threadIdx.x == 0 && col0 == 0)) return;
  if (w.to == 0) {
    if (col0 == 0) put_nothing<T>(a, w, threadIdx.x, blockDim.x);
    return;
  }
  // Two teams, each with its scores, output and softmax: of a row tile each, or, where one is all there can be, of every
  // other tile of tokens (their results are parts of their own).
  const bool shared = a.per_chunk[w.kind] == 2u;
  const int teams = shared || w.rows > 128u ? 2 : 1;
  const TableView& tv = a.tv;
  const uint32_t n_tiles = (w.to - w.from + S::kTok - 1u) / S::kTok;

  if (threadIdx.x == 0) {
    for (int b = 0; b < 4; ++b) {
      bar_init(smem_address(&ctl->k_full[b]), 1);
      bar_init(smem_address(&ctl->k_empty[b]), shared ? 1 : teams);
      bar_init(smem_address(&ctl->v_full[b]), 1);
      bar_init(smem_address(&ctl->v_empty[b]), shared ? 1 : teams);
      bar_init(smem_address(&ctl->s_full[b]), 1);
      bar_init(smem_address(&ctl->p_ready[b]), 128);
    }
    for (int b = 0; b < 2; ++b) {
      bar_init(smem_address(&ctl->pv_done[b]), 1);
      bar_init(smem_address(&ctl->o_done[b]), 1);
      bar_init(smem_address(&ctl->q_ready[b]), 128);
    }
    ctl->gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    proxy_fence();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_address(&ctl->tmem)), "r"(S::kTmem) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = ctl->tmem;
  volatile uint32_t* const gave_up = &ctl->gave_up;
  uint32_t* const status = tv.status;

  if (warp < S::kFirst) {
    // (one instruction for the four warps of the warpgroup, whatever their roles; 72 registers and 216 for the softmax make their
    // code spill: a document's prefix and suffixes 117 us, these 114)
    if (S::kTiles == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 120;");
    if (warp == 0 || warp == 3) {
      // ---- blocks: a warp for each part of the stages ----
      const int part = warp == 0 ? 0 : 1;
      const uint32_t bytes = part ? S::kVBytes : S::kKBytes, panels = part ? S::kBPanels : S::kAPanels;
      const int32_t kv = part && !S::kLatent ? 1 : 0;
      // boxes of a tile; the lanes look the blocks of 32 of them up at a time, before they are needed
      const uint32_t rows_per_box = box_rows, boxes = S::kTok / rows_per_box, ahead = 32u / boxes;
      auto look = [&](uint32_t t) {   // of tiles t .. t + ahead - 1: the place of box lane % boxes of tile t + lane / boxes
        const uint32_t at = w.from + (t * boxes + lane) * rows_per_box;
        if ((uint32_t)lane >= boxes * ahead || at >= w.to) return outside;
        const uint32_t b = tv.by_tokens(at), ch = tv.chunk((uint64_t)w.seg.row + b, w.head);
        return ch == ~0u ? outside : ch * tv.block_tokens + at - b * tv.block_tokens;
      };
      uint32_t next = look(0), now = outside;
      bool ok = true;
      for (uint32_t t = 0; t < n_tiles && ok; ++t) {
        const uint32_t st = t % S::kStages, round = t / S::kStages;
        if (t % ahead == 0) {
          now = next;
          if (t + ahead < n_tiles) next = look(t + ahead);
        }
        const uint32_t first = t % ahead * boxes, tile0 = w.from + t * S::kTok;
        uint32_t bits[S::kTok / 32];
        if (part == 0) {
  #pragma unroll
          for (int m = 0; m < S::kTok / 32; ++m) {
            const uint32_t tok = m * 32 + lane;
            bits[m] = __ballot_sync(~0u, __shfl_sync(~0u, now, first + tok / rows_per_box) != outside && tile0 + tok < w.to);
          }
        }
        if (round) ok = bar_wait(smem_address(part ? &ctl->v_empty[st] : &ctl->k_empty[st]), (round - 1) & 1, gave_up, status);
        ok = __all_sync(~0u, ok);
        if (!ok) break;
        const uint32_t bar = smem_address(part ? &ctl->v_full[st] : &ctl->k_full[st]);
        if (lane == 0) {
          if (part == 0) {   // (ahead of the copies that the scores wait for)
  #pragma unroll
            for (int m = 0; m < S::kTok / 32; ++m) ctl->mask[t % S::kMasks][m] = bits[m];
          }
          bar_expect(bar, bytes);
        }
        __syncwarp();
        const uint32_t dst = smem_address(ring) + st * (S::kKBytes + S::kVBytes) + (part ? S::kKBytes : 0);
        const uint32_t at = __shfl_sync(~0u, now, first + lane % boxes);      // (lane < boxes: its box's rows)
        if (part && !S::kLatent) {             // values lie block by block, all panels of a block in one box
          if ((uint32_t)lane < boxes) tma_box(dst + lane * rows_per_box * 128u * S::kBPanels, &map_wide, 0, (int32_t)at, 1, bar);
        } else if (boxes == 1u) {              // a block (or more) is a tile: the panels in wide boxes, and (MLA) the last one of the scores'
          if (lane == 0) tma_box(dst, &map_wide, panel_at<S>(part, 0, col0) / 64, (int32_t)at, kv, bar);
          if (S::kLatent && part == 0 && lane == 0) tma_box(dst + (S::kAPanels - 1) * S::kPanelBytes, &map, S::kDk / 64 - 1, (int32_t)at, 0, bar);
        } else {                               // a lane for each box of each panel
          for (uint32_t x0 = 0; x0 < boxes * panels; x0 += 32u) {
            const uint32_t x = x0 + lane, p = x / boxes, box = x - p * boxes;
            const uint32_t y = __shfl_sync(~0u, now, first + box);
            if (x < boxes * panels) tma_box(dst + p * S::kPanelBytes + box * rows_per_box * 128u, &map, panel_at<S>(part, p, col0) / 64, (int32_t)y, kv, bar);
          }
        }
      }
    } else {
      // ---- matrix instructions: a warp for each row tile; the whole warp waits, one thread issues ----
      const int r = warp - 1;
      const uint32_t mine = shared ? (n_tiles + 1u - r) / 2u : n_tiles;
      if (r < teams && mine) {
        if (S::kDv == S::kCols || col0 == 0) issue<T, S, 0>(ctl, tmem, smem_address(q_s), smem_address(ring), r, mine, shared, box_rows, status);
        else issue<T, S, S::kDv - S::kCols>(ctl, tmem, smem_address(q_s), smem_address(ring), r, mine, shared, box_rows, status);
      }
    }
  } else {
    // ---- softmax: a thread per row ----
    if (S::kTiles == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");   // 128 x (120 + 2 x 192) of 384 x 168
    const int r = (warp - S::kFirst) / 4;
    const uint32_t lane_at = (uint32_t)(warp & 3) * 32u;   // a warp reaches the lanes of its number modulo four
    const uint32_t row = (shared ? 0u : r * 128u) + lane_at + lane;
    const uint32_t my_tiles = shared ? (n_tiles + 1u - r) / 2u : n_tiles;
    if (r < teams && !my_tiles) {
      if (row < w.rows) {     // (a chunk of one tile: nothing for the second team)
        uint32_t seq, head;
        row_of(a, w, row, seq, head);
        put_lse(a, seq, head, part_of(a, w) + r, -INFINITY);
      }
    } else if (r < teams) {
      const bool mine = row < w.rows;
      const uint32_t o_at = tmem + (lane_at << 16) + r * S::kCols;
      if (r == 0 || !shared) {
        load_queries<T, S>(a, w, q_s, tmem, r, lane_at + lane, lane_at, q_sign, q_bits);
        bar_arrive(smem_address(&ctl->q_ready[r]));
      }
      float m = -INFINITY, l = 0.0f;
      for (uint32_t i = 0; i < my_tiles; ++i) {
        const uint32_t t = shared ? 2u * i + r : i;
        const int slot = 2 * r + (int)(i & 1);
        const uint32_t s_at = tmem + (lane_at << 16) + S::kSAt + slot * S::kTok;
        // (The tile's mask was written ahead of the copies that the scores have waited for.  It is written again eight tiles on,
        // when the scores four tiles on are complete, which have waited for this tile's output.)
        // A wait that gives up lets the loop run out: every later one returns at once, and nothing leaves its bounds.
        bar_wait(smem_address(&ctl->s_full[slot]), (i >> 1) & 1, gave_up, status);
        __syncwarp();
        fence_after();
        uint32_t bits[S::kTok];
        float* const s = reinterpret_cast<float*>(bits);
#pragma unroll
        for (int c = 0; c < S::kTok / 32; ++c) tmem_load(bits + c * 32, s_at + c * 32);
        tmem_wait_load();
#pragma unroll
        for (int c = 0; c < S::kTok / 32; ++c) tmem_loaded(bits + c * 32);
        uint32_t mask[S::kTok / 32], all = ~0u;
#pragma unroll
        for (int c = 0; c < S::kTok / 32; ++c) {
          mask[c] = ctl->mask[t % S::kMasks][c];
          all &= mask[c];
        }
        if (all != ~0u) {
#pragma unroll
          for (int e = 0; e < S::kTok; ++e)
            if (!(mask[e / 32] >> (e % 32) & 1u)) s[e] = -INFINITY;
        }
        float top[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) top[k] = fmaxf(s[k], s[k + 8]);
#pragma unroll
        for (int e = 16; e < S::kTok; e += 16)
#pragma unroll
          for (int k = 0; k < 8; ++k) top[k] = max3(top[k], s[e + k], s[e + k + 8]);
        const float mx = fmaxf(max3(max3(top[0], top[1], top[2]), top[3], top[4]), max3(top[5], top[6], top[7])) * a.scale2;
        // the base follows the maximum when it has grown by 8 (or from nothing)
        float turn_by = 1.0f;
        if (mx > m + 8.0f || (m == -INFINITY && mx > m)) {
          turn_by = exp2_(m - mx);
          m = mx;
          l *= turn_by;
        }
        const float base = m == -INFINITY ? 0.0f : m;
        const Pair scale(a.scale2, a.scale2), minus(-base, -base);
        if (i > 0 && __any_sync(~0u, turn_by != 1.0f)) {
          // (no product of this row tile is under way: the next waits for these probabilities)
          bar_wait(smem_address(&ctl->pv_done[r]), (i - 1) & 1, gave_up, status);
          __syncwarp();
          fence_after();
#pragma unroll 1
          for (int c = 0; c < S::kCols / 32; ++c) {
            uint32_t o[32];
            tmem_load(o, o_at + c * 32);
            tmem_wait_load();
            tmem_loaded(o);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * turn_by);
            tmem_store(o_at + c * 32, o);
          }
          tmem_wait_store();
        }
        Pair sums[4] = {Pair(0.0f, 0.0f), Pair(0.0f, 0.0f), Pair(0.0f, 0.0f), Pair(0.0f, 0.0f)};
#pragma unroll
        for (int e = 0; e < S::kTok; e += 2) {
          float x, y;
          fma2(Pair(s[e], s[e + 1]), scale, minus).get(x, y);
          x = exp2_(x);
          y = exp2_(y);
          sums[kWeights ? e / 16 : e / 2 % 4] = add2(sums[kWeights ? e / 16 : e / 2 % 4], Pair(x, y));   // (with weights: by grains)
          bits[e / 2] = pack2<T>(x, y);
        }
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          float lo, hi;
          sums[g].get(lo, hi);
          const float both = lo + hi;
          l += both;
          if (kWeights && mine && col0 == 0 && w.from + t * S::kTok + g * 16u < w.to)
            grain_at(a, w, (w.from + t * S::kTok) / 16u + g)[row] = base + log2_(both);
        }
#pragma unroll
        for (int c = 0; c < S::kTok / 64; ++c) tmem_store(s_at + c * 32, bits + c * 32);
        tmem_wait_store();
        // what lies behind the last token, in its block, would meet probabilities of zero: it may be anything
        const uint32_t left = w.to - (w.from + t * S::kTok);
        if (left < (uint32_t)S::kTok && left % box_rows) {
          bar_wait(smem_address(&ctl->v_full[t % S::kStages]), (t / S::kStages) & 1, gave_up, status);
          uint8_t* const vt = ring + (t % S::kStages) * (S::kKBytes + S::kVBytes) + S::kKBytes;
          const uint32_t end = (left + box_rows - 1u) / box_rows * box_rows;
          for (uint32_t x = lane_at + lane; x < (end - left) * (S::kCols / 8u); x += 128u) {
            const uint32_t tok = left + x / (S::kCols / 8u), c = x % (S::kCols / 8u);
            const uint32_t to = S::kLatent ? c / 8u * S::kPanelBytes + tok * 128u
                                           : (tok / box_rows * S::kBPanels + c / 8u) * box_rows * 128u + tok % box_rows * 128u;
            *reinterpret_cast<uint4*>(vt + to + (c % 8u) * 16u) = make_uint4(0, 0, 0, 0);
          }
          proxy_fence();
        }
        fence_before();
        bar_arrive(smem_address(&ctl->p_ready[slot]));
      }
      if (__all_sync(~0u, bar_wait(smem_address(&ctl->o_done[r]), 0, gave_up, status))) {
        fence_after();
        uint32_t seq = 0, head = 0;
        if (mine) row_of(a, w, row, seq, head);
        const uint32_t part = part_of(a, w) + (shared ? r : 0);
        const float inv = l != 0.0f ? 1.0f / l : 0.0f;
        // A warp's 32 rows x 32 columns at a time change places in shared memory (16-byte chunks of a row exchanged by the row), so
        // that eight lanes write a row's 128 bytes instead of each a row's 16.
        uint8_t* const place = outs + (warp - S::kFirst) * 4096;
        const bool narrow_ok = (reinterpret_cast<uintptr_t>(a.out) & 7u) == 0 && a.out_seq % 4 == 0 && a.out_head % 4 == 0;
        const uint64_t row_at = !mine ? ~0ull : a.direct ? (uint64_t)((int64_t)seq * a.out_seq + (int64_t)head * a.out_head)
                                                         : (((uint64_t)seq * a.q_heads + head) * a.n_parts + part) * a.dv;
#pragma unroll 1
        for (int c = 0; c < S::kCols / 32; ++c) {
          uint32_t o[32];
          tmem_load(o, o_at + c * 32);
          tmem_wait_load();
          tmem_loaded(o);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            *reinterpret_cast<float4*>(place + lane * 128 + ((e ^ (lane & 7)) * 16)) =
                make_float4(__uint_as_float(o[4 * e]) * inv, __uint_as_float(o[4 * e + 1]) * inv, __uint_as_float(o[4 * e + 2]) * inv,
                            __uint_as_float(o[4 * e + 3]) * inv);
          __syncwarp();
#pragma unroll 2
          for (int k = 0; k < 8; ++k) {
            const int of = k * 4 + lane / 8, e = lane % 8;
            const uint64_t at = (uint64_t)__shfl_sync(~0u, (uint32_t)row_at, of) | (uint64_t)__shfl_sync(~0u, (uint32_t)(row_at >> 32), of) << 32;
            const float4 v = *reinterpret_cast<const float4*>(place + of * 128 + ((e ^ (of & 7)) * 16));
            if (at == ~0ull) continue;
            const uint32_t col = col0 + c * 32 + e * 4;
            if (!a.direct) {
              *reinterpret_cast<float4*>(a.part_o + at + col) = v;
            } else if (narrow_ok) {
              *reinterpret_cast<uint2*>(static_cast<T*>(a.out) + (int64_t)at + col) = make_uint2(pack2<T>(v.x, v.y), pack2<T>(v.z, v.w));
            } else {
              T* const to = static_cast<T*>(a.out) + (int64_t)at + col;
              to[0] = narrow<T>(v.x);
              to[1] = narrow<T>(v.y);
              to[2] = narrow<T>(v.z);
              to[3] = narrow<T>(v.w);
            }
          }
          __syncwarp();
        }
        if (mine && col0 == 0) put_lse(a, seq, head, part, l != 0.0f ? m + log2_(l) : -INFINITY);
      }
    }
  }
  fence_before();
  __syncthreads();
  fence_after();
  if (warp == 1) {
    if (ctl->gave_up) {
      // copies and products in flight end before the memory is given back
      if (lane == 0) {
        commit(smem_address(&ctl->pv_done[0]));
        for (uint32_t k = 0; k < 1u << 16; ++k) asm volatile("nanosleep.u32 1000;");
      }
      __syncwarp();
    }
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kTmem));
  }
}

template <typename F>
int registers_of(F* kernel) {
  cudaFuncAttributes f{};
  return cudaFuncGetAttributes(&f, kernel) == cudaSuccess ? f.numRegs : 0;
}

template <typename T, typename S>
cudaError_t launch(const AttendArgs& a, bool prefix, bool suffix, cudaStream_t s) {
  const TableView& tv = a.tv;
  const uint32_t box = tv.block_tokens < (uint32_t)S::kTok ? tv.block_tokens : (uint32_t)S::kTok;
  const uint64_t rows = tv.n * tv.n_chunks * tv.block_tokens;
  CUtensorMap map, map_wide;
  if (!block_map(tv, S::kDk, box, 1, 1, &map) || !block_map(tv, S::kDk, box, S::kBPanels, 1, &map_wide)) return cudaErrorInvalidValue;
  const uint64_t tile = S::kTiles * 128;
  const uint64_t np = prefix ? ((uint64_t)a.max_members * a.group + tile - 1) / tile * a.chunks[0] * tv.heads * a.n_groups : 0;
  const uint64_t ns = suffix ? (a.group + tile - 1) / tile * (uint64_t)a.chunks[1] * tv.heads * a.n_seqs : 0;
  const uint64_t grid = (np + ns) * (S::kDv / S::kCols);
  if (grid == 0) return cudaSuccess;
  auto* kernel = a.weight ? tiles_kernel<T, S, true> : tiles_kernel<T, S, false>;
  if (S::kTiles == 2) {
    // (the softmax's warps take up registers that the launch has to have given the CTA: fewer, and they would wait for good)
    static const bool enough[2] = {registers_of(tiles_kernel<T, S, false>) * S::kThreads >= 128 * (120 + 2 * 192),
                                   registers_of(tiles_kernel<T, S, true>) * S::kThreads >= 128 * (120 + 2 * 192)};
    if (!enough[a.weight ? 1 : 0]) return cudaErrorInvalidConfiguration;
  }
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem);
  if (e != cudaSuccess) return e;
  AttendArgs b = a;
  // the base follows the largest product, and what is masked is -inf before it is scaled: a negative scale
  // turns the queries around instead, a scale of 0 makes them zeros
  uint32_t sign = 0, bits = ~0u;
  if (b.scale2 < 0.0f) {
    b.scale2 = -b.scale2;
    sign = 0x80008000u;
  } else if (b.scale2 == 0.0f) {
    b.scale2 = 1.0f;
    bits = 0;
  }
  return launch_overlapped_smem(kernel, (unsigned)grid, (unsigned)S::kThreads, S::kSmem, s, b, map, map_wide, (uint32_t)np, box, (uint32_t)rows, sign, bits);
}

using Heads128 = Shape<128, 128, 128, 2, 64, 4>;
using Heads64 = Shape<64, 64, 64, 2, 64, 4>;
using Latents = Shape<576, 512, 256, 1, 64, 2>;

template <typename T>
cudaError_t launch_typed(const AttendArgs& a, bool mla, bool prefix, bool suffix, cudaStream_t s) {
  if (mla) return launch<T, Latents>(a, prefix, suffix, s);
  return a.dk == 128 ? launch<T, Heads128>(a, prefix, suffix, s) : launch<T, Heads64>(a, prefix, suffix, s);
}

}  // namespace

bool tiles_take(uint32_t dk, uint32_t dv, bool mla, uint32_t block_tokens, uint64_t slab_rows) {
  const uint32_t tok = mla ? Latents::kTok : Heads128::kTok;
  if (mla ? dk != 576 || dv != 512 : dk != 128 && dk != 64) return false;
  if (block_tokens % 16 != 0 || (tok % block_tokens != 0 && block_tokens % tok != 0)) return false;
  // (a box's place is a signed number of rows)
  return slab_rows < 0x7fff0000ull && has_block_map();
}

cudaError_t launch_attend_tiles(const AttendArgs& a, int dtype, bool mla, bool prefix, bool suffix, cudaStream_t s) {
  return dtype == KV_DTYPE_BF16 ? launch_typed<__nv_bfloat16>(a, mla, prefix, suffix, s) : launch_typed<__half>(a, mla, prefix, suffix, s);
}

}  // namespace kvt
