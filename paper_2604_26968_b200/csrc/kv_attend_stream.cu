// kv_attend where few rows read a block: a stream of blocks through independent warps (and the encoder of the maps
// by which the kernels here and in kv_attend_tiles.cu copy blocks).
//
// A warp takes chunks of segments, one after the other, in units of 16 tokens of one block; a block that is not in HBM is no unit.  It has a ring
// of units of its own, filled by TMA (one box of 16 rows: K's panels of 64 elements, swizzled, then V's) which it issues
// itself as it empties them: no warp waits for another.  A unit's scores (16 rows x 16 tokens) and output are mma.sync
// products whose operands come from the ring by ldmatrix, free of bank conflicts thanks to the swizzle.  The output is
// rescaled only when a maximum has grown.
// Bound: HBM.  A unit takes a warp about 2,000 cycles, most of them latencies of its short products and reductions, so it takes
// eight to sixteen warps on every SM, each with two to three units under way; a chunk's start (its segment, its blocks' handles and
// places, the first copies: five reads one after the other) costs as much as three units.
#include "kv_attend_device.cuh"
#include "kv_attend_tma.cuh"

namespace kvt {
namespace {

constexpr int kUnit = kStreamUnit;        // tokens
constexpr int kStreamWarps = 4;
constexpr uint32_t kMaxUnits = kStreamTokens / kUnit;

template <int D>
struct Stream {
  static constexpr int kPanels = D / 64, kPanelBytes = kUnit * 128, kUnitBytes = 2 * kPanels * kPanelBytes;
  static constexpr int kSlots = D == 64 ? 3 : 2;
  static constexpr int kCtas = D == 64 ? 4 : 3;   // of an SM
  static constexpr size_t kRing = (size_t)kStreamWarps * kSlots * kUnitBytes;
  static constexpr size_t kSmem = 1024 + kRing + kStreamWarps * (kMaxUnits * 8 + kSlots * 8 + 8);
};

template <typename T, int D, bool kWeights>
__global__ void __launch_bounds__(kStreamWarps * 32, Stream<D>::kCtas)
    stream_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap map, uint32_t first_kind_items, uint32_t items,
                  uint32_t behind_tiles) {
  using S = Stream<D>;
  extern __shared__ uint8_t raw[];
  uint8_t* const smem = raw + ((1024u - (smem_address(raw) & 1023u)) & 1023u);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  uint8_t* const ring = smem + warp * (S::kSlots * S::kUnitBytes);
  uint2* const units = reinterpret_cast<uint2*>(smem + S::kRing) + warp * kMaxUnits;      // (first row in the slab, first token)
  unsigned long long* const bar = reinterpret_cast<unsigned long long*>(smem + S::kRing + kStreamWarps * kMaxUnits * 8) + warp * (S::kSlots + 1);
  volatile uint32_t* const gave_up = reinterpret_cast<uint32_t*>(bar + S::kSlots);
  // Behind a launch of the tiles kernel, which has waited for all that is ahead of it, the two may run side by side; this
  // one then ends only when that one has.
  if (behind_tiles) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  else wait_for_kernel_ahead();
  struct AtEnd {
    uint32_t wait;
    __device__ ~AtEnd() {
      if (wait) asm volatile("griddepcontrol.wait;" ::: "memory");
    }
  } at_end{behind_tiles};

  const TableView& tv = a.tv;
  if (lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map) : "memory");
#pragma unroll
    for (int b = 0; b < S::kSlots; ++b) bar_init(smem_address(bar + b), 1);
    *gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    proxy_fence();
  }
  __syncwarp();
  // lanes' places in the ring's operands: rows of a unit's panels, 16-byte chunks exchanged by the row
  const uint32_t k_row = (lane >> 4) * 8 + (lane & 7), v_row = (lane >> 3 & 1) * 8 + (lane & 7);
  uint32_t k_off[4], v_off[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    k_off[c] = smem_address(ring) + k_row * 128 + (((2 * c + (lane >> 3 & 1)) ^ (k_row & 7)) * 16);
    v_off[c] = smem_address(ring) + S::kPanels * S::kPanelBytes + v_row * 128 + (((2 * c + (lane >> 4)) ^ (v_row & 7)) * 16);
  }
  uint32_t slot = 0, parity = 0;
  bool ok = true;
  for (uint32_t item = blockIdx.x * kStreamWarps + warp; item < items && ok; item += gridDim.x * kStreamWarps) {
    Item w;
    const bool second = item >= first_kind_items;
    if (!item_of<true>(a, second ? kKindSuffix : kKindPrefix, second ? item - first_kind_items : item, 16, w, lane == 0)) continue;
    if (w.to == 0) {
      put_nothing<T>(a, w, lane, 32);
      continue;
    }
    uint32_t n_units = 0;
    {
      const uint32_t n = (w.to - w.from + kUnit - 1u) / kUnit;
      uint32_t ch[kMaxUnits / 32];
#pragma unroll
      for (int k = 0; k < (int)kMaxUnits / 32; ++k) {
        const uint32_t u = k * 32u + lane;
        ch[k] = u < n ? tv.chunk((uint64_t)w.seg.row + tv.by_tokens(w.from + u * kUnit), w.head) : ~0u;
      }
#pragma unroll
      for (int k = 0; k < (int)kMaxUnits / 32; ++k) {
        const uint32_t at = w.from + (k * 32u + lane) * kUnit;
        const uint32_t there = __ballot_sync(~0u, ch[k] != ~0u);
        if (ch[k] != ~0u)
          units[n_units + __popc(there & ((1u << lane) - 1u))] = make_uint2(ch[k] * tv.block_tokens + (at - tv.by_tokens(at) * tv.block_tokens), at);
        n_units += __popc(there);
      }
    }
    __syncwarp();
    // unit j into a slot: the panels of K, then those of V, in one box
    auto issue = [&](uint32_t j, uint32_t to) {
      if (j < n_units && lane == 0) {
        const uint32_t b = smem_address(bar + to);
        bar_expect(b, S::kUnitBytes);
        tma_box(smem_address(ring + to * S::kUnitBytes), &map, 0, (int32_t)units[j].x, 0, b);
      }
    };
#pragma unroll
    for (int k = 0; k < S::kSlots; ++k) issue(k, slot + k < S::kSlots ? slot + k : slot + k - S::kSlots);
    // queries straight into the operands' registers: rows lane / 4 and 8 further on, elements 2 (lane % 4) and 8 further on
    uint32_t q[D / 16][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t r = lane / 4 + h * 8;
      const bool there = r < w.rows;
      uint32_t seq = 0, head = 0;
      if (there) row_of(a, w, r, seq, head);
      const uint16_t* const src = static_cast<const uint16_t*>(a.q) + (int64_t)seq * a.q_seq + (int64_t)head * a.q_head + (lane & 3) * 2;
      const bool words = (reinterpret_cast<uintptr_t>(src) & 3u) == 0;
#pragma unroll
      for (int k = 0; k < D / 16; ++k)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint16_t* const x = src + k * 16 + e * 8;
          q[k][h + 2 * e] = !there ? 0u : words ? *reinterpret_cast<const uint32_t*>(x) : (uint32_t)x[0] | (uint32_t)x[1] << 16;
        }
    }

    float o[D / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < D / 8; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[j][e] = 0.0f;
    for (uint32_t j = 0; j < n_units; ++j) {
      ok = __all_sync(~0u, bar_wait(smem_address(bar + slot), parity, gave_up, tv.status));
      if (!ok) break;
      uint8_t* const unit = ring + slot * S::kUnitBytes;
      const uint32_t in_ring = slot * S::kUnitBytes;
      const uint32_t at = units[j].y, left = w.to - at;
      const bool tail = left < (uint32_t)kUnit;
      if (tail) {
        // what lies behind the last token would meet probabilities of zero: it may be anything
        for (uint32_t x = lane; x < (kUnit - left) * S::kPanels * 8u; x += 32u) {
          const uint32_t tok = left + x / (S::kPanels * 8u), c = x % (S::kPanels * 8u);
          *reinterpret_cast<uint4*>(unit + (S::kPanels + c / 8u) * S::kPanelBytes + tok * 128u + (c % 8u) * 16u) = make_uint4(0, 0, 0, 0);
        }
        proxy_fence();      // (the warp's next chunk has its first units copied into this slot: behind these zeros)
        __syncwarp();
      }
      // scores, the even and the odd steps of the sum on their own
      float s[2][2][4];
#pragma unroll
      for (int x = 0; x < 16; ++x) s[x / 8][x / 4 % 2][x % 4] = 0.0f;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        uint32_t b[4];
        ldmatrix4(b, k_off[k % 4] + in_ring + k / 4 * S::kPanelBytes);
        mma<T>(s[k & 1][0], q[k], b[0], b[1]);
        mma<T>(s[k & 1][1], q[k], b[2], b[3]);
      }
      float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[0][n][e] = (s[0][n][e] + s[1][n][e]) * a.scale2;
          if (tail && n * 8u + (lane & 3) * 2u + (e & 1) >= left) s[0][n][e] = -INFINITY;
          top[e >> 1] = fmaxf(top[e >> 1], s[0][n][e]);
        }
      float turn[2] = {1.0f, 1.0f};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float mx = quad_max(top[h]);
        if (mx > m[h]) {
          turn[h] = exp2_(m[h] - mx);
          m[h] = mx;
          l[h] *= turn[h];
        }
      }
      if (__any_sync(~0u, turn[0] != 1.0f || turn[1] != 1.0f)) {
#pragma unroll
        for (int d = 0; d < D / 8; ++d) {
          o[d][0] *= turn[0];
          o[d][1] *= turn[0];
          o[d][2] *= turn[1];
          o[d][3] *= turn[1];
        }
      }
      const float base[2] = {m[0] == -INFINITY ? 0.0f : m[0], m[1] == -INFINITY ? 0.0f : m[1]};
      float part[2] = {0.0f, 0.0f};
      uint32_t p[4];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = exp2_(s[0][n][e] - base[e >> 1]);
          s[0][n][e] = x;
          part[e >> 1] += x;
        }
        p[2 * n] = pack2<T>(s[0][n][0], s[0][n][1]);
        p[2 * n + 1] = pack2<T>(s[0][n][2], s[0][n][3]);
      }
      l[0] += part[0];
      l[1] += part[1];
      if (kWeights) {
        float* const grain = grain_at(a, w, at / 16u);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float sum = quad_sum(part[h]);
          const uint32_t r = lane / 4 + h * 8;
          if ((lane & 3) == 0 && r < w.rows) grain[r] = base[h] + log2_(sum);
        }
      }
#pragma unroll
      for (int d = 0; d < D / 16; ++d) {
        uint32_t b[4];
        ldmatrix4t(b, v_off[d % 4] + in_ring + d / 4 * S::kPanelBytes);
        mma<T>(o[2 * d], p, b[0], b[1]);
        mma<T>(o[2 * d + 1], p, b[2], b[3]);
      }
      __syncwarp();
      issue(j + S::kSlots, slot);
      if (++slot == S::kSlots) {
        slot = 0;
        parity ^= 1u;
      }
    }
    if (!ok) break;
    const uint32_t part = part_of(a, w);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float sum = quad_sum(l[h]);
      const uint32_t r = lane / 4 + h * 8;
      if (r >= w.rows) continue;
      uint32_t seq, head;
      row_of(a, w, r, seq, head);
      const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
      for (int j = 0; j < D / 8; ++j) put2<T>(a, seq, head, part, j * 8 + (lane & 3) * 2, o[j][2 * h] * inv, o[j][2 * h + 1] * inv);
      if ((lane & 3) == 0) put_lse(a, seq, head, part, sum != 0.0f ? m[h] + log2_(sum) : -INFINITY);
    }
  }
  if (!ok) {
    // copies in flight end before the memory is given back
    for (uint32_t k = 0; k < 1u << 16; ++k) asm volatile("nanosleep.u32 1000;");
  }
}

typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                           const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's encoder (its address does not change while the process runs).
Encode encoder() {
  static const Encode f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &r) != cudaSuccess || r != cudaDriverEntryPointSuccess) {
      (void)cudaGetLastError();
      p = nullptr;
    }
    return reinterpret_cast<Encode>(p);
  }();
  return f;
}

template <typename T, int D>
cudaError_t launch(const AttendArgs& a, bool prefix, bool suffix, bool behind_tiles, cudaStream_t s) {
  using S = Stream<D>;
  const TableView& tv = a.tv;
  CUtensorMap map;
  if (!block_map(tv, D, kUnit, D / 64, 2, &map)) return cudaErrorInvalidValue;
  const uint64_t np = prefix ? ((uint64_t)a.max_members * a.group + 15) / 16 * a.chunks[0] * tv.heads * a.n_groups : 0;
  const uint64_t ns = suffix ? (a.group + 15) / 16 * (uint64_t)a.chunks[1] * tv.heads * a.n_seqs : 0;
  if (np + ns == 0) return cudaSuccess;
  auto* kernel = a.weight ? stream_kernel<T, D, true> : stream_kernel<T, D, false>;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem);
  if (e != cudaSuccess) return e;
  const uint64_t ctas = (np + ns + kStreamWarps - 1) / kStreamWarps, most = (uint64_t)sm_count() * S::kCtas;
  return launch_overlapped_smem(kernel, (unsigned)(ctas < most ? ctas : most), (unsigned)kStreamWarps * 32, S::kSmem, s, a, map,
                                (uint32_t)np, (uint32_t)(np + ns), behind_tiles ? 1u : 0u);
}

}  // namespace

bool has_block_map() { return encoder() != nullptr; }

bool block_map(const TableView& tv, uint32_t dk, uint32_t box_rows, uint32_t box_panels, uint32_t box_kv, CUtensorMap* map) {
  const Encode f = encoder();
  const uint64_t rows = tv.n * tv.n_chunks * tv.block_tokens, values = (uint64_t)(tv.n_chunks - 1u) * tv.heads * tv.block_tokens;
  const cuuint64_t dims[4] = {64, rows - values, dk / 64, tv.n_chunks}, strides[3] = {(cuuint64_t)dk * 2, 128, values ? values * dk * 2 : 128};
  const cuuint32_t box[4] = {64, box_rows, box_panels, box_kv}, steps[4] = {1, 1, 1, 1};
  return f && f(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 4, tv.slab, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool stream_takes(uint32_t dk, uint32_t dv, bool mla, uint32_t block_tokens, uint64_t slab_rows) {
  return !mla && (dk == 128 || dk == 64) && block_tokens % kUnit == 0 && slab_rows < 0x7fff0000ull && has_block_map();
}

uint32_t stream_warps(uint32_t dk) { return kStreamWarps * (dk == 64 ? Stream<64>::kCtas : Stream<128>::kCtas); }

cudaError_t launch_attend_stream(const AttendArgs& a, int dtype, bool prefix, bool suffix, bool behind_tiles, cudaStream_t s) {
  if (dtype == KV_DTYPE_BF16)
    return a.dk == 128 ? launch<__nv_bfloat16, 128>(a, prefix, suffix, behind_tiles, s) : launch<__nv_bfloat16, 64>(a, prefix, suffix, behind_tiles, s);
  return a.dk == 128 ? launch<__half, 128>(a, prefix, suffix, behind_tiles, s) : launch<__half, 64>(a, prefix, suffix, behind_tiles, s);
}

}  // namespace kvt
