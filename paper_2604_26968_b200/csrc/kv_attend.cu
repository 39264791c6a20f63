// Attention of one query token per sequence over the pool's blocks; sequences of a group share a prefix
// (kv_attend).
//
//   out_j = sum_t p_t v_t,  p_t = exp(scale q_j k_t - lse_j),  lse_j = log sum_t exp(scale q_j k_t)
//
// over the tokens t of the sequence's prefix and suffix whose blocks are in HBM.  The query heads of a
// KV head -- of all members of a group, where it is a prefix -- are the rows of one small matrix product
// per block, so that a block's K and V leave HBM once for all of them.  A segment's tokens are cut into
// chunks that different CTAs work on; a part (one row, one chunk) is its normalised output and the log2 of
// its sum of exponentials, and finish_kernel adds them up with weights 2^(lse_part - lse).
#include "kv_attend_device.cuh"

namespace kvt {
namespace {

// 16 bytes to shared memory, zeros if !there
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
constexpr int kTile = 64;   // tokens of a tile

// Rows of up to 256 elements.  kM x kN warps: kM share out the rows (16 each), kN the tokens of a tile
// (each then has its own maximum, sum and output, joined at the end).  K and V tiles of 64 tokens go through
// shared memory in kStages stages filled by cp.async, 16-byte chunks of a row exchanged by row & 7, which
// keeps ldmatrix free of bank conflicts.  Tokens that are not there are zeros in both tiles and -inf in the
// scores, so nothing of what lies in such places reaches a sum.
// What comes here: rows of other than 64 or 128 elements, blocks of other than 16 n tokens (and blocks that no tile is made of, by
// 33 rows or more).  64 runs of up to 1,500 tokens: heads of 96, 4 rows, 78 us (0.35 of the bytes' time); heads of 256, 4 rows, 110 us (0.33);
// blocks of 8 tokens 81 us (0.45).  Where many rows read a block, the products bound it: a prefix of 8,000 tokens by 256 rows a head of 256
// 159 us, by blocks of 8 173 us (0.08 of the bytes' time).
template <typename T, int D, int kM, int kN, int kStages>
__global__ void __launch_bounds__(kM * kN * 32) rows_kernel(const __grid_constant__ AttendArgs a, uint32_t first_kind_items) {
  constexpr int kWarps = kM * kN, kThreadsHere = kWarps * 32;
  constexpr int kTok = kTile / kN;          // tokens of a warp in a tile
  constexpr int kRowBytes = D * 2;
  constexpr int kTileBytes = kTile * kRowBytes;
  constexpr bool kQRegs = D <= 128;
  extern __shared__ __align__(128) uint8_t smem[];
  uint8_t* const kv = smem;                                    // [stages][K, V][64][D]
  uint8_t* const q_s = smem + kStages * 2 * kTileBytes;        // [16 kM][D]
  uint32_t* const chunk_s = reinterpret_cast<uint32_t*>(q_s + kM * 16 * kRowBytes);   // chunk of each block
  wait_for_kernel_ahead();

  Item w;
  const bool second = blockIdx.x >= first_kind_items;
  if (!item_of(a, second ? kKindSuffix : kKindPrefix, second ? blockIdx.x - first_kind_items : blockIdx.x, kM * 16, w,
               threadIdx.x == 0))
    return;
  if (w.to == 0) {
    put_nothing<T>(a, w, threadIdx.x, blockDim.x);
    return;
  }
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int wm = warp / kN, wn = warp % kN;
  const TableView& tv = a.tv;
  const uint32_t block0 = tv.by_tokens(w.from), blocks = tv.by_tokens(w.to - 1u) + 1u - block0;
  for (uint32_t b = threadIdx.x; b < blocks; b += kThreadsHere) chunk_s[b] = tv.chunk((uint64_t)w.seg.row + block0 + b, w.head);

  // queries: rows that are not there and dimensions beyond the head's are zeros
  for (uint32_t i = threadIdx.x; i < kM * 16 * (D / 8); i += kThreadsHere) {
    const uint32_t r = i / (D / 8), c = i % (D / 8);
    uint4 v = make_uint4(0, 0, 0, 0);
    if (r < w.rows && c * 8u < a.dk) {
      uint32_t seq, head;
      row_of(a, w, r, seq, head);
      v = load8(static_cast<const T*>(a.q) + (int64_t)seq * a.q_seq + (int64_t)head * a.q_head + c * 8u);
    }
    *reinterpret_cast<uint4*>(q_s + r * kRowBytes + ((c ^ (r & 7u)) * 16u)) = v;
  }
  __syncthreads();

  const uint32_t tiles = (w.to - w.from + kTile - 1u) / kTile;
  // tile `t` into stage t % kStages
  auto fetch = [&](uint32_t t) {
    uint8_t* const k_dst = kv + (t % kStages) * 2 * kTileBytes;
#pragma unroll 4
    for (uint32_t i = threadIdx.x; i < kTile * (D / 8); i += kThreadsHere) {
      const uint32_t tok = i / (D / 8), c = i % (D / 8);
      const uint32_t at = w.from + t * kTile + tok, b = tv.by_tokens(at);
      const uint32_t ch = at < w.to ? chunk_s[b - block0] : ~0u;
      const bool there = ch != ~0u && c * 8u < a.dk;
      const uint8_t* src = tv.slab;
      if (there) src += (uint64_t)ch * tv.chunk_bytes + ((at - b * tv.block_tokens) * a.dk + c * 8u) * 2u;
      const uint32_t off = tok * kRowBytes + ((c ^ (tok & 7u)) * 16u);
      copy16(smem_address(k_dst + off), src, there);
      copy16(smem_address(k_dst + kTileBytes + off), there ? src + (uint64_t)tv.heads * tv.chunk_bytes : src, there);
    }
  };
#pragma unroll
  for (int t = 0; t < kStages - 1; ++t) {
    if ((uint32_t)t < tiles) fetch(t);
    copy_commit();
  }
  const uint32_t q_row = wm * 16 + (lane & 7) + (lane >> 3 & 1) * 8;
  const uint32_t q_base = smem_address(q_s + q_row * kRowBytes);
  uint32_t qf[kQRegs ? D / 16 : 1][4];
  if (kQRegs) {
#pragma unroll
    for (int k = 0; k < (kQRegs ? D / 16 : 1); ++k) ldmatrix4(qf[k], q_base + (((2 * k + (lane >> 4)) ^ (q_row & 7)) * 16));
  }
  float o[D / 8][4];
#pragma unroll
  for (int j = 0; j < D / 8; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[j][e] = 0.0f;
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};

  for (uint32_t t = 0; t < tiles; ++t) {
    copy_wait<kStages - 2>();
    __syncthreads();   // tile t is there for every warp, and every warp is done with tile t - 1
    if (t + kStages - 1 < tiles) fetch(t + kStages - 1);
    copy_commit();
    const uint8_t* const kt = kv + (t % kStages) * 2 * kTileBytes;
    const uint8_t* const vt = kt + kTileBytes;
    // scores of the warp's tokens
    float s[kTok / 8][4];
#pragma unroll
    for (int j = 0; j < kTok / 8; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[j][e] = 0.0f;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      uint32_t qk[4];
      if (kQRegs) {
#pragma unroll
        for (int e = 0; e < 4; ++e) qk[e] = qf[kQRegs ? k : 0][e];
      } else {
        ldmatrix4(qk, q_base + (((2 * k + (lane >> 4)) ^ (q_row & 7)) * 16));
      }
#pragma unroll
      for (int j = 0; j < kTok / 16; ++j) {
        const uint32_t tok = wn * kTok + j * 16 + (lane >> 4) * 8 + (lane & 7);
        uint32_t b[4];
        ldmatrix4(b, smem_address(kt + tok * kRowBytes) + (((2 * k + (lane >> 3 & 1)) ^ (tok & 7)) * 16));
        mma<T>(s[2 * j], qk, b[0], b[1]);
        mma<T>(s[2 * j + 1], qk, b[2], b[3]);
      }
    }
    // tokens that are not there
    const uint32_t tok0 = w.from + t * kTile + wn * kTok;
    bool all = tok0 + kTok <= w.to;
    if (all) {
      const uint32_t b1 = tv.by_tokens(tok0 + kTok - 1u) - block0;
      for (uint32_t b = tv.by_tokens(tok0) - block0; b <= b1; ++b) all = all && chunk_s[b] != ~0u;
    }
    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int j = 0; j < kTok / 8; ++j) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s[j][e] *= a.scale2;
      if (!all) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t at = tok0 + j * 8 + (lane & 3) * 2 + e;
          if (at >= w.to || chunk_s[tv.by_tokens(at) - block0] == ~0u) s[j][e] = s[j][e + 2] = -INFINITY;
        }
      }
      top[0] = fmaxf(top[0], fmaxf(s[j][0], s[j][1]));
      top[1] = fmaxf(top[1], fmaxf(s[j][2], s[j][3]));
    }
    float base[2], turn[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const float mx = fmaxf(m[r], quad_max(top[r]));
      base[r] = mx == -INFINITY ? 0.0f : mx;     // nothing there so far
      turn[r] = exp2_(m[r] - base[r]);
      m[r] = mx;
      l[r] *= turn[r];
    }
#pragma unroll
    for (int j = 0; j < D / 8; ++j) {
      o[j][0] *= turn[0];
      o[j][1] *= turn[0];
      o[j][2] *= turn[1];
      o[j][3] *= turn[1];
    }
    if (a.weight && a.grain_tokens == 1u) {
#pragma unroll
      for (int j = 0; j < kTok / 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t at = tok0 + j * 8 + (lane & 3) * 2 + (e & 1), r = wm * 16 + lane / 4 + (e >> 1) * 8;
          if (at < w.to && r < w.rows) grain_at(a, w, at)[r] = s[j][e];
        }
    }
#pragma unroll
    for (int j = 0; j < kTok / 16; ++j) {
      float part[2] = {0.0f, 0.0f};
#pragma unroll
      for (int i = 2 * j; i < 2 * j + 2; ++i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][e] = exp2_(s[i][e] - base[e >> 1]);
        part[0] += s[i][0] + s[i][1];
        part[1] += s[i][2] + s[i][3];
      }
      l[0] += part[0];
      l[1] += part[1];
      if (a.weight && a.grain_tokens == 16u && tok0 + j * 16 < w.to) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float sum = quad_sum(part[h]);
          const uint32_t r = wm * 16 + lane / 4 + h * 8;
          if ((lane & 3) == 0 && r < w.rows) grain_at(a, w, (tok0 + j * 16) / 16u)[r] = base[h] + log2_(sum);
        }
      }
      const uint32_t p[4] = {pack2<T>(s[2 * j][0], s[2 * j][1]), pack2<T>(s[2 * j][2], s[2 * j][3]),
                             pack2<T>(s[2 * j + 1][0], s[2 * j + 1][1]), pack2<T>(s[2 * j + 1][2], s[2 * j + 1][3])};
      const uint32_t tok = wn * kTok + j * 16 + (lane >> 3 & 1) * 8 + (lane & 7);
      const uint32_t v_base = smem_address(vt + tok * kRowBytes);
#pragma unroll
      for (int d = 0; d < D / 16; ++d) {
        uint32_t b[4];
        ldmatrix4t(b, v_base + (((2 * d + (lane >> 4)) ^ (tok & 7)) * 16));
        mma<T>(o[2 * d], p, b[0], b[1]);
        mma<T>(o[2 * d + 1], p, b[2], b[3]);
      }
    }
  }
  l[0] = quad_sum(l[0]);
  l[1] = quad_sum(l[1]);
  const uint32_t part = part_of(a, w);
  if (kN == 1) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t r = wm * 16 + lane / 4 + h * 8;
      if (r >= w.rows) continue;
      uint32_t seq, head;
      row_of(a, w, r, seq, head);
      const float inv = l[h] != 0.0f ? 1.0f / l[h] : 0.0f;
#pragma unroll
      for (int j = 0; j < D / 8; ++j) {
        const uint32_t d = j * 8 + (lane & 3) * 2;
        if (d < a.dv) put2<T>(a, seq, head, part, d, o[j][2 * h] * inv, o[j][2 * h + 1] * inv);
      }
      if ((lane & 3) == 0) put_lse(a, seq, head, part, l[h] != 0.0f ? m[h] + log2_(l[h]) : -INFINITY);
    }
    return;
  }
  copy_wait<0>();
  __syncthreads();
  join_warps<D, kM, kN>(smem, wm, wn, o, m, l);
  put_joined<T, D, kM, kN>(a, w, part, smem);
}

// MLA: one row per token is key (all dk elements) and value (the first dv) of every query head.  kM x kN warps:
// kM share out the rows; for the scores kN share out the tokens of a tile, for the output its columns, so that a
// warp's share of the 512 columns fits its registers.  Between the two the probabilities pass through shared memory.
// What comes here: up to 32 query heads a block, and rows of other than 512 + 64 elements.  A tile has 64 rows, filled or not: 64 runs of up to
// 4,000 tokens by 16 heads take 229 us, 0.12 of the bytes' time.
template <typename T, int kM, int kN>
struct Latent {
  static constexpr int D = 576, V = 512, kTok = kTile / kN, kCols = V / kN, kStages = 2;
  static constexpr int kRowBytes = D * 2, kTileBytes = kTile * kRowBytes, kRows = kM * 16;
  static constexpr size_t kSmem = kStages * kTileBytes + kRows * kRowBytes + kRows * kTile * 2 + 2 * kN * kRows * 4 + (kMaxChunkBlocks + 2) * 4;
};

template <typename T, int kM, int kN>
__global__ void __launch_bounds__(kM * kN * 32) latent_kernel(const __grid_constant__ AttendArgs a, uint32_t first_kind_items) {
  using L = Latent<T, kM, kN>;
  constexpr int kThreadsHere = kM * kN * 32, kRowBytes = L::kRowBytes, kRows = L::kRows, kTok = L::kTok, kCols = L::kCols;
  extern __shared__ __align__(128) uint8_t smem[];
  uint8_t* const kv = smem;
  uint8_t* const q_s = kv + L::kStages * L::kTileBytes;                       // [rows][576]
  uint8_t* const p_s = q_s + kRows * kRowBytes;                               // [rows][64]
  float* const top_s = reinterpret_cast<float*>(p_s + kRows * kTile * 2);     // [kN][rows]
  float* const sum_s = top_s + kN * kRows;                                    // [kN][rows]
  uint32_t* const chunk_s = reinterpret_cast<uint32_t*>(sum_s + kN * kRows);
  wait_for_kernel_ahead();
  Item w;
  const bool second = blockIdx.x >= first_kind_items;
  if (!item_of(a, second ? kKindSuffix : kKindPrefix, second ? blockIdx.x - first_kind_items : blockIdx.x, kRows, w, threadIdx.x == 0))
    return;
  if (w.to == 0) {
    put_nothing<T>(a, w, threadIdx.x, blockDim.x);
    return;
  }
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int wm = warp / kN, wn = warp % kN;
  const TableView& tv = a.tv;
  const uint32_t block0 = tv.by_tokens(w.from), blocks = tv.by_tokens(w.to - 1u) + 1u - block0;
  for (uint32_t b = threadIdx.x; b < blocks; b += kThreadsHere) chunk_s[b] = tv.chunk((uint64_t)w.seg.row + block0 + b, w.head);
  for (uint32_t i = threadIdx.x; i < kRows * (L::D / 8); i += kThreadsHere) {
    const uint32_t r = i / (L::D / 8), c = i % (L::D / 8);
    uint4 v = make_uint4(0, 0, 0, 0);
    if (r < w.rows && c * 8u < a.dk) {
      uint32_t seq, head;
      row_of(a, w, r, seq, head);
      v = load8(static_cast<const T*>(a.q) + (int64_t)seq * a.q_seq + (int64_t)head * a.q_head + c * 8u);
    }
    *reinterpret_cast<uint4*>(q_s + r * kRowBytes + ((c ^ (r & 7u)) * 16u)) = v;
  }
  __syncthreads();
  const uint32_t tiles = (w.to - w.from + kTile - 1u) / kTile;
  auto fetch = [&](uint32_t t) {
    uint8_t* const dst = kv + (t % L::kStages) * L::kTileBytes;
#pragma unroll 4
    for (uint32_t i = threadIdx.x; i < kTile * (L::D / 8); i += kThreadsHere) {
      const uint32_t tok = i / (L::D / 8), c = i % (L::D / 8);
      const uint32_t at = w.from + t * kTile + tok, b = tv.by_tokens(at);
      const uint32_t ch = at < w.to ? chunk_s[b - block0] : ~0u;
      const bool there = ch != ~0u && c * 8u < a.dk;
      const uint8_t* src = tv.slab;
      if (there) src += (uint64_t)ch * tv.chunk_bytes + ((at - b * tv.block_tokens) * a.dk + c * 8u) * 2u;
      copy16(smem_address(dst + tok * kRowBytes + ((c ^ (tok & 7u)) * 16u)), src, there);
    }
  };
  fetch(0);
  copy_commit();
  const uint32_t a_row = wm * 16 + (lane & 7) + (lane >> 3 & 1) * 8;
  const uint32_t q_base = smem_address(q_s + a_row * kRowBytes), p_base = smem_address(p_s + a_row * kTile * 2);
  float o[kCols / 8][4];
#pragma unroll
  for (int j = 0; j < kCols / 8; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[j][e] = 0.0f;
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};

  for (uint32_t t = 0; t < tiles; ++t) {
    copy_wait<0>();
    __syncthreads();
    if (t + 1 < tiles) fetch(t + 1);
    copy_commit();
    const uint8_t* const kt = kv + (t % L::kStages) * L::kTileBytes;
    float s[kTok / 8][4];
#pragma unroll
    for (int j = 0; j < kTok / 8; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[j][e] = 0.0f;
    const int steps = (a.dk + 15) / 16;
#pragma unroll 4
    for (int k = 0; k < steps; ++k) {
      uint32_t qk[4];
      ldmatrix4(qk, q_base + (((2 * k + (lane >> 4)) ^ (a_row & 7)) * 16));
#pragma unroll
      for (int j = 0; j < kTok / 16; ++j) {
        const uint32_t tok = wn * kTok + j * 16 + (lane >> 4) * 8 + (lane & 7);
        uint32_t b[4];
        ldmatrix4(b, smem_address(kt + tok * kRowBytes) + (((2 * k + (lane >> 3 & 1)) ^ (tok & 7)) * 16));
        mma<T>(s[2 * j], qk, b[0], b[1]);
        mma<T>(s[2 * j + 1], qk, b[2], b[3]);
      }
    }
    const uint32_t tok0 = w.from + t * kTile + wn * kTok;
    bool all = tok0 + kTok <= w.to;
    if (all) {
      const uint32_t b1 = tv.by_tokens(tok0 + kTok - 1u) - block0;
      for (uint32_t b = tv.by_tokens(tok0) - block0; b <= b1; ++b) all = all && chunk_s[b] != ~0u;
    }
    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int j = 0; j < kTok / 8; ++j) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s[j][e] *= a.scale2;
      if (!all) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t at = tok0 + j * 8 + (lane & 3) * 2 + e;
          if (at >= w.to || chunk_s[tv.by_tokens(at) - block0] == ~0u) s[j][e] = s[j][e + 2] = -INFINITY;
        }
      }
      top[0] = fmaxf(top[0], fmaxf(s[j][0], s[j][1]));
      top[1] = fmaxf(top[1], fmaxf(s[j][2], s[j][3]));
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      top[h] = quad_max(top[h]);
      if ((lane & 3) == 0) top_s[wn * kRows + wm * 16 + lane / 4 + h * 8] = top[h];
    }
    __syncthreads();
    float base[2], turn[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float mx = m[h];
#pragma unroll
      for (int n = 0; n < kN; ++n) mx = fmaxf(mx, top_s[n * kRows + wm * 16 + lane / 4 + h * 8]);
      base[h] = mx == -INFINITY ? 0.0f : mx;
      turn[h] = exp2_(m[h] - base[h]);
      m[h] = mx;
      l[h] *= turn[h];
    }
    if (a.weight && a.grain_tokens == 1u) {
#pragma unroll
      for (int j = 0; j < kTok / 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t at = tok0 + j * 8 + (lane & 3) * 2 + (e & 1), r = wm * 16 + lane / 4 + (e >> 1) * 8;
          if (at < w.to && r < w.rows) grain_at(a, w, at)[r] = s[j][e];
        }
    }
#pragma unroll
    for (int j = 0; j < kTok / 16; ++j) {
      float part[2] = {0.0f, 0.0f};
#pragma unroll
      for (int i = 2 * j; i < 2 * j + 2; ++i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][e] = exp2_(s[i][e] - base[e >> 1]);
        part[0] += s[i][0] + s[i][1];
        part[1] += s[i][2] + s[i][3];
        // 16-byte chunks of a row's 128 bytes are exchanged by row & 7, as in the tiles
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t r = wm * 16 + lane / 4 + h * 8, c = (wn * kTok + i * 8) / 8;
          *reinterpret_cast<uint32_t*>(p_s + r * kTile * 2 + ((c ^ (r & 7u)) * 16u) + (lane & 3) * 4) = pack2<T>(s[i][2 * h], s[i][2 * h + 1]);
        }
      }
      l[0] += part[0];
      l[1] += part[1];
      if (a.weight && a.grain_tokens == 16u && tok0 + j * 16 < w.to) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float sum = quad_sum(part[h]);
          const uint32_t r = wm * 16 + lane / 4 + h * 8;
          if ((lane & 3) == 0 && r < w.rows) grain_at(a, w, (tok0 + j * 16) / 16u)[r] = base[h] + log2_(sum);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < kCols / 8; ++j) {
      o[j][0] *= turn[0];
      o[j][1] *= turn[0];
      o[j][2] *= turn[1];
      o[j][3] *= turn[1];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kTile / 16; ++k) {
      uint32_t p[4];
      ldmatrix4(p, p_base + (((2 * k + (lane >> 4)) ^ (a_row & 7)) * 16));
      const uint32_t tok = k * 16 + (lane >> 3 & 1) * 8 + (lane & 7);
      const uint32_t v_base = smem_address(kt + tok * kRowBytes);
#pragma unroll
      for (int d = 0; d < kCols / 16; ++d) {
        uint32_t b[4];
        ldmatrix4t(b, v_base + (((wn * (kCols / 8) + 2 * d + (lane >> 4)) ^ (tok & 7)) * 16));
        mma<T>(o[2 * d], p, b[0], b[1]);
        mma<T>(o[2 * d + 1], p, b[2], b[3]);
      }
    }
  }
  // the sums of the kN warps' tokens
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    l[h] = quad_sum(l[h]);
    if ((lane & 3) == 0) sum_s[wn * kRows + wm * 16 + lane / 4 + h * 8] = l[h];
  }
  __syncthreads();
  const uint32_t part = part_of(a, w);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t r = wm * 16 + lane / 4 + h * 8;
    if (r >= w.rows) continue;
    float sum = 0.0f;
#pragma unroll
    for (int n = 0; n < kN; ++n) sum += sum_s[n * kRows + r];
    const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
    uint32_t seq, head;
    row_of(a, w, r, seq, head);
#pragma unroll
    for (int j = 0; j < kCols / 8; ++j) {
      const uint32_t d = wn * kCols + j * 8 + (lane & 3) * 2;
      if (d < a.dv) put2<T>(a, seq, head, part, d, o[j][2 * h] * inv, o[j][2 * h + 1] * inv);
    }
    if (wn == 0 && (lane & 3) == 0) put_lse(a, seq, head, part, sum != 0.0f ? m[h] + log2_(sum) : -INFINITY);
  }
}

// ---- parts to outputs, grains to weights -------------------------------------------------------------

constexpr int kFinishRows = kFinishThreads / 32;

// The parts of a sequence: np of its group's prefix, ns of its suffix, the latter behind the places of all prefix chunks.
struct Parts {
  uint32_t np, ns, suffix_at;
  __device__ __forceinline__ uint32_t place(uint32_t i) const { return i < np ? i : suffix_at + i - np; }
};
__device__ __forceinline__ Parts parts_of(const AttendArgs& a, uint32_t seq, uint32_t group) {
  Parts p{0, 0, a.chunks[0] * a.per_chunk[0]};
  const Segment sfx = a.checked(a.suffix, seq, a.max_suffix, false);
  if (group != ~0u)
    p.np = (a.checked(a.prefix, group, a.max_prefix, false).tokens + a.chunk_tokens[0] - 1u) / a.chunk_tokens[0] * a.per_chunk[0];
  p.ns = (sfx.tokens + a.chunk_tokens[1] - 1u) / a.chunk_tokens[1] * a.per_chunk[1];
  return p;
}
// The group of a sequence (or ~0u), asked by a whole warp.
__device__ __forceinline__ uint32_t group_of_warp(const AttendArgs& a, uint32_t seq) {
  if (a.n_groups >= 32u) return a.group_of(seq);
  if (!a.n_groups) return ~0u;
  const uint32_t lane = threadIdx.x % 32u, start = lane <= a.n_groups ? a.group_start[lane] : ~0u;
  const uint32_t g = __popc(__ballot_sync(~0u, lane < a.n_groups && start <= seq)) - 1u;   // the last group that starts at or before it
  const uint32_t lo = __shfl_sync(~0u, start, g & 31u), hi = __shfl_sync(~0u, start, (g + 1u) & 31u);
  return g != ~0u && lo <= seq && seq < hi && hi <= a.n_seqs && hi - lo <= a.max_members ? g : ~0u;
}

// out and lse of rows (sequence, query head), a warp for each.
template <typename T>
__device__ __forceinline__ void join_rows(const AttendArgs& a, uint64_t row) {
  const uint32_t lane = threadIdx.x % 32;
  if (row >= (uint64_t)a.n_seqs * a.q_heads) {
    wait_for_kernel_ahead();
    return;
  }
  const uint32_t seq = (uint32_t)(row / a.q_heads), head = (uint32_t)(row - (uint64_t)seq * a.q_heads);
  const Parts parts = parts_of(a, seq, group_of_warp(a, seq));
  const uint32_t n = parts.np + parts.ns;
  wait_for_kernel_ahead();      // (what is read above was there before the call's first kernel began)
  const float* const lse = a.part_lse + row * a.n_parts;
  const float first = lane < n ? lse[parts.place(lane)] : -INFINITY;
  float top = first;
  for (uint32_t i = lane + 32u; i < n; i += 32u) top = fmaxf(top, lse[parts.place(i)]);
#pragma unroll
  for (int d = 16; d; d /= 2) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
  const float base = top == -INFINITY ? 0.0f : top;
  float sum = exp2_(first - base);
  for (uint32_t i = lane + 32u; i < n; i += 32u) sum += exp2_(lse[parts.place(i)] - base);
#pragma unroll
  for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(~0u, sum, d);
  const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
  if (lane == 0) {
    const float total = sum != 0.0f ? base + log2_(sum) : -INFINITY;
    if (a.lse) a.lse[row] = total * 0.69314718055994530942f;
    if (a.weight) a.total[row] = total;
  }
  T* const out = static_cast<T*>(a.out) + (int64_t)seq * a.out_seq + (int64_t)head * a.out_head;
  const bool wide = (reinterpret_cast<uintptr_t>(out) & 7u) == 0;
  for (uint32_t d0 = 0; d0 < a.dv; d0 += 128u) {      // four neighbouring elements a lane
    const uint32_t d = d0 + lane * 4u;
    float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (uint32_t i0 = 0; i0 < n; i0 += 32u) {
      const float mine = i0 == 0 ? first : (i0 + lane < n ? lse[parts.place(i0 + lane)] : -INFINITY);
      const float share = exp2_(mine - base) * inv;
      const uint32_t most = min(32u, n - i0);
      for (uint32_t i = 0; i < most; i += 8u) {
        float4 v[8];
        float c[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          c[k] = __shfl_sync(~0u, share, (i + k) & 31u);
          const bool some = __shfl_sync(~0u, mine, (i + k) & 31u) != -INFINITY && i + k < most;   // (a part of nothing has not been written)
          v[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          if (some && d < a.dv) v[k] = *reinterpret_cast<const float4*>(a.part_o + (row * a.n_parts + parts.place(i0 + i + k)) * a.dv + d);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          x.x = __fmaf_rn(c[k], v[k].x, x.x);
          x.y = __fmaf_rn(c[k], v[k].y, x.y);
          x.z = __fmaf_rn(c[k], v[k].z, x.z);
          x.w = __fmaf_rn(c[k], v[k].w, x.w);
        }
      }
    }
    if (d >= a.dv) continue;
    if (wide) {
      *reinterpret_cast<uint2*>(out + d) = make_uint2(pack2<T>(x.x, x.y), pack2<T>(x.z, x.w));
    } else {
      out[d] = narrow<T>(x.x);
      out[d + 1] = narrow<T>(x.y);
      out[d + 2] = narrow<T>(x.z);
      out[d + 3] = narrow<T>(x.w);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kFinishThreads) finish_kernel(const __grid_constant__ AttendArgs a) {
  join_rows<T>(a, (uint64_t)blockIdx.x * kFinishRows + threadIdx.x / 32);
}

// Weight of the blocks of prefixes (the first prefix_ctas CTAs) and suffixes: the sum over a block's rows of what the kernels have
// left for its grains, taken from the rows' sums; 2^shift threads for a block and kWeightRows of its rows.
__global__ void __launch_bounds__(kFinishThreads) weight_kernel(const __grid_constant__ AttendArgs a, uint32_t prefix_ctas, uint32_t prefix_shift,
                                                               uint32_t suffix_shift) {
  const int kind = blockIdx.x < prefix_ctas ? kKindPrefix : kKindSuffix;
  const uint32_t shift = kind == kKindPrefix ? prefix_shift : suffix_shift, lanes = 1u << shift;
  // (fewer than 2^32 items, kMaxWeightItems: 64-bit divisions were most of this kernel's time)
  const uint32_t item = (blockIdx.x - (kind == kKindPrefix ? 0u : prefix_ctas)) * (kFinishThreads >> shift) + (threadIdx.x >> shift);
  const uint32_t lane = threadIdx.x & (lanes - 1u);
  const uint32_t most_blocks = ((kind == kKindPrefix ? a.max_prefix : a.max_suffix) + a.tv.block_tokens - 1u) / a.tv.block_tokens;
  const uint32_t most_rows = kind == kKindPrefix ? a.max_members * a.group : a.group, shares = (most_rows + kWeightRows - 1u) / kWeightRows;
  const uint32_t sb = item / shares, sh = sb / most_blocks, index = sh / a.tv.heads;
  const uint32_t row0 = (item - sb * shares) * kWeightRows, b = sb - sh * most_blocks, head = sh - index * a.tv.heads;
  unsigned long long w = 0;
  uint32_t handle = KV_NONE;
  if (index < (kind == kKindPrefix ? a.n_groups : a.n_seqs)) {
    uint32_t seq0 = index, rows = a.group, stride = a.group;
    Segment seg;
    if (kind == kKindPrefix) {
      uint32_t lo, hi;
      a.members(index, lo, hi, false);
      seq0 = lo;
      rows = (hi - lo) * a.group;
      stride = a.max_members * a.group;
      seg = a.checked(a.prefix, index, a.max_prefix, false);
    } else {
      seg = a.checked(a.suffix, index, a.max_suffix, false);
    }
    const uint32_t from = b * a.tv.block_tokens;
    const uint64_t at = (uint64_t)seg.row + b;
    rows = min(rows, row0 + kWeightRows);
    const bool there = from < seg.tokens && row0 < rows && a.tv.chunk(at, head) != ~0u;
    if (there) handle = a.tv.table[(at * a.tv.layers + a.tv.layer) * a.tv.heads + head];
    wait_for_kernel_ahead();      // (what is read above was there before the call's first kernel began)
    if (there) {
      const uint32_t to = min(seg.tokens, from + a.tv.block_tokens);
      const uint32_t g0 = from / a.grain_tokens, g1 = (to + a.grain_tokens - 1u) / a.grain_tokens;
      const float* const total = a.direct ? a.part_lse : a.total;
      const float* const grain = a.grain[kind] + (uint64_t)sh * a.grains[kind] * stride;
      float sum = 0.0f;
#pragma unroll 4
      for (uint32_t r = row0 + lane; r < rows; r += lanes) {
        const uint32_t member = a.by_group(r);
        const float lse = total[(uint64_t)(seq0 + member) * a.q_heads + head * a.group + (r - member * a.group)];
        if (!(fabsf(lse) < INFINITY)) continue;      // a row with nothing to attend to, or whose scores are no numbers: the others count
        for (uint32_t g = g0; g < g1; ++g) sum += exp2_(grain[(uint64_t)g * stride + r] - lse);
      }
      w = __float2ull_rn(fminf(sum * 0x1p32f, 0x1p62f));      // in units of 2^-32
    }
  } else {
    wait_for_kernel_ahead();
  }
  for (uint32_t d = lanes / 2u; d; d /= 2u) w += __shfl_xor_sync(~0u, w, d);
  if (lane == 0 && w) atomicAdd(a.weight + handle, w);
}

// ---- launches ---------------------------------------------------------------------------------------

template <typename F>
cudaError_t launch_items(F* kernel, unsigned threads, size_t smem, const AttendArgs& a, uint32_t row_tile_prefix,
                         uint32_t row_tile_suffix, bool prefix, bool suffix, cudaStream_t s) {
  const uint64_t rows = (uint64_t)a.max_members * a.group;
  const uint64_t np = prefix ? (rows + row_tile_prefix - 1) / row_tile_prefix * a.chunks[0] * a.tv.heads * a.n_groups : 0;
  const uint64_t ns = suffix ? (a.group + row_tile_suffix - 1) / row_tile_suffix * (uint64_t)a.chunks[1] * a.tv.heads * a.n_seqs : 0;
  if (np + ns == 0) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  return launch_overlapped_smem(kernel, (unsigned)(np + ns), threads, smem, s, a, (uint32_t)np);
}

template <typename T, int D, int kM, int kN>
cudaError_t launch_rows(const AttendArgs& a, bool prefix, bool suffix, cudaStream_t s) {
  constexpr int kStages = D <= 64 ? 4 : (D <= 128 ? 3 : 2);
  constexpr size_t tiles = (size_t)kStages * 2 * kTile * D * 2;
  constexpr size_t join = kN > 1 ? (size_t)kN * kM * 16 * (D + 2) * 4 : 0;
  static_assert(join <= tiles, "the join of the warps uses the tiles' memory");
  return launch_items(rows_kernel<T, D, kM, kN, kStages>, kM * kN * 32, tiles + kM * 16 * D * 2 + (kMaxChunkBlocks + 2) * 4, a, kM * 16, kM * 16,
                      prefix, suffix, s);
}

template <typename T, int D>
cudaError_t launch_rows_by(const AttendArgs& a, uint32_t rows, bool prefix, bool suffix, cudaStream_t s) {
  if (rows <= 16) return launch_rows<T, D, 1, 4>(a, prefix, suffix, s);
  if (rows <= 32) return launch_rows<T, D, 2, 2>(a, prefix, suffix, s);
  return launch_rows<T, D, 4, 1>(a, prefix, suffix, s);
}

template <typename T>
cudaError_t launch_typed(const AttendArgs& a, int dtype, bool mla, cudaStream_t s) {
  cudaError_t e = cudaSuccess;
  const bool prefix = a.chunks[0] > 0, tp = prefix && a.tiles[0], ts = a.tiles[1];
  const bool sp = prefix && a.stream[0], ss = a.stream[1], rp = prefix && !tp && !sp, rs = !ts && !ss;
  if (tp || ts) e = launch_attend_tiles(a, dtype, mla, tp, ts, s);
  if (e != cudaSuccess) return e;
  if (sp || ss) {
    e = launch_attend_stream(a, dtype, sp, ss, tp || ts, s);
    if (e != cudaSuccess) return e;
  }
  if (mla) {
    using L = Latent<T, 4, 2>;
    if (rp || rs) e = launch_items(latent_kernel<T, 4, 2>, 4 * 2 * 32, L::kSmem, a, L::kRows, L::kRows, rp, rs, s);
  } else if (rp || rs) {
    auto go = [&](uint32_t rows, bool p, bool f) {
      return a.dk <= 64 ? launch_rows_by<T, 64>(a, rows, p, f, s) : a.dk <= 128 ? launch_rows_by<T, 128>(a, rows, p, f, s)
                                                                               : launch_rows_by<T, 256>(a, rows, p, f, s);
    };
    const uint32_t rows = a.max_members * a.group;
    auto size = [](uint32_t r) { return r <= 16 ? 1 : r <= 32 ? 2 : 4; };
    if (rp && (!rs || size(rows) != size(a.group))) {
      e = go(rows, true, false);
      if (e == cudaSuccess && rs) e = go(a.group, false, true);
    } else {
      e = go(a.group, rp, rs);
    }
  }
  if (e != cudaSuccess) return e;
  const uint64_t rows = (uint64_t)a.n_seqs * a.q_heads;
  const uint64_t join = (rows + kFinishRows - 1) / kFinishRows;
  if (!a.direct) {
    e = launch_overlapped(finish_kernel<T>, (unsigned)join, (unsigned)kFinishThreads, s, a);
    if (e != cudaSuccess) return e;
  }
  if (!a.weight) return cudaSuccess;
  uint64_t ctas[2] = {0, 0};
  uint32_t shift[2] = {0, 0};
  for (int kind = prefix ? 0 : 1; kind < 2; ++kind) {
    const uint32_t most = kind == kKindPrefix ? a.max_prefix : a.max_suffix;
    const uint64_t blocks = ((uint64_t)most + a.tv.block_tokens - 1u) / a.tv.block_tokens;
    const uint32_t r = kind == kKindPrefix ? a.max_members * a.group : a.group;
    shift[kind] = weight_shift(r);
    const uint64_t items = (uint64_t)(kind == kKindPrefix ? a.n_groups : a.n_seqs) * a.tv.heads * blocks * ((r + kWeightRows - 1u) / kWeightRows);
    ctas[kind] = ((items << shift[kind]) + kFinishThreads - 1) / kFinishThreads;
  }
  if (ctas[0] + ctas[1] == 0) return cudaSuccess;
  return launch_overlapped(weight_kernel, (unsigned)(ctas[0] + ctas[1]), (unsigned)kFinishThreads, s, a, (uint32_t)ctas[0], shift[0], shift[1]);
}

}  // namespace

cudaError_t launch_attend(const AttendArgs& a, int dtype, bool mla, cudaStream_t s) {
  return dtype == KV_DTYPE_BF16 ? launch_typed<__nv_bfloat16>(a, dtype, mla, s) : launch_typed<__half>(a, dtype, mla, s);
}

}  // namespace kvt
