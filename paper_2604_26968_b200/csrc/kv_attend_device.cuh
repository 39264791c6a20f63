// Device helpers shared by the kernels of kv_attend: what a CTA works on, and where results go.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kv_attend.cuh"

namespace kvt {

__device__ __forceinline__ uint32_t smem_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ float exp2_(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float log2_(float x) {
  float y;
  asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <>
__device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <typename T>
__device__ __forceinline__ T narrow(float x);
template <>
__device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half narrow<__half>(float x) { return __float2half_rn(x); }

// Eight 16-bit elements, wherever they lie.
__device__ __forceinline__ uint4 load8(const void* src) {
  if ((reinterpret_cast<uintptr_t>(src) & 15u) == 0) return *reinterpret_cast<const uint4*>(src);
  uint32_t e[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) e[k] = reinterpret_cast<const uint16_t*>(src)[k];
  return make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
}

// What a CTA works on: rows [row0, row0 + rows) of a segment and KV head, tokens [from, to) of it.
struct Item {
  Segment seg;
  uint32_t index, head, row0, rows, seq0, from, to, chunk;
  int kind;
};

// Item number i of the launch: kind's segments x heads x chunks x row tiles, row tiles innermost (they
// read the same blocks); or (by_chunk) chunks outermost, the later ones of which are often not there.
// False: there is nothing to do.
template <bool by_chunk = false>
__device__ __forceinline__ bool item_of(const AttendArgs& a, int kind, uint32_t i, uint32_t row_tile, Item& w, bool tell) {
  const uint32_t most = kind == kKindPrefix ? a.max_members * a.group : a.group;
  const uint32_t tiles = (most + row_tile - 1u) / row_tile;
  const uint32_t rt = i % tiles;
  i /= tiles;
  if (by_chunk) {
    const uint32_t segments = (kind == kKindPrefix ? a.n_groups : a.n_seqs) * a.tv.heads;
    w.chunk = i / segments;
    i -= w.chunk * segments;
  } else {
    w.chunk = i % a.chunks[kind];
    i /= a.chunks[kind];
  }
  w.index = i / a.tv.heads;
  w.head = i - w.index * a.tv.heads;
  w.kind = kind;
  if (kind == kKindPrefix) {
    uint32_t lo, hi;
    a.members(w.index, lo, hi, tell);
    w.seq0 = lo;
    w.rows = (hi - lo) * a.group;
    w.seg = a.checked(a.prefix, w.index, a.max_prefix, tell);
  } else {
    w.seq0 = w.index;
    w.rows = a.group;
    w.seg = a.checked(a.suffix, w.index, a.max_suffix, tell);
  }
  w.row0 = rt * row_tile;
  w.from = w.chunk * a.chunk_tokens[kind];
  if (w.row0 >= w.rows || (w.from >= w.seg.tokens && !(a.direct && w.chunk == 0))) return false;
  w.rows = min(w.rows - w.row0, row_tile);
  w.to = min(w.seg.tokens, w.from + a.chunk_tokens[kind]);
  return true;
}

// Row r of an item: its sequence and query head.
__device__ __forceinline__ void row_of(const AttendArgs& a, const Item& w, uint32_t r, uint32_t& seq, uint32_t& head) {
  const uint32_t at = w.row0 + r, member = a.by_group(at);
  seq = w.seq0 + member;
  head = w.head * a.group + (at - member * a.group);
}

// Writes elements [d, d + 2) of a row's part.
template <typename T>
__device__ __forceinline__ void put2(const AttendArgs& a, uint32_t seq, uint32_t head, uint32_t part, uint32_t d, float x, float y) {
  if (a.direct) {
    T* o = static_cast<T*>(a.out) + (int64_t)seq * a.out_seq + (int64_t)head * a.out_head + d;
    o[0] = narrow<T>(x);
    o[1] = narrow<T>(y);
  } else {
    float* o = a.part_o + (((uint64_t)seq * a.q_heads + head) * a.n_parts + part) * a.dv + d;
    *reinterpret_cast<float2*>(o) = make_float2(x, y);
  }
}
__device__ __forceinline__ void put_lse(const AttendArgs& a, uint32_t seq, uint32_t head, uint32_t part, float lse2) {
  const uint64_t row = (uint64_t)seq * a.q_heads + head;
  if (!a.direct || a.weight) a.part_lse[row * a.n_parts + part] = lse2;
  if (a.direct && a.lse) a.lse[row] = lse2 * 0.69314718055994530942f;
}

__device__ __forceinline__ uint32_t part_of(const AttendArgs& a, const Item& w) {
  return w.kind == kKindPrefix ? w.chunk * a.per_chunk[0] : a.chunks[0] * a.per_chunk[0] + w.chunk * a.per_chunk[1];
}

// A sequence without tokens, where no join follows; by `threads` threads.
template <typename T>
__device__ void put_nothing(const AttendArgs& a, const Item& w, uint32_t thread, uint32_t threads) {
  for (uint32_t i = thread; i < w.rows * (a.dv / 2u); i += threads) {
    const uint32_t r = i / (a.dv / 2u), d = i % (a.dv / 2u) * 2u;
    uint32_t seq, head;
    row_of(a, w, r, seq, head);
    put2<T>(a, seq, head, 0, d, 0.0f, 0.0f);
    if (d == 0) put_lse(a, seq, head, 0, -INFINITY);
  }
}

// Where the weight of grain `gr` of the item's segment for its first row goes.
__device__ __forceinline__ float* grain_at(const AttendArgs& a, const Item& w, uint32_t gr) {
  const uint64_t rows = w.kind == kKindPrefix ? (uint64_t)a.max_members * a.group : a.group;
  return a.grain[w.kind] + (((uint64_t)w.index * a.tv.heads + w.head) * a.grains[w.kind] + gr) * rows + w.row0;
}

// ---- products of 16 rows on mma.sync ----

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr));
}
__device__ __forceinline__ void ldmatrix4t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr));
}
template <typename T>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float quad_max(float x) {
  x = fmaxf(x, __shfl_xor_sync(~0u, x, 1));
  return fmaxf(x, __shfl_xor_sync(~0u, x, 2));
}
__device__ __forceinline__ float quad_sum(float x) {
  x += __shfl_xor_sync(~0u, x, 1);
  return x + __shfl_xor_sync(~0u, x, 2);
}

// kN warps that have worked on different tokens for the same 16 kM rows join: maxima and sums, then outputs.  All threads of
// the CTA; memory: kN * 16 kM * (D + 2) floats, which nobody uses any more.
template <int D, int kM, int kN>
__device__ __forceinline__ void join_warps(uint8_t* memory, int wm, int wn, const float (&o)[D / 8][4], const float (&m)[2], const float (&l)[2]) {
  float* const o_s = reinterpret_cast<float*>(memory);                        // [kN][16 kM][D]
  float* const ml_s = o_s + kN * kM * 16 * D;                                 // [kN][16 kM][2]
  const int lane = threadIdx.x % 32;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = wm * 16 + lane / 4 + h * 8;
    if ((lane & 3) == 0) {
      ml_s[(wn * kM * 16 + r) * 2] = m[h];
      ml_s[(wn * kM * 16 + r) * 2 + 1] = l[h];
    }
#pragma unroll
    for (int j = 0; j < D / 8; ++j)
      *reinterpret_cast<float2*>(o_s + (wn * kM * 16 + r) * D + ((j ^ (r & 7)) * 8 + (lane & 3) * 2)) = make_float2(o[j][2 * h], o[j][2 * h + 1]);
  }
}
template <typename T, int D, int kM, int kN>
__device__ __forceinline__ void put_joined(const AttendArgs& a, const Item& w, uint32_t part, const uint8_t* memory) {
  const float* const o_s = reinterpret_cast<const float*>(memory);
  const float* const ml_s = o_s + kN * kM * 16 * D;
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < w.rows * (D / 2); i += blockDim.x) {
    const uint32_t r = i / (D / 2), d = i % (D / 2) * 2u;
    if (d >= a.dv) continue;
    float top = -INFINITY;
#pragma unroll
    for (int n = 0; n < kN; ++n) top = fmaxf(top, ml_s[(n * kM * 16 + r) * 2]);
    const float from = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f, x = 0.0f, y = 0.0f;
#pragma unroll
    for (int n = 0; n < kN; ++n) {
      const float c = exp2_(ml_s[(n * kM * 16 + r) * 2] - from);
      const float2 v = *reinterpret_cast<const float2*>(o_s + (n * kM * 16 + r) * D + (((d / 8u) ^ (r & 7u)) * 8u + d % 8u));
      sum += c * ml_s[(n * kM * 16 + r) * 2 + 1];
      x += c * v.x;
      y += c * v.y;
    }
    const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
    uint32_t seq, head;
    row_of(a, w, r, seq, head);
    put2<T>(a, seq, head, part, d, x * inv, y * inv);
    if (d == 0) put_lse(a, seq, head, part, sum != 0.0f ? top + log2_(sum) : -INFINITY);
  }
}

}  // namespace kvt
