// New tokens enter the cache: rotary positions for their queries and keys, keys and values into
// the pool's blocks (kv_append).
//
// Pair (x_i, x_j) of a head turns by the angle pos[axis(i)] * inv_freq[i]:
//   x_i' = x_i cos - x_j sin,  x_j' = x_j cos + x_i sin     (32 bits, rounded once at the end)
// The angle is formed and reduced to [-pi, pi] in 64 bits: at position 10^6 a 32-bit product would be
// off by 0.03 rad.  A token's angles are shared by all its heads, so a CTA takes a token, forms them
// once in shared memory and then streams the heads through registers in 16-byte vectors.
// Bound: HBM, each element read once and written once.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kv_attend.cuh"

namespace kvt {
namespace {

constexpr int kAppendThreads = 256;

__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ void from_float(float x, __nv_bfloat16& y) { y = __float2bfloat16_rn(x); }
__device__ __forceinline__ void from_float(float x, __half& y) { y = __float2half_rn(x); }

template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
  T x[V];
};

// cos and sin of pos * freq
__device__ __forceinline__ float2 turn(int32_t pos, float freq) {
  const double a = __dmul_rn((double)pos, (double)freq);   // exact: 31 + 24 bits are at most two too many
  const double k = rint(__dmul_rn(a, 0.15915494309189533577));
  const float r = (float)__fma_rn(-k, 6.283185307179586477, a);
  float2 cs;
  sincosf(r, &cs.y, &cs.x);
  return cs;
}

template <typename T>
__device__ __forceinline__ void rotate(T& a, T& b, float2 cs) {
  const float x = to_float(a), y = to_float(b);
  from_float(__fmaf_rn(x, cs.x, -__fmul_rn(y, cs.y)), a);
  from_float(__fmaf_rn(y, cs.x, __fmul_rn(x, cs.y)), b);
}

// A head's elements are dealt out in tasks: first the rotated ones -- a vector of first halves and the
// one of their partners, or (interleaved) a vector of whole pairs -- then the others, a vector each.
template <typename T, int V, bool kInterleaved>
struct Task {
  Vec<T, V> a, b;
  const T* src;
  T* dst;
  uint32_t at, partner;   // elements; partner ~0u: one vector
  uint32_t pair;          // first pair of a rotated vector, ~0u: copied
};

template <typename T, int V, bool kInterleaved>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(AppendArgs a, uint32_t q_tasks, uint32_t k_tasks,
                                                                uint32_t v_tasks, uint32_t turned, uint32_t per_head,
                                                                Divisor by_head, Divisor by_value) {
  __shared__ float2 cs[128];
  extern __shared__ uint32_t chunk[];   // [heads]
  wait_for_kernel_ahead();
  const TableView& tv = a.tv;
  const uint64_t t = blockIdx.x;
  const int64_t slot = a.slot[t];
  if (slot < 0) return;                                           // padding
  const uint64_t row = (uint64_t)slot / tv.block_tokens;
  const uint32_t in_block = (uint32_t)((uint64_t)slot - row * tv.block_tokens);
  if (row >= tv.n_rows) {
    if (threadIdx.x == 0) tv.flag(KV_DEV_BAD_INDEX);
    return;
  }
  for (uint32_t h = threadIdx.x; h < tv.heads; h += kAppendThreads) {
    chunk[h] = tv.chunk(row, h);
    if (chunk[h] == ~0u) tv.flag(KV_DEV_BLOCK_NOT_RESIDENT);
  }
  for (uint32_t i = threadIdx.x; i < a.rot_dim / 2u; i += kAppendThreads)
    cs[i] = turn(a.pos[a.axis[i] * a.n + t], a.inv_freq[i]);
  __syncthreads();
  const uint32_t half = a.rot_dim / 2u;
  const uint32_t total = q_tasks + k_tasks + v_tasks;
  constexpr int kBatch = 4;
  for (uint32_t t0 = threadIdx.x; t0 < total; t0 += kAppendThreads * kBatch) {
    Task<T, V, kInterleaved> w[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      Task<T, V, kInterleaved>& k = w[u];
      const uint32_t i = t0 + u * kAppendThreads;
      k.dst = nullptr;
      if (i >= total) continue;
      if (i < q_tasks + k_tasks) {
        const uint32_t head = by_head(i), e = i - head * per_head;
        if (head < a.q_heads) {
          k.src = static_cast<const T*>(a.q) + (int64_t)t * a.q_tok + head * a.q_head;
          k.dst = static_cast<T*>(a.q_out) + (int64_t)t * a.o_tok + head * a.o_head;
        } else {
          const uint32_t h = head - a.q_heads;
          k.src = static_cast<const T*>(a.k) + (int64_t)t * a.k_tok + h * a.k_head;
          if (chunk[h] == ~0u) continue;
          k.dst = reinterpret_cast<T*>(tv.slab + (uint64_t)chunk[h] * tv.chunk_bytes) + in_block * a.dk;
        }
        k.partner = ~0u;
        k.pair = ~0u;
        if (e < turned) {
          if (kInterleaved) {
            k.pair = V > 1 ? e * (V / 2) : e;
            k.at = a.rot_first + 2u * k.pair;
            if (V == 1) k.partner = k.at + 1u;
          } else {
            k.pair = e * V;
            k.at = a.rot_first + k.pair;
            k.partner = k.at + half;
          }
        } else {
          const uint32_t r = (e - turned) * V;
          k.at = r < a.rot_first ? r : r + a.rot_dim;
        }
      } else {
        const uint32_t j = i - q_tasks - k_tasks, h = by_value(j);
        k.src = static_cast<const T*>(a.v) + (int64_t)t * a.v_tok + h * a.v_head;
        if (chunk[h] == ~0u) continue;
        k.dst = reinterpret_cast<T*>(tv.slab + ((uint64_t)chunk[h] + tv.heads) * tv.chunk_bytes) + in_block * a.dv;
        k.at = (j - h * (a.dv / V)) * V;
        k.partner = k.pair = ~0u;
      }
      k.a = *reinterpret_cast<const Vec<T, V>*>(k.src + k.at);
      if (k.partner != ~0u) k.b = *reinterpret_cast<const Vec<T, V>*>(k.src + k.partner);
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      Task<T, V, kInterleaved>& k = w[u];
      if (!k.dst) continue;
      if (k.pair != ~0u) {
        if (kInterleaved && V > 1) {
#pragma unroll
          for (int p = 0; p < V / 2; ++p) rotate(k.a.x[2 * p], k.a.x[2 * p + 1], cs[k.pair + p]);
        } else {
#pragma unroll
          for (int p = 0; p < V; ++p) rotate(k.a.x[p], k.b.x[p], cs[k.pair + p]);
        }
      }
      *reinterpret_cast<Vec<T, V>*>(k.dst + k.at) = k.a;
      if (k.partner != ~0u) *reinterpret_cast<Vec<T, V>*>(k.dst + k.partner) = k.b;
    }
  }
}

template <typename T, int V, bool kInterleaved>
cudaError_t launch(const AppendArgs& a, cudaStream_t s) {
  const uint32_t turned = kInterleaved && V > 1 ? a.rot_dim / V : a.rot_dim / 2u / V;
  const uint32_t per_head = turned + (a.dk - a.rot_dim) / V;
  const uint32_t v_per_head = a.dv / V;
  return launch_overlapped_smem(append_kernel<T, V, kInterleaved>, (unsigned)a.n, (unsigned)kAppendThreads,
                                a.tv.heads * sizeof(uint32_t), s, a, a.q_heads * per_head, a.tv.heads * per_head,
                                a.v ? a.tv.heads * v_per_head : 0u, turned, per_head, Divisor(per_head),
                                Divisor(v_per_head ? v_per_head : 1u));
}

template <typename T>
cudaError_t launch_typed(const AppendArgs& a, bool wide, cudaStream_t s) {
  if (wide) return a.interleaved ? launch<T, 8, true>(a, s) : launch<T, 8, false>(a, s);
  return a.interleaved ? launch<T, 1, true>(a, s) : launch<T, 1, false>(a, s);
}

}  // namespace

cudaError_t launch_append(const AppendArgs& a, int dtype, bool wide, cudaStream_t s) {
  return dtype == KV_DTYPE_BF16 ? launch_typed<__nv_bfloat16>(a, wide, s) : launch_typed<__half>(a, wide, s);
}

}  // namespace kvt
