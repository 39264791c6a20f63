// New tokens enter the cache: rotary positions for their queries and keys, keys and values into
// the pool's blocks (kv_append).
//
// Pair (x_i, x_j) of a head turns by the angle pos[axis(i)] * inv_freq[i]:
//   x_i' = x_i cos - x_j sin,  x_j' = x_j cos + x_i sin     (32 bits, rounded once at the end)
// The angle is formed and reduced to [-pi, pi] in 64 bits: at position 10^6 a 32-bit product would be
// off by 0.03 rad.  A token's angles are shared by all its heads: a warp (or, of few tokens, a CTA) takes a token,
// forms them once in shared memory and streams the heads through registers in 16-byte vectors, the first of which are on
// their way meanwhile.
// Bound: HBM, each element read once and written once: 16,411 tokens of 32 + 8 + 8 heads of 128, 78 us, 0.80 of the copy rate.  Element by
// element, where a vector is not 16-byte aligned: 212 us.
#include "kv_attend_device.cuh"

namespace kvt {
namespace {

constexpr int kAppendThreads = 256;

__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ void from_float(float x, __nv_bfloat16& y) { y = __float2bfloat16_rn(x); }
__device__ __forceinline__ void from_float(float x, __half& y) { y = __float2half_rn(x); }

// Eight elements as four words, or one element.
template <typename T, int V>
struct Vec;
template <typename T>
struct alignas(16) Vec<T, 8> {
  uint32_t x[4];
};
template <typename T>
struct Vec<T, 1> {
  T x[1];
};

// cos and sin of pos * freq, the product rounded to 64 bits and reduced by 2 pi in two parts (the first alone would leave 4e-17 of the
// angle: 8e-5 rad at 2 10^12)
__device__ __forceinline__ float2 turn(int32_t pos, float freq) {
  const double a = __dmul_rn((double)pos, (double)freq);
  const double k = rint(__dmul_rn(a, 0.15915494309189533577));
  const float r = (float)__fma_rn(-k, 2.4492935982947064e-16, __fma_rn(-k, 6.283185307179586477, a));
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
template <typename T>
__device__ __forceinline__ float2 unpack2(uint32_t v);
template <>
__device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
template <>
__device__ __forceinline__ float2 unpack2<__half>(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
// Two pairs at a time: (a.lo, b.lo) and (a.hi, b.hi), or (kInterleaved) (a.lo, a.hi).
template <typename T>
__device__ __forceinline__ void rotate2(uint32_t& a, uint32_t& b, float2 c0, float2 c1) {
  const float2 x = unpack2<T>(a), y = unpack2<T>(b);
  a = pack2<T>(__fmaf_rn(x.x, c0.x, -__fmul_rn(y.x, c0.y)), __fmaf_rn(x.y, c1.x, -__fmul_rn(y.y, c1.y)));
  b = pack2<T>(__fmaf_rn(y.x, c0.x, __fmul_rn(x.x, c0.y)), __fmaf_rn(y.y, c1.x, __fmul_rn(x.y, c1.y)));
}
template <typename T>
__device__ __forceinline__ void rotate_inside(uint32_t& a, float2 c) {
  const float2 x = unpack2<T>(a);
  a = pack2<T>(__fmaf_rn(x.x, c.x, -__fmul_rn(x.y, c.y)), __fmaf_rn(x.y, c.x, __fmul_rn(x.x, c.y)));
}

// How a token's elements are dealt out: a head's in tasks, first the rotated ones -- a vector of first halves and the one of
// their partners, or (interleaved) a vector of whole pairs -- then the others, a vector each; query heads, key heads, values.
struct Tasks {
  uint32_t q, k, v, total, turned, per_head;
  Divisor by_head, by_value;
};

template <typename T, int V>
struct Task {
  Vec<T, V> a, b;
  uint32_t head, at, partner;   // elements; partner ~0u: one vector
  uint32_t pair;                // first pair of a rotated vector, ~0u: copied
};

// kTeam threads work on a token (kTeam < the CTA's threads: a warp), blockIdx.y: on which share of its tasks.
template <typename T, int V, bool kInterleaved, int kTeam>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const __grid_constant__ AppendArgs a, const __grid_constant__ Tasks n) {
  constexpr int kTeams = kAppendThreads / kTeam;
  extern __shared__ float2 shared[];   // for each team: cos and sin of the pairs, then the chunks of the heads
  wait_for_kernel_ahead();
  const TableView& tv = a.tv;
  const uint32_t team = threadIdx.x / kTeam, me = threadIdx.x % kTeam, half = a.rot_dim / 2u;
  const uint64_t t = (uint64_t)blockIdx.x * kTeams + team;
  if (t >= a.n) return;
  float2* const cs = shared + team * half;
  uint32_t* const chunk = reinterpret_cast<uint32_t*>(shared + kTeams * half) + team * tv.heads;
  const int64_t slot = a.slot[t];
  constexpr int kBatch = 2;     // ... and the next ones are while these are turned and stored
  const uint32_t share = (n.total + gridDim.y - 1u) / gridDim.y;
  const uint32_t from = blockIdx.y * share + me, to = min(n.total, (blockIdx.y + 1u) * share);
  auto load = [&](Task<T, V> (&w)[kBatch], uint32_t t0) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      Task<T, V>& k = w[u];
      const uint32_t i = t0 + u * kTeam;
      if (i >= to) continue;
      const T* src;
      k.partner = k.pair = ~0u;
      if (i < n.q + n.k) {
        k.head = n.by_head(i);
        const uint32_t e = i - k.head * n.per_head;
        src = k.head < a.q_heads ? static_cast<const T*>(a.q) + (int64_t)t * a.q_tok + k.head * a.q_head
                                 : static_cast<const T*>(a.k) + (int64_t)t * a.k_tok + (k.head - a.q_heads) * a.k_head;
        if (e < n.turned) {
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
          const uint32_t r = (e - n.turned) * V;
          k.at = r < a.rot_first ? r : r + a.rot_dim;
        }
      } else {
        const uint32_t j = i - n.q - n.k;
        k.head = n.by_value(j);
        src = static_cast<const T*>(a.v) + (int64_t)t * a.v_tok + k.head * a.v_head;
        k.at = (j - k.head * (a.dv / V)) * V;
      }
      k.a = *reinterpret_cast<const Vec<T, V>*>(src + k.at);
      if (k.partner != ~0u) k.b = *reinterpret_cast<const Vec<T, V>*>(src + k.partner);
    }
  };
  Task<T, V> first[kBatch], second[kBatch];
  if (from < to) load(first, from);                     // (on their way while the angles and places are found)
  const bool padding = slot < 0;
  const uint64_t row = padding ? 0 : (uint64_t)slot / tv.block_tokens;
  const uint32_t in_block = (uint32_t)((uint64_t)slot - row * tv.block_tokens);
  const bool beyond = !padding && row >= tv.n_rows;
  if (beyond && me == 0) tv.flag(KV_DEV_BAD_INDEX);
  if (padding || beyond) return;                        // (the whole team)
  for (uint32_t h = me; h < tv.heads; h += kTeam) {
    chunk[h] = tv.chunk(row, h);
    if (chunk[h] == ~0u) tv.flag(KV_DEV_BLOCK_NOT_RESIDENT);
  }
  // (the pairs of one vector lie apart, so that lanes, which have neighbouring vectors, meet no bank conflicts)
  constexpr uint32_t kPairs = V == 1 ? 1u : kInterleaved ? V / 2 : V;
  const uint32_t vecs = half / kPairs;
  for (uint32_t i = me; i < half; i += kTeam) cs[i % kPairs * vecs + i / kPairs] = turn(a.pos[a.axis[i] * a.n + t], a.inv_freq[i]);
  if (kTeam == 32) __syncwarp();
  else __syncthreads();
  auto store = [&](Task<T, V> (&w)[kBatch], uint32_t t0) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      Task<T, V>& k = w[u];
      const uint32_t i = t0 + u * kTeam;
      if (i >= to) continue;
      T* dst;
      if (i < n.q) {
        dst = static_cast<T*>(a.q_out) + (int64_t)t * a.o_tok + k.head * a.o_head;
      } else {
        const bool value = i >= n.q + n.k;
        const uint32_t c = chunk[value ? k.head : k.head - a.q_heads];
        if (c == ~0u) continue;
        dst = reinterpret_cast<T*>(tv.slab + (uint64_t)(value ? c + tv.heads : c) * tv.chunk_bytes) + in_block * (value ? a.dv : a.dk);
      }
      if (k.pair != ~0u) {
        const float2* const turns = cs + k.pair / kPairs;
        if constexpr (V == 1) {
          rotate(k.a.x[0], k.b.x[0], turns[0]);
        } else if constexpr (kInterleaved) {
#pragma unroll
          for (int p = 0; p < 4; ++p) rotate_inside<T>(k.a.x[p], turns[p * vecs]);
        } else {
#pragma unroll
          for (int p = 0; p < 4; ++p) rotate2<T>(k.a.x[p], k.b.x[p], turns[2 * p * vecs], turns[(2 * p + 1) * vecs]);
        }
      }
      *reinterpret_cast<Vec<T, V>*>(dst + k.at) = k.a;
      if (k.partner != ~0u) *reinterpret_cast<Vec<T, V>*>(dst + k.partner) = k.b;
    }
  };
  constexpr uint32_t kStep = kTeam * kBatch;
  for (uint32_t t0 = from; t0 < to; t0 += 2 * kStep) {
    load(second, t0 + kStep);
    store(first, t0);
    load(first, t0 + 2 * kStep);
    store(second, t0 + kStep);
  }
}

template <typename T, int V, bool kInterleaved>
cudaError_t launch(const AppendArgs& a, cudaStream_t s) {
  Tasks n;
  n.turned = kInterleaved && V > 1 ? a.rot_dim / V : a.rot_dim / 2u / V;
  n.per_head = n.turned + (a.dk - a.rot_dim) / V;
  n.q = a.q_heads * n.per_head;
  n.k = a.tv.heads * n.per_head;
  n.v = a.v ? a.tv.heads * (a.dv / V) : 0u;
  n.total = n.q + n.k + n.v;
  n.by_head = Divisor(n.per_head);
  n.by_value = Divisor(a.dv / V ? a.dv / V : 1u);
  // A warp per token where there are enough tokens to fill the SMs with warps and a token is not much work, else a CTA, or
  // several where few tokens have much to do.
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cfg.stream = s;
  cfg.blockDim = dim3(kAppendThreads);
  count_launches(1);
  const size_t per_team = a.rot_dim / 2u * sizeof(float2) + a.tv.heads * sizeof(uint32_t);
  constexpr uint64_t kWarps = kAppendThreads / 32;
  if (a.n >= 148u * 16u && n.total <= 1024u && per_team * kWarps <= 48u * 1024u) {
    cfg.gridDim = dim3((unsigned)((a.n + kWarps - 1) / kWarps));
    cfg.dynamicSmemBytes = per_team * kWarps;
    return cudaLaunchKernelEx(&cfg, append_kernel<T, V, kInterleaved, 32>, a, n);
  }
  const uint64_t most = (n.total + kAppendThreads * 4u - 1u) / (kAppendThreads * 4u), want = a.n < 592u ? 592u / a.n : 1u;
  cfg.gridDim = dim3((unsigned)a.n, (unsigned)(most < want ? (most ? most : 1) : want));
  cfg.dynamicSmemBytes = per_team;
  return cudaLaunchKernelEx(&cfg, append_kernel<T, V, kInterleaved, kAppendThreads>, a, n);
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
