// Eviction score from accumulated attention weight (kv_attention_score).
//
// Weight arrives by handle in fixed point (units of 2^-32, integer atomics: the sum does not depend on
// their order).  Per RESIDENT entry of handle g, once an epoch, in binary32 with each operation rounded
// once:  acc[g] = decay*acc[g] + float(weight[g]) * 2^-32;  weight[g] = 0;  score = acc[g], or +inf while
// the entry is young.  FREE entries get +inf.
// Bound: HBM; 37 bytes an entry, 16 of them gathered by handle (a block's heads have neighbouring
// handles, so a 32-byte sector is mostly used whole).
#include "kv_attend.cuh"

namespace kvt {
namespace {

constexpr int kScoreThreads = 256;

__device__ __forceinline__ float score_entry(uint32_t state, uint32_t tag, uint32_t last, uint32_t epoch, float decay,
                                             uint32_t protect, unsigned long long* weight, float* acc, uint64_t n_tags,
                                             uint32_t* status) {
  if (state != KV_STATE_RESIDENT) return INFINITY;
  if (tag >= n_tags) {
    atomicOr(status, KV_DEV_BAD_INDEX);
    return INFINITY;
  }
  const unsigned long long w = weight[tag];
  const float a = __fadd_rn(__fmul_rn(decay, acc[tag]), __fmul_rn(__ull2float_rn(w), 0x1p-32f));
  acc[tag] = a;
  if (w) weight[tag] = 0ull;
  return (int32_t)(epoch - last) < (int32_t)protect ? INFINITY : a;
}

__global__ void __launch_bounds__(kScoreThreads) attention_score_kernel(EntryState st, uint32_t epoch, float decay,
                                                                        uint32_t protect, unsigned long long* weight,
                                                                        float* acc, uint64_t n_tags, uint32_t* status) {
  wait_for_kernel_ahead();
  const uint64_t i = ((uint64_t)blockIdx.x * kScoreThreads + threadIdx.x) * 4u;
  if (i + 4u <= st.n) {
    const uchar4 s = *reinterpret_cast<const uchar4*>(st.state + i);
    const uint4 t = *reinterpret_cast<const uint4*>(st.tag + i);
    const uint4 l = *reinterpret_cast<const uint4*>(st.last_epoch + i);
    float4 r;
    r.x = score_entry(s.x, t.x, l.x, epoch, decay, protect, weight, acc, n_tags, status);
    r.y = score_entry(s.y, t.y, l.y, epoch, decay, protect, weight, acc, n_tags, status);
    r.z = score_entry(s.z, t.z, l.z, epoch, decay, protect, weight, acc, n_tags, status);
    r.w = score_entry(s.w, t.w, l.w, epoch, decay, protect, weight, acc, n_tags, status);
    *reinterpret_cast<float4*>(st.score + i) = r;
  } else {
    for (uint64_t j = i; j < st.n; ++j)
      st.score[j] = score_entry(st.state[j], st.tag[j], st.last_epoch[j], epoch, decay, protect, weight, acc, n_tags, status);
  }
}

}  // namespace

cudaError_t launch_attention_score(const EntryState& st, uint32_t epoch, float decay, uint32_t protect,
                                   unsigned long long* weight, float* acc, uint64_t n_tags, uint32_t* status,
                                   cudaStream_t s) {
  const uint64_t per_block = kScoreThreads * 4ull;
  return launch_overlapped(attention_score_kernel, (unsigned)((st.n + per_block - 1u) / per_block), (unsigned)kScoreThreads, s,
                           st, epoch, decay, protect, weight, acc, n_tags, status);
}

}  // namespace kvt
