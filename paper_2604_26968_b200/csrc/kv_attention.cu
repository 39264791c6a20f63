// Eviction score from accumulated attention weight (kv_attention_score).
//
// Weight arrives by handle in fixed point (units of 2^-32, integer atomics: the sum does not depend on
// their order).  Per RESIDENT entry of handle g, once an epoch, in binary32 with each operation rounded
// once:  acc[g] = decay*acc[g] + float(weight[g]) * 2^-32;  weight[g] = 0;  score = acc[g], or +inf while
// the entry is young.  FREE entries get +inf.
// Bound: HBM.  Handles go in order, a thread for four of them: block table, weights and accumulators (28 bytes a handle)
// are streamed, and only the score (4 bytes) is reached through the table.  A second launch goes over the entries in order and
// overwrites the scores of those that are FREE or young.  Where no two neighbouring entries have neighbouring handles
// (18.8 M entries): 262 us for both, 310 with weight in every entry and nothing in the L2; entries in order, weights and accumulators reached by handle, 1,186; the last epoch and the
// entry's own handle reached through the table as well, 1,040.  3.1 M entries with handles in runs of eight: 16 + 6 us.
#include "kv_attend.cuh"

namespace kvt {
namespace {

constexpr int kScoreThreads = 256;
__device__ __forceinline__ float fold(float acc, unsigned long long w, float decay) {
  return __fadd_rn(__fmul_rn(decay, acc), __fmul_rn(__ull2float_rn(w), 0x1p-32f));
}

__global__ void __launch_bounds__(kScoreThreads) fold_weights_kernel(float* score, uint64_t n_entries, const uint32_t* loc, uint64_t n_tags,
                                                                     float decay, unsigned long long* weight, float* acc) {
  wait_for_kernel_ahead();
  const uint64_t g = ((uint64_t)blockIdx.x * kScoreThreads + threadIdx.x) * 4u;
  if (g >= n_tags) return;
  const uint32_t n = (uint32_t)min((unsigned long long)(n_tags - g), 4ull);
  uint32_t e[4] = {KV_NONE, KV_NONE, KV_NONE, KV_NONE};
  if (n == 4u) {
    const uint4 x = __ldcs(reinterpret_cast<const uint4*>(loc + g));
    e[0] = x.x; e[1] = x.y; e[2] = x.z; e[3] = x.w;
  } else {
    for (uint32_t k = 0; k < n; ++k) e[k] = loc[g + k];
  }
  bool any = false, all = true;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    any = any || e[k] < n_entries;
    all = all && e[k] < n_entries;
  }
  if (!any) return;
  if (all) {
    const ulonglong2 w0 = __ldcs(reinterpret_cast<const ulonglong2*>(weight + g)), w1 = __ldcs(reinterpret_cast<const ulonglong2*>(weight + g) + 1);
    float4 x = __ldcs(reinterpret_cast<const float4*>(acc + g));
    x.x = fold(x.x, w0.x, decay);
    x.y = fold(x.y, w0.y, decay);
    x.z = fold(x.z, w1.x, decay);
    x.w = fold(x.w, w1.y, decay);
    __stcs(reinterpret_cast<float4*>(acc + g), x);
    if (w0.x | w0.y) __stcs(reinterpret_cast<ulonglong2*>(weight + g), make_ulonglong2(0, 0));
    if (w1.x | w1.y) __stcs(reinterpret_cast<ulonglong2*>(weight + g) + 1, make_ulonglong2(0, 0));
    score[e[0]] = x.x;
    score[e[1]] = x.y;
    score[e[2]] = x.z;
    score[e[3]] = x.w;
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (e[k] >= n_entries) continue;      // in the host tier, or nowhere
    const unsigned long long w = weight[g + k];
    const float x = fold(acc[g + k], w, decay);
    acc[g + k] = x;
    if (w) weight[g + k] = 0ull;
    score[e[k]] = x;
  }
}

// Scores of entries that are FREE, or young, are +inf.
__global__ void __launch_bounds__(kScoreThreads) keep_young_kernel(EntryState st, uint32_t epoch, int32_t protect) {
  const uint64_t i = ((uint64_t)blockIdx.x * kScoreThreads + threadIdx.x) * 4u;
  bool keep[4] = {false, false, false, false};
  if (i + 4u <= st.n) {
    const uchar4 s = *reinterpret_cast<const uchar4*>(st.state + i);
    keep[0] = s.x != KV_STATE_RESIDENT;
    keep[1] = s.y != KV_STATE_RESIDENT;
    keep[2] = s.z != KV_STATE_RESIDENT;
    keep[3] = s.w != KV_STATE_RESIDENT;
    if (protect > 0) {
      const uint4 l = *reinterpret_cast<const uint4*>(st.last_epoch + i);
      keep[0] = keep[0] || (int32_t)(epoch - l.x) < protect;
      keep[1] = keep[1] || (int32_t)(epoch - l.y) < protect;
      keep[2] = keep[2] || (int32_t)(epoch - l.z) < protect;
      keep[3] = keep[3] || (int32_t)(epoch - l.w) < protect;
    }
  } else {
    for (uint64_t j = i; j < st.n; ++j)
      keep[j - i] = st.state[j] != KV_STATE_RESIDENT || (protect > 0 && (int32_t)(epoch - st.last_epoch[j]) < protect);
  }
  wait_for_kernel_ahead();      // (what is read above was there before the kernel ahead began; it writes scores)
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (keep[k]) st.score[i + k] = INFINITY;
}

}  // namespace

bool stream_captured(cudaStream_t s) {
  cudaStreamCaptureStatus now = cudaStreamCaptureStatusNone;
  if (cudaStreamIsCapturing(s, &now) == cudaSuccess) return now != cudaStreamCaptureStatusNone;
  (void)cudaGetLastError();
  return true;
}

cudaError_t launch_attention_score(const EntryState& st, const uint32_t* loc, uint64_t n_tags, uint32_t epoch, float decay, uint32_t protect,
                                   unsigned long long* weight, float* acc, cudaStream_t s) {
  constexpr uint64_t per_cta = kScoreThreads * 4ull;
  if (n_tags > KV_NONE) n_tags = KV_NONE;
  // (a pool without handles: one CTA that finds nothing, as the kernel behind counts on one between itself and all that came before)
  const uint64_t fold_ctas = n_tags ? (n_tags + per_cta - 1u) / per_cta : 1u;
  const cudaError_t e = launch_overlapped(fold_weights_kernel, (unsigned)fold_ctas, (unsigned)kScoreThreads, s, st.score,
                                          st.n, loc, n_tags, decay, weight, acc);
  if (e != cudaSuccess) return e;
  return launch_overlapped(keep_young_kernel, (unsigned)((st.n + per_cta - 1u) / per_cta), (unsigned)kScoreThreads, s, st, epoch, (int32_t)protect);
}

}  // namespace kvt
