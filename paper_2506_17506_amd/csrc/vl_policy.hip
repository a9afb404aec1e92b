// Advantages of samples within their groups, from the violations counted in them, and the clipped policy
// loss of the samples' tokens with its gradient in their log probabilities.
#include "vl_dev.h"

using namespace vl;

namespace {

constexpr uint32_t kThreads = 256;

template <class F, class V>
__device__ V block_reduce(V v, V *room, F join) {
  room[threadIdx.x] = v;
  __syncthreads();
  for (uint32_t d = kThreads / 2; d; d /= 2) {
    if (threadIdx.x < d) room[threadIdx.x] = join(room[threadIdx.x], room[threadIdx.x + d]);
    __syncthreads();
  }
  v = room[0];
  __syncthreads();
  return v;
}

__device__ inline double reward_of(const vl_counts *counts, const float *extra, vl_reward_weights w, uint32_t k) {
  double r = extra ? (double)extra[k] : 0.0;
  if (counts) {
    const vl_counts c = counts[k];
    r += (c.kinds == 0 ? (double)w.ok : 0.0) + (double)w.cons * c.n_cons + (double)w.real * c.n_real + (double)w.safe * c.n_safe;
  }
  return r;
}

__global__ __launch_bounds__(kThreads) void k_advantages(const vl_counts *counts, const float *extra, uint32_t n, const uint32_t *group_off,
                                                         uint32_t n_group, vl_reward_weights w, float eps, float *reward, float *advantage) {
  __shared__ double sums[kThreads];
  auto add = [](double x, double y) { return x + y; };
  for (uint32_t g = blockIdx.x; g < n_group; g += gridDim.x) {
    const uint32_t k0 = min(group_off[g], n), k1 = min(group_off[g + 1], n);
    if (k0 >= k1) continue;
    // distances to the first sample's reward: all equal ones give 0 exactly
    const double first = reward_of(counts, extra, w, k0);
    double s = 0;
    for (uint32_t k = k0 + threadIdx.x; k < k1; k += kThreads) s += reward_of(counts, extra, w, k) - first;
    const double mean = block_reduce(s, sums, add) / (k1 - k0);
    double v = 0;
    for (uint32_t k = k0 + threadIdx.x; k < k1; k += kThreads) {
      const double d = reward_of(counts, extra, w, k) - first - mean;
      v += d * d;
    }
    const double dev = sqrt(block_reduce(v, sums, add) / (k1 - k0)) + (double)eps;
    for (uint32_t k = k0 + threadIdx.x; k < k1; k += kThreads) {
      const double r = reward_of(counts, extra, w, k);
      if (reward) reward[k] = (float)r;
      if (advantage) advantage[k] = (float)((r - first - mean) / dev);
    }
  }
}

struct Part { double loss, kl; uint64_t n_token, n_clipped; };

// exp(q) - q - 1 without cancellation near 0
__device__ inline float exp_gap(float q) {
  if (fabsf(q) < 0.25f)   // q^2 (1/2 + q/6 + ... + q^6/40320): the next term is below 2^-25 of the first
    return q * q * (0.5f + q * (1.0f / 6 + q * (1.0f / 24 + q * (1.0f / 120 + q * (1.0f / 720 + q * (1.0f / 5040 + q * (1.0f / 40320)))))));
  return expm1f(q) - q;
}

__global__ __launch_bounds__(kThreads) void k_policy(vl_policy_batch b, float *grad, Part *parts) {
  __shared__ double sums[kThreads];
  __shared__ uint64_t numbers[kThreads];
  double loss = 0, kls = 0;
  uint64_t tokens = 0, clips = 0;
  for (uint32_t c = blockIdx.x; c < b.n_sample; c += gridDim.x) {
    const uint64_t i0 = min(b.start[c], b.n), i1 = min(i0 + b.len[c], b.n);
    const float a = b.advantage[c], w = b.weight[c];
    for (uint64_t i = i0 + threadIdx.x; i < i1; i += kThreads) {
      const float lp = b.logprob[i], old = b.logprob_old[i];
      const double d = (double)lp - (double)old;
      const bool clip = (a > 0.0f && d > (double)b.log_hi) || (a < 0.0f && d < (double)b.log_lo);
      float l = -a * expf(clip ? (a > 0.0f ? b.log_hi : b.log_lo) : (float)d), dx = clip ? 0.0f : l;
      if (b.logprob_ref) {
        const float q = b.logprob_ref[i] - lp, gap = exp_gap(q);
        l += b.kl * gap;
        dx -= b.kl * expm1f(q);
        kls += (double)w * gap;
      }
      grad[i] = w * dx;
      loss += (double)w * l;
      clips += clip;
      ++tokens;
    }
  }
  auto add = [](auto x, auto y) { return x + y; };
  Part p;
  p.loss = block_reduce(loss, sums, add);
  p.kl = block_reduce(kls, sums, add);
  p.n_token = block_reduce(tokens, numbers, add);
  p.n_clipped = block_reduce(clips, numbers, add);
  if (threadIdx.x == 0) parts[blockIdx.x] = p;
}

__global__ __launch_bounds__(kThreads) void k_policy_join(const Part *parts, uint32_t n, vl_policy_stats *stats) {
  __shared__ double sums[kThreads];
  __shared__ uint64_t numbers[kThreads];
  Part p = {0, 0, 0, 0};
  for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
    p.loss += parts[i].loss; p.kl += parts[i].kl; p.n_token += parts[i].n_token; p.n_clipped += parts[i].n_clipped;
  }
  auto add = [](auto x, auto y) { return x + y; };
  p.loss = block_reduce(p.loss, sums, add);
  p.kl = block_reduce(p.kl, sums, add);
  p.n_token = block_reduce(p.n_token, numbers, add);
  p.n_clipped = block_reduce(p.n_clipped, numbers, add);
  if (threadIdx.x == 0) *stats = vl_policy_stats{(float)p.loss, (float)p.kl, p.n_token, p.n_clipped};
}

int32_t check_batch(const vl_policy_batch *b) {
  if (!b || !b->logprob || !b->logprob_old || !b->start || !b->len || !b->advantage || !b->weight || (b->kl != 0.0f && !b->logprob_ref)) return VL_E_NULL;
  if (b->reserved0 != 0 || !(b->log_lo <= b->log_hi) || !(fabsf(b->kl) <= 3.402823466e38f)) return VL_E_RANGE;
  if (b->n == 0 || b->n >> 60 || b->n_sample == 0 || b->n_sample > 0x7FFFFFFFu) return VL_E_SHAPE;
  if (((uintptr_t)b->logprob | (uintptr_t)b->logprob_old | (uintptr_t)b->logprob_ref | (uintptr_t)b->len | (uintptr_t)b->advantage | (uintptr_t)b->weight) & 3 ||
      (uintptr_t)b->start & 7) return VL_E_SHAPE;
  return VL_OK;
}

uint32_t policy_blocks(const vl_policy_batch *b) { return b->n_sample < 4096u ? b->n_sample : 4096u; }

}  // namespace

extern "C" int32_t vl_group_advantages(const vl_counts *counts, const float *extra, uint32_t n, const uint32_t *group_off, uint32_t n_group,
                                       const vl_reward_weights *weights, float eps, float *reward, float *advantage, vl_stream stream_) {
  if ((!counts && !extra) || !group_off || !weights || (!reward && !advantage)) return VL_E_NULL;
  if (n == 0 || n > 0x7FFFFFFFu || n_group == 0 || n_group > 0x7FFFFFFFu) return VL_E_SHAPE;
  if (((uintptr_t)counts | (uintptr_t)extra | (uintptr_t)group_off | (uintptr_t)reward | (uintptr_t)advantage) & 3) return VL_E_SHAPE;
  const float most = 3.402823466e38f;
  if (!(fabsf(weights->ok) <= most) || !(fabsf(weights->cons) <= most) || !(fabsf(weights->real) <= most) || !(fabsf(weights->safe) <= most) ||
      !(eps > 0.0f) || eps > most) return VL_E_RANGE;
  const uint32_t blocks = n_group < 65536u ? n_group : 65536u;
  k_advantages<<<blocks, kThreads, 0, (hipStream_t)stream_>>>(counts, extra, n, group_off, n_group, *weights, eps, reward, advantage);
  VL_HIP(hipGetLastError());
  return VL_OK;
}

extern "C" int32_t vl_policy_loss_work(const vl_policy_batch *batch, uint64_t *bytes) {
  if (!bytes) return VL_E_NULL;
  const int32_t rc = check_batch(batch);
  if (rc == VL_OK) *bytes = (uint64_t)policy_blocks(batch) * sizeof(Part);
  return rc;
}

extern "C" int32_t vl_policy_loss(const vl_policy_batch *batch, float *grad, vl_policy_stats *stats, void *work, uint64_t work_bytes, vl_stream stream_) {
  if (!grad || !stats || !work) return VL_E_NULL;
  uint64_t need = 0;
  const int32_t rc = vl_policy_loss_work(batch, &need);
  if (rc != VL_OK) return rc;
  if (work_bytes < need || (uintptr_t)work & 15 || (uintptr_t)grad & 3 || (uintptr_t)stats & 7) return VL_E_SHAPE;
  hipStream_t stream = (hipStream_t)stream_;
  const uint32_t blocks = policy_blocks(batch);
  k_policy<<<blocks, kThreads, 0, stream>>>(*batch, grad, (Part *)work);
  k_policy_join<<<1, kThreads, 0, stream>>>((const Part *)work, blocks, stats);
  VL_HIP(hipGetLastError());
  return VL_OK;
}
