// Advantages of samples within their groups, from the violations counted in them, and the clipped policy
// loss of the samples' tokens with its gradient in their log probabilities.
#include <algorithm>

#include "vl_dev.h"

using namespace vl;

namespace {

__device__ inline uint64_t least_of(uint64_t x, uint64_t y) { return x < y ? x : y; }

// sum over the wavefront, in every lane
template <class V>
__device__ inline V wave_sum(V x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d, 64);
  return x;
}
// sum over kTeam threads (a wavefront, or the whole workgroup), in every one of them
template <uint32_t kTeam, class V>
__device__ inline V team_sum(V x, V *room) {
  x = wave_sum(x);
  if constexpr (kTeam > 64) {
    if ((threadIdx.x & 63u) == 0) room[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0;
#pragma unroll 4
    for (uint32_t w = 0; w < kTeam / 64; ++w) x += room[w];
    __syncthreads();
  }
  return x;
}

struct Rewards {
  const uint8_t VL_GLOBAL *counts;
  const float VL_GLOBAL *extra;
  double ok, cons, real, safe;
};
typedef u32x4 u32x4_any __attribute__((aligned(4)));
__device__ inline double reward_of(const Rewards &w, uint32_t k) {
  double r = w.extra ? (double)w.extra[k] : 0.0;
  if (w.counts) {
    const u32x4 c = *(const u32x4_any VL_GLOBAL *)(w.counts + (uint64_t)k * sizeof(vl_counts));   // kinds, n_cons, n_real, n_safe
    r += (c.x == 0 ? w.ok : 0.0) + w.cons * c.y + w.real * c.z + w.safe * c.w;
  }
  return r;
}

constexpr uint32_t kKeep = 4;   // rewards of a thread that stay in registers

// kTeam threads per group.  What bounds it: the trips to memory, for the group's offsets and then for its records.  Rewards are
// taken as distances to the group's first, so that equal ones have a spread of exactly 0.
template <uint32_t kTeam>
__global__ __launch_bounds__(kTeam < 256 ? 256 : kTeam) void k_advantages(Rewards w, uint32_t n, const uint32_t VL_GLOBAL *group_off, uint32_t n_group, double eps,
                                                                         float VL_GLOBAL *reward, float VL_GLOBAL *advantage) {
  __shared__ double room[kTeam < 64 ? 1 : kTeam / 64];
  const uint32_t teams = kTeam < 256 ? 256 / kTeam : 1, me = threadIdx.x % kTeam;
  for (uint32_t g = blockIdx.x * teams + threadIdx.x / kTeam; g < n_group; g += gridDim.x * teams) {
    const uint32_t k0 = min(group_off[g], n), k1 = min(group_off[g + 1], n);
    if (k0 >= k1) continue;
    const double first = reward_of(w, k0), size = k1 - k0;
    double kept[kKeep], s = 0, v = 0;
#pragma unroll
    for (uint32_t i = 0; i < kKeep; ++i) {
      const uint32_t k = k0 + me + i * kTeam;
      kept[i] = k >= k0 && k < k1 ? reward_of(w, k) : first;
    }
#pragma unroll
    for (uint32_t i = 0; i < kKeep; ++i) s += kept[i] - first;
    for (uint64_t k = (uint64_t)k0 + me + kKeep * kTeam; k < k1; k += kTeam) s += reward_of(w, (uint32_t)k) - first;
    const double mean = team_sum<kTeam>(s, room) / size;
#pragma unroll
    for (uint32_t i = 0; i < kKeep; ++i) {
      const double d = kept[i] - first - mean;
      if ((uint64_t)k0 + me + i * kTeam < k1) v += d * d;
    }
    for (uint64_t k = (uint64_t)k0 + me + kKeep * kTeam; k < k1; k += kTeam) {
      const double d = reward_of(w, (uint32_t)k) - first - mean;
      v += d * d;
    }
    const double scale = 1.0 / (sqrt(team_sum<kTeam>(v, room) / size) + eps);
#pragma unroll
    for (uint32_t i = 0; i < kKeep; ++i) {
      const uint64_t k = (uint64_t)k0 + me + i * kTeam;
      if (k >= k1) break;
      if (reward) reward[k] = (float)kept[i];
      if (advantage) advantage[k] = (float)((kept[i] - first - mean) * scale);
    }
    for (uint64_t k = (uint64_t)k0 + me + kKeep * kTeam; k < k1; k += kTeam) {
      const double r = reward_of(w, (uint32_t)k);
      if (reward) reward[k] = (float)r;
      if (advantage) advantage[k] = (float)((r - first - mean) * scale);
    }
  }
}

struct Batch {
  const float VL_GLOBAL *logprob, *logprob_old, *logprob_ref;
  const uint64_t VL_GLOBAL *start;
  const uint32_t VL_GLOBAL *len;
  const float VL_GLOBAL *advantage, *weight;
  float VL_GLOBAL *grad;
  uint64_t n;
  uint32_t n_sample, slices;
  float log_lo, log_hi, kl;
};
struct Part { double loss, kl; uint64_t n_token, n_clipped; };

constexpr uint32_t kPolicyThreads = 256, kPolicyWaves = kPolicyThreads / 64;
constexpr uint32_t kGroups = 2, kStep = kGroups * 256;   // a lane takes kGroups times four tokens, a wavefront kStep, at once
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));

// exp(q) - q - 1 and exp(q) - 1.  Near 0 from the series of the first, q^2 (1/2 + q/6 + ... + q^6/40320), whose next term is
// below 2^-30 of the sum for |q| < 1/4: the difference would cancel.
__device__ inline void exp_gap(float q, float &gap, float &less_one) {
  if (fabsf(q) < 0.25f) {
    gap = q * q * (0.5f + q * (1.0f / 6 + q * (1.0f / 24 + q * (1.0f / 120 + q * (1.0f / 720 + q * (1.0f / 5040 + q * (1.0f / 40320)))))));
    less_one = gap + q;
  } else {
    const float e = expf(q);
    less_one = e - 1.0f;
    gap = less_one - q;
  }
}

struct Sample { uint64_t from, to; float a, w; };

// A wavefront takes a slice of a sample at a time.  What bounds it: the arrays' bytes.  Whether d is past a bound is decided in 64
// bits, where the difference of two numbers of 32 is exact (unless they are so far apart that no rounding matters), and every loss goes into a sum of 64 bits.
template <bool kRef>
__global__ __launch_bounds__(kPolicyThreads) void k_policy(Batch b, Part VL_GLOBAL *parts) {
  __shared__ Part room[kPolicyWaves];
  const uint32_t lane = threadIdx.x & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint64_t n_unit = (uint64_t)b.n_sample * b.slices, stride = (uint64_t)gridDim.x * kPolicyWaves;
  double loss = 0, kls = 0;
  uint64_t tokens = 0, clips = 0;
  auto sample_of = [&](uint64_t unit) {
    const uint32_t c = (uint32_t)unit / b.slices, slice = (uint32_t)unit - c * b.slices;   // (fewer than 2^32 units)
    const uint64_t i0 = least_of(b.start[c], b.n), i1 = least_of(i0 + b.len[c], b.n), per = ((i1 - i0 + b.slices - 1) / b.slices + kStep - 1) / kStep * kStep;
    return Sample{least_of(i0 + slice * per, i1), least_of(i0 + (slice + 1) * per, i1), b.advantage[c], b.weight[c]};
  };
  for (uint64_t unit = (uint64_t)blockIdx.x * kPolicyWaves + wave; unit < n_unit; unit += stride) {
    const Sample s = sample_of(unit);
    const float bound = s.a > 0.0f ? b.log_hi : b.log_lo;
    const double hi = s.a > 0.0f ? (double)b.log_hi : (double)__builtin_huge_valf(), lo = s.a < 0.0f ? (double)b.log_lo : -(double)__builtin_huge_valf();
    double sum = 0, kl_sum = 0;
    uint32_t n_clip = 0;
    auto token = [&](float lp, float old, float ref) {
      const double d = (double)lp - (double)old;
      const bool clip = d > hi || d < lo;
      float l = -s.a * expf(clip ? bound : (float)d), g = clip ? 0.0f : l;
      if (kRef) {
        float gap, less_one;
        exp_gap(ref - lp, gap, less_one);
        l += b.kl * gap;
        g -= b.kl * less_one;
        kl_sum += gap;
      }
      sum += l;
      n_clip += clip;
      return s.w * g;
    };
    for (uint64_t i = s.from; i < s.to; i += kStep) {
      const uint64_t at = i + lane * 4;
      if (i + kStep <= s.to) {
        f32x4 lp[kGroups], old[kGroups], ref[kGroups] = {};
#pragma unroll
        for (uint32_t u = 0; u < kGroups; ++u) {
          lp[u] = *(const f32x4_any VL_GLOBAL *)(b.logprob + at + u * 256);
          old[u] = *(const f32x4_any VL_GLOBAL *)(b.logprob_old + at + u * 256);
          if (kRef) ref[u] = *(const f32x4_any VL_GLOBAL *)(b.logprob_ref + at + u * 256);
        }
#pragma unroll
        for (uint32_t u = 0; u < kGroups; ++u) {
          f32x4 g;
#pragma unroll
          for (uint32_t j = 0; j < 4; ++j) g[j] = token(lp[u][j], old[u][j], ref[u][j]);
          *(f32x4_any VL_GLOBAL *)(b.grad + at + u * 256) = g;
        }
      } else {
        for (uint64_t k = i + lane; k < s.to; k += 64) b.grad[k] = token(b.logprob[k], b.logprob_old[k], kRef ? b.logprob_ref[k] : 0.0f);
      }
    }
    loss += (double)s.w * sum;
    if (kRef) kls += (double)s.w * kl_sum;
    tokens += s.to - s.from;   // (the same in all lanes)
    clips += n_clip;
  }
  const Part p = {wave_sum(loss), kRef ? wave_sum(kls) : 0.0, tokens, wave_sum((unsigned long long)clips)};
  if (lane == 0) room[wave] = p;
  __syncthreads();
  if (threadIdx.x == 0) {
    Part all = room[0];
    for (uint32_t w = 1; w < kPolicyWaves; ++w) {
      all.loss += room[w].loss; all.kl += room[w].kl; all.n_token += room[w].n_token; all.n_clipped += room[w].n_clipped;
    }
    parts[blockIdx.x].loss = all.loss;
    parts[blockIdx.x].kl = all.kl;
    parts[blockIdx.x].n_token = all.n_token;
    parts[blockIdx.x].n_clipped = all.n_clipped;
  }
}

constexpr uint32_t kJoinThreads = 1024;
__global__ __launch_bounds__(kJoinThreads) void k_policy_join(const Part VL_GLOBAL *parts, uint32_t n, vl_policy_stats VL_GLOBAL *stats) {
  __shared__ double sums[kJoinThreads / 64];
  __shared__ unsigned long long numbers[kJoinThreads / 64];
  Part p = {0, 0, 0, 0};
  for (uint32_t i = threadIdx.x; i < n; i += kJoinThreads) {
    p.loss += parts[i].loss; p.kl += parts[i].kl; p.n_token += parts[i].n_token; p.n_clipped += parts[i].n_clipped;
  }
  p.loss = team_sum<kJoinThreads>(p.loss, sums);
  p.kl = team_sum<kJoinThreads>(p.kl, sums);
  p.n_token = team_sum<kJoinThreads>((unsigned long long)p.n_token, numbers);
  p.n_clipped = team_sum<kJoinThreads>((unsigned long long)p.n_clipped, numbers);
  if (threadIdx.x == 0) {
    stats->loss = (float)p.loss;
    stats->kl = (float)p.kl;
    stats->n_token = p.n_token;
    stats->n_clipped = p.n_clipped;
  }
}

int32_t check_batch(const vl_policy_batch *b) {
  if (!b || !b->logprob || !b->logprob_old || !b->start || !b->len || !b->advantage || !b->weight || (b->kl != 0.0f && !b->logprob_ref)) return VL_E_NULL;
  if (b->reserved0 != 0 || !(b->log_lo <= b->log_hi) || !(fabsf(b->kl) <= 3.402823466e38f)) return VL_E_RANGE;
  if (b->n == 0 || b->n >> 60 || b->n_sample == 0 || b->n_sample > 0x7FFFFFFFu) return VL_E_SHAPE;
  if (((uintptr_t)b->logprob | (uintptr_t)b->logprob_old | (uintptr_t)b->logprob_ref | (uintptr_t)b->len | (uintptr_t)b->advantage | (uintptr_t)b->weight) & 3 ||
      (uintptr_t)b->start & 7) return VL_E_SHAPE;
  return VL_OK;
}

// Slices of a sample, of about 2,048 tokens by the longest one, and workgroups for them, eight per compute unit at most
struct Launch { uint32_t slices, blocks; };
Launch launch_of(const vl_policy_batch *b) {
  const uint64_t want = std::max<uint64_t>(1, b->max_len / 2048), most = std::max<uint64_t>(1, 0xFFFFFFFFull / b->n_sample);
  const uint32_t slices = (uint32_t)std::min({want, most, (uint64_t)1024});
  return Launch{slices, (uint32_t)std::min<uint64_t>(2048, ((uint64_t)b->n_sample * slices + kPolicyWaves - 1) / kPolicyWaves)};
}

}  // namespace

extern "C" int32_t vl_group_advantages(const vl_counts *counts, const float *extra, uint32_t n, const uint32_t *group_off, uint32_t n_group,
                                       const vl_reward_weights *weights, float eps, float *reward, float *advantage, vl_stream stream_) {
  if ((!counts && !extra) || !group_off || !weights || (!reward && !advantage)) return VL_E_NULL;
  if (n == 0 || n > 0x7FFFFFFFu || n_group == 0 || n_group > 0x7FFFFFFFu) return VL_E_SHAPE;
  if (((uintptr_t)counts | (uintptr_t)extra | (uintptr_t)group_off | (uintptr_t)reward | (uintptr_t)advantage) & 3) return VL_E_SHAPE;
  const float most = 3.402823466e38f;
  if (!(fabsf(weights->ok) <= most) || !(fabsf(weights->cons) <= most) || !(fabsf(weights->real) <= most) || !(fabsf(weights->safe) <= most) ||
      !(eps > 0.0f) || eps > most) return VL_E_RANGE;
  const Rewards w = {(const uint8_t VL_GLOBAL *)counts, (const float VL_GLOBAL *)extra, weights->ok, weights->cons, weights->real, weights->safe};
  // threads by the groups' mean size: up to four rewards each stay in registers
  const uint32_t mean = n / n_group, teams = mean <= 256 ? 4 : 1;
  const uint32_t blocks = std::min((n_group + teams - 1) / teams, 65536u);
  if (mean <= 256) k_advantages<64><<<blocks, 256, 0, (hipStream_t)stream_>>>(w, n, (const uint32_t VL_GLOBAL *)group_off, n_group, eps, (float VL_GLOBAL *)reward, (float VL_GLOBAL *)advantage);
  else if (mean <= 1024) k_advantages<256><<<blocks, 256, 0, (hipStream_t)stream_>>>(w, n, (const uint32_t VL_GLOBAL *)group_off, n_group, eps, (float VL_GLOBAL *)reward, (float VL_GLOBAL *)advantage);
  else k_advantages<1024><<<blocks, 1024, 0, (hipStream_t)stream_>>>(w, n, (const uint32_t VL_GLOBAL *)group_off, n_group, eps, (float VL_GLOBAL *)reward, (float VL_GLOBAL *)advantage);
  VL_HIP(hipGetLastError());
  return VL_OK;
}

extern "C" int32_t vl_policy_loss_work(const vl_policy_batch *batch, uint64_t *bytes) {
  if (!bytes) return VL_E_NULL;
  const int32_t rc = check_batch(batch);
  if (rc == VL_OK) *bytes = (uint64_t)launch_of(batch).blocks * sizeof(Part);
  return rc;
}

extern "C" int32_t vl_policy_loss(const vl_policy_batch *batch, float *grad, vl_policy_stats *stats, void *work, uint64_t work_bytes, vl_stream stream_) {
  if (!grad || !stats || !work) return VL_E_NULL;
  const int32_t rc = check_batch(batch);
  if (rc != VL_OK) return rc;
  const Launch launch = launch_of(batch);
  if (work_bytes < launch.blocks * sizeof(Part) || (uintptr_t)work & 15 || (uintptr_t)grad & 3 || (uintptr_t)stats & 7) return VL_E_SHAPE;
  hipStream_t stream = (hipStream_t)stream_;
  const Batch b = {(const float VL_GLOBAL *)batch->logprob, (const float VL_GLOBAL *)batch->logprob_old, (const float VL_GLOBAL *)batch->logprob_ref,
                   (const uint64_t VL_GLOBAL *)batch->start, (const uint32_t VL_GLOBAL *)batch->len, (const float VL_GLOBAL *)batch->advantage,
                   (const float VL_GLOBAL *)batch->weight, (float VL_GLOBAL *)grad, batch->n, batch->n_sample, launch.slices,
                   batch->log_lo, batch->log_hi, batch->kl};
  Part VL_GLOBAL *parts = (Part VL_GLOBAL *)work;
  (b.logprob_ref ? k_policy<true> : k_policy<false>)<<<launch.blocks, kPolicyThreads, 0, stream>>>(b, parts);
  k_policy_join<<<1, kJoinThreads, 0, stream>>>(parts, launch.blocks, (vl_policy_stats VL_GLOBAL *)stats);
  VL_HIP(hipGetLastError());
  return VL_OK;
}
