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
// sums over kTeam threads (a wavefront, or the whole workgroup), in every one of them
template <uint32_t kTeam>
__device__ inline void team_sums(double &x, double &y, double (*room)[kTeam / 64]) {
  x = wave_sum(x);
  y = wave_sum(y);
  if constexpr (kTeam > 64) {
    if ((threadIdx.x & 63u) == 0) {
      room[0][threadIdx.x >> 6] = x;
      room[1][threadIdx.x >> 6] = y;
    }
    __syncthreads();
    x = y = 0;
#pragma unroll 4
    for (uint32_t w = 0; w < kTeam / 64; ++w) {
      x += room[0][w];
      y += room[1][w];
    }
    __syncthreads();
  }
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
// taken as distances d to the group's first, so that equal ones have a spread of exactly 0, and the variance as mean(d^2) - mean(d)^2
// in one pass: as one of the K distances is 0, the variance is mean(d)^2 / K at least, so the difference loses a factor of
// K + 1 at most of 64 bits' precision.
template <uint32_t kTeam>
__global__ __launch_bounds__(kTeam < 256 ? 256 : kTeam) void k_advantages(Rewards w, uint32_t n, const uint32_t VL_GLOBAL *group_off, uint32_t n_group, double eps,
                                                                         float VL_GLOBAL *reward, float VL_GLOBAL *advantage) {
  __shared__ double room[2][kTeam / 64];
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
    for (uint32_t i = 0; i < kKeep; ++i) {
      const double d = kept[i] - first;
      s += d;
      v += d * d;
    }
    for (uint64_t k = (uint64_t)k0 + me + kKeep * kTeam; k < k1; k += kTeam) {
      const double d = reward_of(w, (uint32_t)k) - first;
      s += d;
      v += d * d;
    }
    team_sums<kTeam>(s, v, room);
    const double mean = s / size, var = v / size - mean * mean, scale = 1.0 / (sqrt(var < 0.0 ? 0.0 : var) + eps);   // (NaN stays NaN)
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

constexpr uint32_t kGroups = 2, kStep = kGroups * 256;   // a lane takes kGroups times four tokens, a wavefront kStep, at once
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));
// Whole steps' numbers are not kept in the caches, read or written: 66 M tokens 162 -> 147 us, 2 M 16.3 -> 13.9; but 5 M with a reference 22.2 -> 23.4.
__device__ inline f32x4 load_once(const float VL_GLOBAL *x) { return __builtin_nontemporal_load((const f32x4_any VL_GLOBAL *)x); }

// exp(q) - q - 1 and exp(q) - 1.  Near 0 from the series of the first, q^2 (1/2 + q/6 + ... + q^7/362880), whose next term is
// below 2^-28 of the sum for |q| < 1/2: the difference would cancel.  Infinite where the exponential is, at q = +infinity too.
__device__ inline void exp_gap(float q, float &gap, float &less_one) {
  if (fabsf(q) < 0.5f) {
    gap = q * q * (0.5f + q * (1.0f / 6 + q * (1.0f / 24 + q * (1.0f / 120 + q * (1.0f / 720 + q * (1.0f / 5040 + q * (1.0f / 40320 + q * (1.0f / 362880))))))));
    less_one = gap + q;
  } else {
    const float e = expf(q);
    less_one = e - 1.0f;
    gap = e == __builtin_huge_valf() ? e : less_one - q;
  }
}

struct Sample { uint64_t from, to; float a, w; };

__device__ inline Part add_parts(Part p, const Part &q) { return Part{p.loss + q.loss, p.kl + q.kl, p.n_token + q.n_token, p.n_clipped + q.n_clipped}; }
__device__ inline void write_stats(vl_policy_stats VL_GLOBAL *stats, const Part &p) {
  stats->loss = (float)p.loss;
  stats->kl = (float)p.kl;
  stats->n_token = p.n_token;
  stats->n_clipped = p.n_clipped;
}

// A wavefront takes a slice of a sample at a time.  What bounds it: the arrays' bytes.  Whether d is past a bound is decided in 64
// bits, where the difference of two numbers of 32 is exact (unless they are so far apart that no rounding matters), and every loss goes into a sum of 64 bits.
// exp(d) and exp(q) are infinite above 88.7 in 32 bits: terms whose factor is 0 are left out, not multiplied by it.
template <bool kRef, uint32_t kWaves>
__global__ __launch_bounds__(kWaves * 64) void k_policy(Batch b, Part VL_GLOBAL *parts, vl_policy_stats VL_GLOBAL *stats) {
  __shared__ Part room[kWaves];
  const uint32_t lane = threadIdx.x & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint64_t n_unit = (uint64_t)b.n_sample * b.slices, stride = (uint64_t)gridDim.x * kWaves;
  double loss = 0, kls = 0;
  uint64_t tokens = 0, clips = 0;
  auto sample_of = [&](uint64_t unit) {
    const uint32_t c = (uint32_t)unit / b.slices, slice = (uint32_t)unit - c * b.slices;   // (fewer than 2^32 units)
    const uint64_t i0 = least_of(b.start[c], b.n), i1 = least_of(i0 + b.len[c], b.n);
    // slices end at multiples of kStep
    const uint64_t base = i0 / kStep * kStep, per = ((i1 - base + kStep - 1) / kStep + b.slices - 1) / b.slices * kStep;
    const uint64_t from = least_of(base + slice * per, i1), to = least_of(base + (slice + 1) * per, i1);
    return Sample{from < i0 ? i0 : from, to < i0 ? i0 : to, b.advantage[c], b.weight[c]};
  };
  for (uint64_t unit = (uint64_t)blockIdx.x * kWaves + wave; unit < n_unit; unit += stride) {
    const Sample s = sample_of(unit);
    const float bound = s.a > 0.0f ? b.log_hi : b.log_lo;
    const double hi = s.a > 0.0f ? (double)b.log_hi : (double)__builtin_huge_valf(), lo = s.a < 0.0f ? (double)b.log_lo : -(double)__builtin_huge_valf();
    double sum = 0, kl_sum = 0;
    uint32_t n_clip = 0;
    auto token = [&](float lp, float old, float ref) {
      const double d = (double)lp - (double)old;
      const bool clip = d > hi || d < lo;
      const float ratio = -s.a * expf(clip ? bound : (float)d);
      float l = s.a == 0.0f ? 0.0f : ratio, g = clip ? 0.0f : l;
      if (kRef) {
        float gap, less_one;
        exp_gap(ref - lp, gap, less_one);
        const float more = b.kl * gap, less = b.kl * less_one;
        l += b.kl == 0.0f ? 0.0f : more;
        g -= b.kl == 0.0f ? 0.0f : less;
        kl_sum += gap;
      }
      sum += l;
      n_clip += clip;
      const float of = s.w * g;
      return s.w == 0.0f ? 0.0f : of;
    };
    // steps start at multiples of kStep in the arrays, so that all but a sample's ends is read in whole lines
    for (uint64_t i = s.from / kStep * kStep; i < s.to; i += kStep) {
      const uint64_t at = i + lane * 4;
      f32x4 lp[kGroups], old[kGroups], ref[kGroups] = {};
      if (i >= s.from && i + kStep <= s.to) {
#pragma unroll
        for (uint32_t u = 0; u < kGroups; ++u) {
          lp[u] = load_once(b.logprob + at + u * 256);
          old[u] = load_once(b.logprob_old + at + u * 256);
          if (kRef) ref[u] = load_once(b.logprob_ref + at + u * 256);
        }
#pragma unroll
        for (uint32_t u = 0; u < kGroups; ++u) {
          f32x4 g;
#pragma unroll
          for (uint32_t j = 0; j < 4; ++j) g[j] = token(lp[u][j], old[u][j], ref[u][j]);
          __builtin_nontemporal_store(g, (f32x4_any VL_GLOBAL *)(b.grad + at + u * 256));
        }
      } else {
#pragma unroll
        for (uint32_t u = 0; u < kGroups; ++u)
#pragma unroll
          for (uint32_t j = 0; j < 4; ++j) {   // (neighbouring lanes take neighbouring tokens)
            const uint64_t k = i + (u * 4 + j) * 64 + lane;
            const bool in = k >= s.from && k < s.to;
            lp[u][j] = in ? b.logprob[k] : 0.0f;
            old[u][j] = in ? b.logprob_old[k] : 0.0f;
            if (kRef) ref[u][j] = in ? b.logprob_ref[k] : 0.0f;
          }
#pragma unroll
        for (uint32_t u = 0; u < kGroups; ++u)
#pragma unroll
          for (uint32_t j = 0; j < 4; ++j) {
            const uint64_t k = i + (u * 4 + j) * 64 + lane;
            if (k >= s.from && k < s.to) b.grad[k] = token(lp[u][j], old[u][j], ref[u][j]);
          }
      }
    }
    if (s.w != 0.0f && s.from < s.to) {   // (the weight of a sample without tokens may be 1 / 0)
      loss += (double)s.w * sum;
      if (kRef) kls += (double)s.w * kl_sum;
    }
    tokens += s.to - s.from;   // (the same in all lanes)
    clips += n_clip;
  }
  const Part p = {wave_sum(loss), kRef ? wave_sum(kls) : 0.0, tokens, wave_sum((unsigned long long)clips)};
  if (lane == 0) room[wave] = p;
  __syncthreads();
  if (threadIdx.x == 0) {
    Part all = room[0];
    for (uint32_t w = 1; w < kWaves; ++w) all = add_parts(all, room[w]);
    if (gridDim.x == 1) {   // nothing to join
      write_stats(stats, all);
      return;
    }
    parts[blockIdx.x].loss = all.loss;
    parts[blockIdx.x].kl = all.kl;
    parts[blockIdx.x].n_token = all.n_token;
    parts[blockIdx.x].n_clipped = all.n_clipped;
  }
}

constexpr uint32_t kJoinThreads = 1024;
__global__ __launch_bounds__(kJoinThreads) void k_policy_join(const Part VL_GLOBAL *parts, uint32_t n, vl_policy_stats VL_GLOBAL *stats) {
  __shared__ Part room[kJoinThreads / 64];
  Part p = {0, 0, 0, 0};
  for (uint32_t i = threadIdx.x; i < n; i += 4 * kJoinThreads) {   // (four at once on their way)
    Part q[4];
#pragma unroll
    for (uint32_t u = 0; u < 4; ++u) {
      const uint32_t at = i + u * kJoinThreads;
      q[u] = at < n ? Part{parts[at].loss, parts[at].kl, parts[at].n_token, parts[at].n_clipped} : Part{0, 0, 0, 0};
    }
#pragma unroll
    for (uint32_t u = 0; u < 4; ++u) p = add_parts(p, q[u]);
  }
#pragma unroll
  for (int d = 32; d; d >>= 1)
    p = add_parts(p, Part{__shfl_xor(p.loss, d), __shfl_xor(p.kl, d), __shfl_xor(p.n_token, d), __shfl_xor(p.n_clipped, d)});
  if ((threadIdx.x & 63u) == 0) room[threadIdx.x >> 6] = p;
  __syncthreads();
  if (threadIdx.x >= 64) return;
  p = threadIdx.x < kJoinThreads / 64 ? room[threadIdx.x] : Part{0, 0, 0, 0};
#pragma unroll
  for (int d = 8; d; d >>= 1)
    p = add_parts(p, Part{__shfl_xor(p.loss, d), __shfl_xor(p.kl, d), __shfl_xor(p.n_token, d), __shfl_xor(p.n_clipped, d)});
  if (threadIdx.x == 0) write_stats(stats, p);
}

int32_t check_batch(const vl_policy_batch *b) {
  if (!b || !b->logprob || !b->logprob_old || !b->start || !b->len || !b->advantage || !b->weight || (b->kl != 0.0f && !b->logprob_ref)) return VL_E_NULL;
  if (b->reserved0 != 0 || !(b->log_lo <= b->log_hi) || !(fabsf(b->kl) <= 3.402823466e38f)) return VL_E_RANGE;
  if (b->n == 0 || b->n >> 60 || b->n_sample == 0 || b->n_sample > 0x7FFFFFFFu) return VL_E_SHAPE;
  if (((uintptr_t)b->logprob | (uintptr_t)b->logprob_old | (uintptr_t)b->logprob_ref | (uintptr_t)b->len | (uintptr_t)b->advantage | (uintptr_t)b->weight) & 3 ||
      (uintptr_t)b->start & 7) return VL_E_SHAPE;
  return VL_OK;
}

// Slices of a sample, of about 2,048 tokens by the longest one, less where that leaves wavefronts idle, and workgroups for them,
// 8,192 at most.  (1,600 samples of 43,000 tokens on average, a slice per wavefront: 147 us, slices of 4,096 tokens 156, of 1,024 142; but
// 40 M tokens 92, 97 and 97.)
// A workgroup of 1,024 threads alone, with nothing to join, takes what is small: two slices per wavefront at most.  (Four
// samples, us alone / joined: 1,000 tokens 5.4 / 8.4, 16,000 7.6 / 9.0, 32,000 13.0 / 9.2; 100 samples of 1,000 in all 15.9 / 8.5.)
constexpr uint32_t kAloneTokens = 16384, kAloneSlices = 32;
struct Launch { uint32_t slices, waves, blocks; };
Launch launch_of(const vl_policy_batch *b) {
  const uint64_t want = std::max<uint64_t>({1, b->max_len / 2048, std::min<uint64_t>(b->max_len / kStep, 8192 / b->n_sample)}), most = std::max<uint64_t>(1, 0xFFFFFFFFull / b->n_sample);
  const uint32_t slices = (uint32_t)std::min({want, most, (uint64_t)1024});
  if (b->n <= kAloneTokens && (uint64_t)b->n_sample * slices <= kAloneSlices) return Launch{slices, 16, 1};
  return Launch{slices, 4, (uint32_t)std::min<uint64_t>(8192, ((uint64_t)b->n_sample * slices + 3) / 4)};
}

uint64_t work_of(const Launch &l) { return l.blocks > 1 ? (uint64_t)l.blocks * sizeof(Part) : 0; }

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
  // Threads by the groups' mean size: up to four rewards each stay in registers.  us by 64 / 256 / 1,024 threads, without the host: 1,024 groups of
  // 100 4.1 / 4.5 / 10.7, 256 of 100 3.3 / 3.2 / 4.7; 256 of 300 5.0 / 3.9 / 5.0, 256 of 1,000 17.6 / 6.5 / 6.6, 1,024 of 1,000 23.7 / 11.3 /
  // 15.5; 1 of 4,000 36.8 / 10.9 / 5.5.  (Few groups of 256: 3.8 / 3.2 / 4.4.)
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
  if (rc == VL_OK) *bytes = work_of(launch_of(batch));
  return rc;
}

extern "C" int32_t vl_policy_loss(const vl_policy_batch *batch, float *grad, vl_policy_stats *stats, void *work, uint64_t work_bytes, vl_stream stream_) {
  if (!grad || !stats) return VL_E_NULL;
  const int32_t rc = check_batch(batch);
  if (rc != VL_OK) return rc;
  const Launch launch = launch_of(batch);
  if ((uintptr_t)grad & 3 || (uintptr_t)stats & 7) return VL_E_SHAPE;
  if (const uint64_t need = work_of(launch)) {
    if (!work) return VL_E_NULL;
    if (work_bytes < need || (uintptr_t)work & 15) return VL_E_SHAPE;
  }
  hipStream_t stream = (hipStream_t)stream_;
  const Batch b = {(const float VL_GLOBAL *)batch->logprob, (const float VL_GLOBAL *)batch->logprob_old, (const float VL_GLOBAL *)batch->logprob_ref,
                   (const uint64_t VL_GLOBAL *)batch->start, (const uint32_t VL_GLOBAL *)batch->len, (const float VL_GLOBAL *)batch->advantage,
                   (const float VL_GLOBAL *)batch->weight, (float VL_GLOBAL *)grad, batch->n, batch->n_sample, launch.slices,
                   batch->log_lo, batch->log_hi, batch->kl};
  Part VL_GLOBAL *parts = (Part VL_GLOBAL *)work;
  vl_policy_stats VL_GLOBAL *to = (vl_policy_stats VL_GLOBAL *)stats;
  (b.logprob_ref ? launch.waves == 16 ? k_policy<true, 16> : k_policy<true, 4> : launch.waves == 16 ? k_policy<false, 16> : k_policy<false, 4>)
      <<<launch.blocks, launch.waves * 64, 0, stream>>>(b, parts, to);
  if (launch.blocks > 1) k_policy_join<<<1, kJoinThreads, 0, stream>>>(parts, launch.blocks, to);
  VL_HIP(hipGetLastError());
  return VL_OK;
}
