// Token scores: log probabilities of given tokens, entropy and the largest logits of each row
// over the tokens its mask leaves, and the gradient of the first two in the logits.
#include "vl_dev.h"

using namespace vl;

namespace {

constexpr float kNoLogit = -__builtin_huge_valf();

struct Rows {
  const uint8_t VL_GLOBAL *logits;
  uint64_t ld;                         // in bytes
  const uint32_t VL_GLOBAL *mask;
  uint64_t mask_ld;
  const int32_t VL_GLOBAL *token;
  uint32_t n_row, n_vocab;
  float scale;
};

struct F32 { typedef float type; static __device__ float wide(float x) { return x; } static __device__ float narrow(float x) { return x; } };
struct F16 { typedef _Float16 type; static __device__ float wide(_Float16 x) { return (float)x; } static __device__ _Float16 narrow(float x) { return (_Float16)x; } };
struct BF16 { typedef __bf16 type; static __device__ float wide(__bf16 x) { return (float)x; } static __device__ __bf16 narrow(float x) { return (__bf16)x; } };

template <class T>
__device__ inline float logit(const Rows &a, uint32_t r, uint32_t t) {
  if (a.mask && !((a.mask[(uint64_t)r * a.mask_ld + (t >> 5)] >> (t & 31u)) & 1u)) return kNoLogit;
  return T::wide(((const typename T::type VL_GLOBAL *)(a.logits + (uint64_t)r * a.ld))[t]);
}

constexpr uint32_t kThreads = 256;

struct Best { float x; uint32_t t; };   // a logit and its token; better: larger, or equal and of a lower token
__device__ inline bool better(Best a, Best b) { return a.x > b.x || (a.x == b.x && a.t < b.t); }

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

template <class T>
__global__ __launch_bounds__(kThreads) void k_scores(Rows a, vl_token_scores out) {
  __shared__ float sums[kThreads];
  __shared__ Best bests[kThreads];
  for (uint32_t r = blockIdx.x; r < a.n_row; r += gridDim.x) {
    const int32_t token = a.token ? a.token[r] : 0;
    const bool padding = token < 0;
    const uint32_t n = padding ? 0u : a.n_vocab;
    float m = kNoLogit;
    for (uint32_t t = threadIdx.x; t < n; t += kThreads) m = fmaxf(m, logit<T>(a, r, t));
    m = block_reduce(m, sums, [](float x, float y) { return fmaxf(x, y); });
    const float from = m == kNoLogit ? 0.0f : m;
    float s = 0, y = 0;
    for (uint32_t t = threadIdx.x; t < n; t += kThreads) {
      const float z = (logit<T>(a, r, t) - from) * a.scale, e = expf(z);
      s += e;
      y += e == 0.0f ? 0.0f : e * z;
    }
    auto add = [](float u, float v) { return u + v; };
    s = block_reduce(s, sums, add);
    y = block_reduce(y, sums, add);
    const bool bad = s != s;
    const float log_sum = logf(s);
    if (threadIdx.x == 0) {
      const bool in = !padding && (uint32_t)token < a.n_vocab;
      const float x = a.token && in ? logit<T>(a, r, (uint32_t)token) : kNoLogit;
      if (out.logprob) out.logprob[r] = padding ? 0.0f : bad ? s : x == kNoLogit ? kNoLogit : (x - from) * a.scale - log_sum;
      if (out.entropy) out.entropy[r] = s == 0.0f ? 0.0f : log_sum - y / s;
      if (out.stat) {
        out.stat[2ull * r] = padding ? 0.0f : bad ? s : m;
        out.stat[2ull * r + 1] = padding ? 0.0f : log_sum;
      }
    }
    Best last = {__builtin_huge_valf(), 0u};
    for (uint32_t k = 0; k < out.n_top; ++k) {
      Best b = {kNoLogit, kNone};
      for (uint32_t t = threadIdx.x; t < n; t += kThreads) {
        const Best c = {logit<T>(a, r, t), t};
        if (c.x != kNoLogit && better(c, b) && better(last, c)) b = c;
      }
      last = b = block_reduce(b, bests, [](Best u, Best v) { return better(u, v) ? u : v; });
      if (threadIdx.x == 0) {
        const uint64_t at = (uint64_t)r * out.n_top + k;
        const bool none = b.t == kNone;
        if (out.top_token) out.top_token[at] = none || bad ? -1 : (int32_t)b.t;
        if (out.top_logprob) out.top_logprob[at] = bad ? s : none ? kNoLogit : (b.x - from) * a.scale - log_sum;
      }
    }
  }
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_score_grad(Rows a, const float *stat, const float *entropy, const float *g_logprob,
                                                         const float *g_entropy, uint8_t *grad, uint64_t grad_ld) {
  for (uint32_t r = blockIdx.x; r < a.n_row; r += gridDim.x) {
    const int32_t token = a.token ? a.token[r] : 0;
    typename T::type *to = (typename T::type *)(grad + (uint64_t)r * grad_ld);
    const float m = stat[2ull * r], log_sum = stat[2ull * r + 1];
    const bool none = token < 0 || m == kNoLogit;
    const float g = none || !g_logprob ? 0.0f : g_logprob[r], e = none || !g_entropy ? 0.0f : g_entropy[r];
    const float h = none || !g_entropy ? 0.0f : entropy[r];
    for (uint32_t t = threadIdx.x; t < a.n_vocab; t += kThreads) {
      float d = 0;
      if (!none && (!a.mask || ((a.mask[(uint64_t)r * a.mask_ld + (t >> 5)] >> (t & 31u)) & 1u))) {
        const float lp = (T::wide(((const typename T::type VL_GLOBAL *)(a.logits + (uint64_t)r * a.ld))[t]) - m) * a.scale - log_sum;
        const float p = expf(lp);
        d = g * ((t == (uint32_t)token ? 1.0f : 0.0f) - p) - (p == 0.0f ? 0.0f : e * p * (lp + h));
        d *= a.scale;
      }
      to[t] = T::narrow(d);
    }
  }
}

constexpr uint32_t kMostRows = 0x7FFFFFFFu;

uint32_t size_of(uint32_t type) { return type == VL_F32 ? 4u : 2u; }

int32_t check_rows(const vl_token_rows *a) {
  if (!a || !a->logits) return VL_E_NULL;
  if (a->type > VL_BF16) return VL_E_RANGE;
  if (a->n_vocab == 0 || a->n_vocab > VL_MAX_VOCAB || !(a->scale > 0.0f) || a->scale > 3.402823466e38f) return VL_E_RANGE;
  if (a->n_row == 0 || a->n_row > kMostRows || (a->n_row > 1 && a->ld < a->n_vocab)) return VL_E_SHAPE;
  if (a->mask && a->mask_ld && a->mask_ld < (a->n_vocab + 31) / 32) return VL_E_SHAPE;
  if (((uintptr_t)a->logits & (size_of(a->type) - 1)) || ((uintptr_t)a->mask & 3) || ((uintptr_t)a->token & 3)) return VL_E_SHAPE;
  return VL_OK;
}

int32_t check_scores(const vl_token_rows *a, const vl_token_scores *o) {
  if (!o) return VL_E_NULL;
  const int32_t rc = check_rows(a);
  if (rc != VL_OK) return rc;
  if (o->reserved0 != 0 || o->n_top > VL_MAX_TOP) return VL_E_RANGE;
  if (!o->logprob && !o->entropy && !o->stat && !o->top_token && !o->top_logprob) return VL_E_NULL;
  if ((o->n_top != 0) != (o->top_token || o->top_logprob)) return VL_E_NULL;
  if (o->logprob && !a->token) return VL_E_NULL;
  if (((uintptr_t)o->logprob | (uintptr_t)o->entropy | (uintptr_t)o->stat | (uintptr_t)o->top_token | (uintptr_t)o->top_logprob) & 3) return VL_E_SHAPE;
  return VL_OK;
}

Rows device_rows(const vl_token_rows *a) {
  return Rows{(const uint8_t VL_GLOBAL *)a->logits, a->ld * size_of(a->type), (const uint32_t VL_GLOBAL *)a->mask, a->mask_ld,
              (const int32_t VL_GLOBAL *)a->token, a->n_row, a->n_vocab, a->scale};
}

}  // namespace

extern "C" int32_t vl_token_logprobs_work(const vl_token_rows *rows, const vl_token_scores *out, uint64_t *bytes) {
  if (!bytes) return VL_E_NULL;
  const int32_t rc = check_scores(rows, out);
  if (rc == VL_OK) *bytes = 0;
  return rc;
}

extern "C" int32_t vl_token_logprobs(const vl_token_rows *rows, const vl_token_scores *out, void *work, uint64_t work_bytes, vl_stream stream_) {
  const int32_t rc = check_scores(rows, out);
  if (rc != VL_OK) return rc;
  (void)work; (void)work_bytes;
  hipStream_t stream = (hipStream_t)stream_;
  const Rows a = device_rows(rows);
  const uint32_t blocks = a.n_row < 65536u ? a.n_row : 65536u;
  (rows->type == VL_F32 ? k_scores<F32> : rows->type == VL_F16 ? k_scores<F16> : k_scores<BF16>)<<<blocks, kThreads, 0, stream>>>(a, *out);
  VL_HIP(hipGetLastError());
  return VL_OK;
}

extern "C" int32_t vl_token_logprobs_grad(const vl_token_rows *rows, const float *stat, const float *entropy, const float *g_logprob,
                                          const float *g_entropy, void *grad, uint64_t grad_ld, vl_stream stream_) {
  if (!stat || !grad || (!g_logprob && !g_entropy) || (g_entropy && !entropy)) return VL_E_NULL;
  const int32_t rc = check_rows(rows);
  if (rc != VL_OK) return rc;
  if (g_logprob && !rows->token) return VL_E_NULL;
  if ((rows->n_row > 1 && grad_ld < rows->n_vocab) || (uintptr_t)grad & (size_of(rows->type) - 1)) return VL_E_SHAPE;
  if (((uintptr_t)stat | (uintptr_t)entropy | (uintptr_t)g_logprob | (uintptr_t)g_entropy) & 3) return VL_E_SHAPE;
  hipStream_t stream = (hipStream_t)stream_;
  const Rows a = device_rows(rows);
  const uint32_t blocks = a.n_row < 65536u ? a.n_row : 65536u;
  (rows->type == VL_F32 ? k_score_grad<F32> : rows->type == VL_F16 ? k_score_grad<F16> : k_score_grad<BF16>)<<<blocks, kThreads, 0, stream>>>(
      a, stat, entropy, g_logprob, g_entropy, (uint8_t *)grad, grad_ld * size_of(rows->type));
  VL_HIP(hipGetLastError());
  return VL_OK;
}
