// Token scores: log probabilities of given tokens, entropy and the largest logits of each row
// over the tokens its mask leaves, and the gradient of the first two in the logits.
//
// A row is read once.  Its logits are taken in chunks of 16 bytes, wherever the row starts (the
// card reads and writes 16 bytes at any address; a chunk that the row's end cuts is taken an element at a time).
// A lane holds the largest logit m of its chunks so far, the sum S of exp(z) for z = scale (x - m), and the sum Y of
// z exp(z): when m grows by d, S is scaled by exp(-d) and Y becomes exp(-d) (Y - d S).  All terms of S have one sign, and
// all of Y, so log S - Y / S, the entropy, loses nothing.  Lanes, wavefronts and parts of rows are joined the
// same way.  z is kept in powers of two (scale * log2 e in one factor), for the card's exp2.
//
// The n best of a row cost the loop next to nothing: a lane also keeps which of its chunks its m came from.  The n lanes
// with the best (m, chunk) hold all of the row's n best: any other lane's best is below n
// larger ones.  Those chunks are read again, and all chunks of such a lane if its second best chunk reaches the worst of those n
// maxima too; what does, seldom much more than n logits, is put in order by counting, for each, how many are better.
#include <algorithm>
#include <type_traits>

#include "vl_dev.h"

using namespace vl;

namespace {

constexpr float kNoLogit = -__builtin_huge_valf();
constexpr float kLeast = -3.402823466e38f;   // stands for m where there is none, so that no difference is of two infinities
constexpr float kFar = -1000.0f;             // (powers of two) exp2 gives 0 long before; keeps 0 * infinity out of Y
constexpr float kLog2e = 1.44269504088896f, kLn2 = 0.69314718055994f;

struct Rows {
  const uint8_t VL_GLOBAL *logits;
  uint64_t ld;                         // in bytes
  const uint8_t VL_GLOBAL *mask;
  uint64_t mask_ld;                    // in bytes
  const int32_t VL_CONSTANT *token;
  uint32_t n_row, n_vocab;
  float scale, scale2;                 // scale2 = scale * log2 e
};
struct Scores {
  float VL_GLOBAL *logprob, *entropy, *stat, *top_logprob;
  int32_t VL_GLOBAL *top_token;
  uint32_t n_top;
};

__device__ inline float as_float(uint32_t x) { return __builtin_bit_cast(float, x); }
__device__ inline uint32_t as_word(float x) { return __builtin_bit_cast(uint32_t, x); }

struct F32 {
  typedef float type;
  typedef u32x4 chunk __attribute__((aligned(4)));
  static constexpr uint32_t kElems = 4, kBits = 32, kNone = 0xFF800000u;   // -infinity, as often as a word holds it
  static __device__ inline float wide(float x) { return x; }
  static __device__ inline float narrow(float x) { return x; }
  static __device__ inline void unpack(u32x4 w, float *x) {
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) x[j] = as_float(w[j]);
  }
  static __device__ inline u32x4 pack(const float *x) {
    u32x4 w;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) w[j] = as_word(x[j]);
    return w;
  }
};
struct F16 {
  typedef _Float16 type;
  typedef _Float16 pair __attribute__((ext_vector_type(2)));
  typedef u32x4 chunk __attribute__((aligned(2)));
  static constexpr uint32_t kElems = 8, kBits = 19, kNone = 0xFC00FC00u;   // (bits: sign, the exponent of 32 bits, ten)
  static __device__ inline float wide(_Float16 x) { return (float)x; }
  static __device__ inline _Float16 narrow(float x) { return (_Float16)x; }
  static __device__ inline void unpack(u32x4 w, float *x) {
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
      const uint32_t both = w[j];   // (a bit cast of a vector's element itself takes the first one)
      const pair p = __builtin_bit_cast(pair, both);
      x[2 * j] = (float)p.x;
      x[2 * j + 1] = (float)p.y;
    }
  }
  static __device__ inline u32x4 pack(const float *x) {
    u32x4 w;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) w[j] = __builtin_bit_cast(uint32_t, pair{(_Float16)x[2 * j], (_Float16)x[2 * j + 1]});
    return w;
  }
};
struct BF16 {
  typedef __bf16 type;
  typedef __bf16 pair __attribute__((ext_vector_type(2)));
  typedef u32x4 chunk __attribute__((aligned(2)));
  static constexpr uint32_t kElems = 8, kBits = 16, kNone = 0xFF80FF80u;
  static __device__ inline float wide(__bf16 x) { return (float)x; }
  static __device__ inline __bf16 narrow(float x) { return (__bf16)x; }
  static __device__ inline void unpack(u32x4 w, float *x) {
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
      x[2 * j] = as_float(w[j] << 16);
      x[2 * j + 1] = as_float(w[j] & 0xFFFF0000u);
    }
  }
  static __device__ inline u32x4 pack(const float *x) {
    u32x4 w;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) w[j] = __builtin_bit_cast(uint32_t, pair{(__bf16)x[2 * j], (__bf16)x[2 * j + 1]});
    return w;
  }
};

constexpr uint32_t kThreads = 256, kWaves = kThreads / 64;
constexpr uint32_t kShortChunks = 128;   // 16-byte chunks of a row that a few lanes hold in registers

template <class T>
__device__ inline u32x4 load_chunk(const uint8_t VL_GLOBAL *row, uint32_t c) {
  return *(const typename T::chunk VL_GLOBAL *)(row + (uint64_t)c * 16);
}
template <class T>
__device__ inline u32x4 load_once(const uint8_t VL_GLOBAL *row, uint32_t c) {   // nothing of it is kept in the caches
  return __builtin_nontemporal_load((const typename T::chunk VL_GLOBAL *)(row + (uint64_t)c * 16));
}
// Long rows of 16 bits a logit are taken from the multiple of 4 bytes at or below their start, `lead` (0 or 1) logits early,
// since loads from odd places cost: 4,096 rows of 50,001 logits 91 us, of 50,000 78.  Chunk c then holds tokens
// c * 8 - lead and up; what stands before the row does not count.  (It lies in the word that holds the row's first logit.)
template <class T>
__device__ inline uint32_t lead_of(const uint8_t VL_GLOBAL *row) { return T::kElems == 8 ? ((uint32_t)(uintptr_t)row >> 1) & 1u : 0u; }
template <class T>
__device__ inline u32x4 load_even(const uint8_t VL_GLOBAL *row, uint32_t lead, uint32_t c) {
  typedef u32x4 words __attribute__((aligned(4)));
  return *(const words VL_GLOBAL *)(row - lead * 2 + (uint64_t)c * 16);
}
template <class T>
__device__ inline u32x4 load_once(const uint8_t VL_GLOBAL *row, uint32_t lead, uint32_t c) {   // nothing of it is kept in the caches
  typedef u32x4 words __attribute__((aligned(4)));
  return __builtin_nontemporal_load((const words VL_GLOBAL *)(row - lead * 2 + (uint64_t)c * 16));
}

// the logits that the mask does not allow become -infinity (bit j of `bits`: logit j is allowed)
template <class T>
__device__ inline void keep_allowed(float *x, uint32_t bits) {
#pragma unroll
  for (uint32_t j = 0; j < T::kElems; ++j) {
    const uint32_t keep = (uint32_t)((int32_t)(bits << (31 - j)) >> 31);
    x[j] = as_float((as_word(x[j]) & keep) | (0xFF800000u & ~keep));
  }
}
template <class T>
__device__ inline uint32_t mask_bits(const uint8_t VL_GLOBAL *mask, uint32_t c) {   // of chunk c, in the low bits
  if (T::kElems == 8) return mask[c];
  return mask[c >> 1] >> ((c & 1) * 4);
}

template <class T>
__device__ inline uint32_t mask_bits(const uint8_t VL_GLOBAL *mask, uint32_t lead, uint32_t c) {
  if (T::kElems == 4 || !lead) return mask_bits<T>(mask, c);
  return (uint32_t)mask[c] << 1 | (c ? mask[c - 1] >> 7 : 0u);   // (nothing allowed in front of the row)
}

// Chunks lane, lane + kStride, ... of a short row, into bits what the mask says of them (all ones without one).  All loads are on their way
// before the first is waited for.
template <class T, uint32_t kStride, uint32_t kChunks>
__device__ inline void load_row(const Rows &a, const uint8_t VL_GLOBAL *row, const uint8_t VL_GLOBAL *mask, uint32_t lane, float (*x)[T::kElems], uint32_t *bits) {
  u32x4 w[kChunks];
#pragma unroll
  for (uint32_t i = 0; i < kChunks; ++i) {
    const uint32_t c = lane + kStride * i;
    w[i] = u32x4{T::kNone, T::kNone, T::kNone, T::kNone};
    if ((c + 1) * T::kElems <= a.n_vocab) w[i] = load_chunk<T>(row, c);
  }
#pragma unroll
  for (uint32_t i = 0; i < kChunks; ++i) {
    const uint32_t c = lane + kStride * i;
    bits[i] = ~0u;
    if (mask && c * T::kElems < a.n_vocab) bits[i] = mask_bits<T>(mask, c);
  }
  const uint32_t cut = a.n_vocab / T::kElems;   // the chunk that the row's end cuts, if it does
  float last[T::kElems];
  if (a.n_vocab % T::kElems) {
#pragma unroll
    for (uint32_t j = 0; j < T::kElems; ++j) {
      const uint32_t t = cut * T::kElems + j;
      last[j] = t < a.n_vocab ? T::wide(((const typename T::type VL_GLOBAL *)row)[t]) : kNoLogit;
    }
  }
#pragma unroll
  for (uint32_t i = 0; i < kChunks; ++i) T::unpack(w[i], x[i]);
  if (a.n_vocab % T::kElems) {
#pragma unroll
    for (uint32_t i = 0; i < kChunks; ++i)
#pragma unroll
      for (uint32_t j = 0; j < T::kElems; ++j) x[i][j] = lane + kStride * i == cut ? last[j] : x[i][j];
  }
}

// a chunk of a long row, with its lead
template <class T>
__device__ inline void load_any(const Rows &a, const uint8_t VL_GLOBAL *row, const uint8_t VL_GLOBAL *mask, uint32_t lead, uint32_t c, float *x) {
  const uint32_t from = c * T::kElems - lead;   // (2^32 - 1 in front of the row)
  if (c * T::kElems + T::kElems <= a.n_vocab + lead) {
    T::unpack(load_even<T>(row, lead, c), x);
    if (mask) keep_allowed<T>(x, mask_bits<T>(mask, lead, c));
    if (lead > c) x[0] = kNoLogit;
    return;
  }
#pragma unroll
  for (uint32_t j = 0; j < T::kElems; ++j) {
    const uint32_t t = from + j;
    const bool in = t < a.n_vocab && (!mask || ((mask[t >> 3] >> (t & 7)) & 1));
    x[j] = in ? T::wide(((const typename T::type VL_GLOBAL *)row)[t]) : kNoLogit;
  }
}

// ---- over a wavefront: rows of 16 lanes, then across rows; the result stands in lane 63
template <class F>
__device__ inline float wave_fold(float x, float none, F f) {
  auto step = [&](auto ctrl, auto rows) {
    const int y = __builtin_amdgcn_update_dpp((int)as_word(none), (int)as_word(x), decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
    x = f(x, as_float((uint32_t)y));
  };
  step(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});   // row_shr:1, 2, 4, 8
  step(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
  step(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
  step(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
  step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});   // row_bcast:15 into rows 1 and 3
  step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});   // row_bcast:31 into rows 2 and 3
  return as_float((uint32_t)__builtin_amdgcn_readlane((int)as_word(x), 63));
}
__device__ inline float wave_max(float x) { return wave_fold(x, kNoLogit, [](float u, float v) { return fmaxf(u, v); }); }
__device__ inline float wave_sum(float x) { return wave_fold(x, 0.0f, [](float u, float v) { return u + v; }); }

// over 16 lanes, in all of them
template <class F>
__device__ inline float quarter_fold(float x, F f) {
  auto step = [&](auto ctrl) {
    const int y = __builtin_amdgcn_update_dpp(0, (int)as_word(x), decltype(ctrl)::value, 0xf, 0xf, false);
    x = f(x, as_float((uint32_t)y));
  };
  step(std::integral_constant<int, 0x128>{});   // row_ror:8, 4, 2, 1
  step(std::integral_constant<int, 0x124>{});
  step(std::integral_constant<int, 0x122>{});
  step(std::integral_constant<int, 0x121>{});
  return x;
}

// ---- a row's sums so far
struct Sums { float m, s, y; };
__device__ inline float ref_of(float m) { return fmaxf(m, kLeast); }
// `from` seen from the larger maximum `m`
__device__ inline Sums rebase(Sums from, float m, float scale2) {
  const float d = fmaxf((ref_of(from.m) - ref_of(m)) * scale2, kFar), f = __builtin_amdgcn_exp2f(d);
  return Sums{m, from.s * f, f * (from.y + d * from.s)};
}

// ---- the best: a logit and its place as one number, larger = better (a larger logit, or an equal one of a lower place).  A
// logit's order takes kBits of the upper word, as many as its type tells apart.
template <class T>
__device__ inline uint32_t ordered(float x) {
  const uint32_t b = as_word(x + 0.0f);   // (one zero)
  return (b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u)) >> (32 - T::kBits);
}
template <class T>
__device__ inline float unordered(uint32_t u) {
  u <<= 32 - T::kBits;
  return as_float(u >> 31 ? u ^ 0x80000000u : ~(u | ((1ull << (32 - T::kBits)) - 1)));
}
__device__ inline uint64_t key_of(uint32_t value, uint32_t place) { return ((uint64_t)value << 32) | (uint32_t)~place; }
__device__ inline uint64_t lane_key(uint64_t k, uint32_t lane) {
  return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)k, lane);
}

__device__ inline uint32_t lanes_below(uint64_t lanes) {   // how many of them are below this one
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, 0));
}

// A number that at least n of the keys which a wavefront's lanes hold (0: none, the others all differ) reach, and at
// most `most` >= n of them; 1 if there are fewer than n.  Bit by bit from the top; places are below 2^place_bits.
template <uint32_t kBits>
__device__ inline uint64_t nth_key(uint64_t k, uint32_t place_bits, uint32_t n, uint32_t most) {
  // (four bits at a time without a branch: one scalar unit serves a compute unit's wavefronts)
  uint32_t value = 0, reached = 0;
#pragma unroll
  for (int32_t top = kBits - 1; top >= 0; top -= 4) {
#pragma unroll
    for (int32_t bit = top; bit > top - 4 && bit >= 0; --bit) {
      const uint32_t attempt = value | (1u << bit), count = __popcll(__ballot((uint32_t)(k >> 32) >= attempt));
      value = count >= n ? attempt : value;
      reached = count >= n ? count : reached;
    }
    if (reached && reached <= most) return (uint64_t)value << 32;
  }
  if (!value) return 1ull;
  uint64_t least = ((uint64_t)value << 32) | (0xFFFFFFFFull & ~((1ull << place_bits) - 1ull));   // (the same in every key)
  for (int32_t bit = (int32_t)place_bits - 1; bit >= 0; --bit) {
    const uint64_t attempt = least | (1ull << bit);
    const uint32_t count = __popcll(__ballot(k >= attempt));
    if (count < n) continue;
    least = attempt;
    if (count <= most) return least;
  }
  return least;
}
__device__ inline uint32_t bits_for(uint32_t n) { return 32u - (uint32_t)__builtin_clz(n | 1u); }   // of numbers up to n

// how many of the first `found` keys are larger; the list goes on with zeros to a multiple of four
__device__ inline uint32_t rank_of(const uint64_t *keys, uint32_t found, uint64_t mine) {
  uint32_t rank = 0;
  for (uint32_t i = 0; i < found; i += 4)
#pragma unroll
    for (uint32_t u = 0; u < 4; ++u) rank += keys[i + u] > mine;
  return rank;
}

// Where keys that may be among a row's n best are gathered.  More than there is room for are possible (many equal
// logits, or a row sorted in an unlucky way); then the row's best are found by insertion instead.
constexpr uint32_t kMoreHot = 4;   // more than n lanes may have their chunks looked at again, so that the search for them ends sooner
template <uint32_t kTeam>
struct Room {
  static constexpr uint32_t kMost = kTeam < 256 ? kTeam : 256;   // (one per thread is put in order)
  uint64_t key[kMost];
  uint32_t n;
};
template <uint32_t kTeam>
__device__ inline void gather(Room<kTeam> &room, uint64_t key) {
  const uint32_t at = atomicAdd(&room.n, 1u);   // (their order does not matter)
  if (at < Room<kTeam>::kMost) room.key[at] = key;
}

// A sorted list, entry i in lane i, 0 where there is none; `worst` is entry n - 1.
struct List {
  uint64_t key = 0, worst = 0;
  __device__ inline void insert(uint64_t k, uint32_t n) {   // (k the same in all lanes)
    if (k <= worst) return;
    const uint32_t lane = threadIdx.x & 63u;
    const uint32_t at = __popcll(__ballot(key > k));
    // entries from `at` on move up one lane
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)key, 0x138, 0xf, 0xf, false);   // wave_shr:1
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(key >> 32), 0x138, 0xf, 0xf, false);
    key = lane < at ? key : lane == at ? k : ((uint64_t)hi << 32) | lo;
    worst = lane_key(key, n - 1);
  }
  // what the lanes where `ask` is set hold
  __device__ inline void insert_lanes(uint64_t k, bool ask, uint32_t n) {
    for (uint64_t todo = __ballot(ask); todo; todo &= todo - 1) insert(lane_key(k, (uint32_t)__builtin_ctzll(todo)), n);
  }
};

// f(is, key) for a chunk's logits, `is` set for those at or above `least`, a (value, chunk), which so may be among the best; key() makes
// the number
template <class T, class F>
__device__ inline void each_candidate(const float *x, uint32_t lead, uint32_t c, uint64_t least, F f) {
  const uint32_t value = (uint32_t)(least >> 32) + (c <= (uint32_t)~least ? 0u : 1u);
  const float from = value <= (0x00800000u >> (32 - T::kBits)) ? kLeast : unordered<T>(value);   // (any but -infinity, at the least)
#pragma unroll
  for (uint32_t j = 0; j < T::kElems; ++j) f(x[j] >= from, [&] { return key_of(ordered<T>(x[j]), c * T::kElems - lead + j); });
}

// ---- what a row's results are made of
struct Final { float m, s, log_sum, scale; bool bad; };
__device__ inline float logprob_of(const Final &f, float x) {
  return f.bad ? f.s : x == kNoLogit ? kNoLogit : (x - ref_of(f.m)) * f.scale - f.log_sum;
}
__device__ inline Final finish(const Rows &a, const Scores &out, uint32_t r, Sums sums, float x, bool write) {
  const Final f = {sums.m, sums.s, logf(sums.s), a.scale, sums.s != sums.s};
  if (write) {
    if (out.logprob) out.logprob[r] = logprob_of(f, x);
    if (out.entropy) out.entropy[r] = f.s == 0.0f ? 0.0f : f.log_sum - kLn2 * sums.y / f.s;
    if (out.stat) {
      out.stat[2ull * r] = f.bad ? f.s : f.m;
      out.stat[2ull * r + 1] = f.log_sum;
    }
  }
  return f;
}
template <class T>
__device__ inline void write_top(const Scores &out, uint32_t r, uint32_t k, uint64_t key, const Final &f) {
  const uint64_t at = (uint64_t)r * out.n_top + k;
  if (out.top_token) out.top_token[at] = key && !f.bad ? (int32_t)~(uint32_t)key : -1;
  if (out.top_logprob) out.top_logprob[at] = f.bad ? f.s : key ? logprob_of(f, unordered<T>((uint32_t)(key >> 32))) : kNoLogit;
}
// a row of padding; `lane` of out.n_top or more
__device__ inline void write_padding(const Scores &out, uint32_t r, uint32_t lane) {
  if (lane == 0) {
    if (out.logprob) out.logprob[r] = 0.0f;
    if (out.entropy) out.entropy[r] = 0.0f;
    if (out.stat) out.stat[2ull * r] = out.stat[2ull * r + 1] = 0.0f;
  }
  if (lane < out.n_top) write_top<F32>(out, r, lane, 0, Final{0, 0, 0, 0, false});
}
// The given token's logit, and what says whether it counts: read at once and looked at last, so that nothing waits for them
// one after the other.
template <class T>
struct Given {
  typename T::type x = (typename T::type)0;
  uint32_t bits = 0;
  __device__ inline float logit() const { return bits & 1u ? T::wide(x) : kNoLogit; }
};
template <class T>
__device__ inline Given<T> given_logit(const Rows &a, uint32_t r, int32_t token) {
  Given<T> g;
  if (!a.token) return g;
  const uint32_t t = min((uint32_t)token, a.n_vocab - 1);
  g.x = ((const typename T::type VL_GLOBAL *)(a.logits + (uint64_t)r * a.ld))[t];
  g.bits = a.mask ? (uint32_t)a.mask[(uint64_t)r * a.mask_ld + (t >> 3)] >> (t & 7) : 1u;
  if (t != (uint32_t)token) g.bits = 0;
  return g;
}

// Short rows of which few alternatives are asked for, if any: 16 or 32 lanes per row, kChunks chunks per lane, so that a wavefront's
// instructions for the reductions and the results serve four rows or two, whose loads are on their way at once.  Alternatives are
// found one by one: the largest logit's first place, then the largest of the others.
template <class T, uint32_t kTeam, uint32_t kChunks, bool kTop>
__global__ __launch_bounds__(kThreads) void k_scores_few_lanes(Rows a, Scores out) {
  constexpr uint32_t kTeams = kThreads / kTeam;
  const uint32_t lane = threadIdx.x % kTeam;
  auto fold = [](float x, auto f) {
    x = quarter_fold(x, f);
    return kTeam == 32 ? f(x, __shfl_xor(x, 16, 64)) : x;
  };
  for (uint32_t first = blockIdx.x * kTeams; first < a.n_row; first += gridDim.x * kTeams) {
    const uint32_t r = first + threadIdx.x / kTeam;
    if (r >= a.n_row) break;
    const uint8_t VL_GLOBAL *row = a.logits + (uint64_t)r * a.ld;
    const uint8_t VL_GLOBAL *mask = a.mask ? a.mask + (uint64_t)r * a.mask_ld : nullptr;
    const int32_t token = a.token ? a.token[r] : 0;
    float x[kChunks][T::kElems];
    uint32_t bits[kChunks];
    load_row<T, kTeam, kChunks>(a, row, mask, lane, x, bits);
    const Given<T> given = given_logit<T>(a, r, token);
#pragma unroll
    for (uint32_t i = 0; i < kChunks; ++i)
      if (mask) keep_allowed<T>(x[i], bits[i]);
    float m = kNoLogit;
#pragma unroll
    for (uint32_t i = 0; i < kChunks; ++i)
#pragma unroll
      for (uint32_t j = 0; j < T::kElems; ++j) m = fmaxf(m, x[i][j]);
    Sums sums = {fold(m, [](float u, float v) { return fmaxf(u, v); }), 0.0f, 0.0f};
    const float ref = ref_of(sums.m);
#pragma unroll
    for (uint32_t i = 0; i < kChunks; ++i)
#pragma unroll
      for (uint32_t j = 0; j < T::kElems; ++j) {
        const float z = (x[i][j] - ref) * a.scale2, e = __builtin_amdgcn_exp2f(z);
        sums.s += e;
        sums.y += e * fmaxf(z, kFar);
      }
    auto add = [](float u, float v) { return u + v; };
    sums.s = fold(sums.s, add);
    sums.y = fold(sums.y, add);
    if (token < 0) {
      write_padding(out, r, lane);
      continue;
    }
    const Final f = finish(a, out, r, sums, given.logit(), lane == 0);
    if constexpr (kTop) {
      m = sums.m;
      for (uint32_t k = 0; ; ++k) {
        uint32_t at = kShortChunks * T::kElems;   // of this lane's logits the first of this size; places counted from the lane's first
#pragma unroll
        for (int32_t i = kChunks - 1; i >= 0; --i)
#pragma unroll
          for (int32_t j = T::kElems - 1; j >= 0; --j) at = x[i][j] == m ? i * kTeam * T::kElems + j : at;
        // (floats hold such places)
        const uint32_t place = (uint32_t)fold((float)(at + lane * T::kElems), [](float u, float v) { return fminf(u, v); });
        if (lane == 0) write_top<T>(out, r, k, m == kNoLogit ? 0ull : key_of(ordered<T>(m), place), f);
        if (k + 1 == out.n_top) break;
        m = kNoLogit;
        at = place - lane * T::kElems;
#pragma unroll
        for (uint32_t i = 0; i < kChunks; ++i)
#pragma unroll
          for (uint32_t j = 0; j < T::kElems; ++j) {
            if (at == i * kTeam * T::kElems + j) x[i][j] = kNoLogit;
            m = fmaxf(m, x[i][j]);
          }
        m = fold(m, [](float u, float v) { return fmaxf(u, v); });
      }
    }
  }
}

// Short rows: a wavefront per row, kChunks chunks per lane, all in registers.
template <class T, uint32_t kChunks>
__global__ __launch_bounds__(kThreads) void k_scores_short(Rows a, Scores out) {
  __shared__ uint64_t room[kWaves][64];
  const uint32_t lane = threadIdx.x & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (uint32_t r = blockIdx.x * kWaves + wave; r < a.n_row; r += gridDim.x * kWaves) {
    const uint8_t VL_GLOBAL *row = a.logits + (uint64_t)r * a.ld;
    const uint8_t VL_GLOBAL *mask = a.mask ? a.mask + (uint64_t)r * a.mask_ld : nullptr;
    const int32_t token = a.token ? a.token[r] : 0;
    if (token < 0) {
      write_padding(out, r, lane);
      continue;
    }
    float x[kChunks][T::kElems];
    uint32_t bits[kChunks];
    load_row<T, 64, kChunks>(a, row, mask, lane, x, bits);
    const Given<T> given = given_logit<T>(a, r, token);
#pragma unroll
    for (uint32_t i = 0; i < kChunks; ++i)
      if (mask) keep_allowed<T>(x[i], bits[i]);
    float m = kNoLogit;
    uint32_t place = 0;
#pragma unroll
    for (uint32_t i = 0; i < kChunks; ++i) {
      float b = x[i][0];
#pragma unroll
      for (uint32_t j = 1; j < T::kElems; ++j) b = fmaxf(b, x[i][j]);
      if (b > m) place = lane + 64 * i;
      m = fmaxf(m, b);
    }
    Sums sums = {wave_max(m), 0.0f, 0.0f};
    const float ref = ref_of(sums.m);
#pragma unroll
    for (uint32_t i = 0; i < kChunks; ++i)
#pragma unroll
      for (uint32_t j = 0; j < T::kElems; ++j) {
        const float z = (x[i][j] - ref) * a.scale2, e = __builtin_amdgcn_exp2f(z);
        sums.s += e;
        sums.y += e * fmaxf(z, kFar);
      }
    sums.s = wave_sum(sums.s);
    if (out.entropy) sums.y = wave_sum(sums.y);
    const Final f = finish(a, out, r, sums, given.logit(), lane == 0);
    if (out.n_top) {
      const uint32_t n = out.n_top;
      const uint64_t key = m == kNoLogit ? 0ull : key_of(ordered<T>(m), place);
      const uint64_t least = nth_key<T::kBits>(key, bits_for(64 * kChunks - 1), n, n + kMoreHot);
      // gathered in the order of the lanes; up to 64 of them, usual unless many are equal, one per lane
      uint32_t found = 0;
      room[wave][lane] = 0;
#pragma unroll
      for (uint32_t i = 0; i < kChunks; ++i)
        each_candidate<T>(x[i], 0, lane + 64 * i, least, [&](bool is, auto key_at) {
          const uint64_t all = __ballot(is);
          if (!all) return;
          const uint32_t at = found + lanes_below(all);
          if (is && at < 64) room[wave][at] = key_at();
          found += __popcll(all);
        });
      if (found <= 64) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (written and read by one wavefront)
        const uint64_t mine = room[wave][lane];
        const uint32_t rank = rank_of(room[wave], found, mine);
        if (lane < found && rank < n) write_top<T>(out, r, rank, mine, f);
        if (lane >= found && lane < n) write_top<T>(out, r, lane, 0, f);
      } else {
        List list;
#pragma unroll
        for (uint32_t i = 0; i < kChunks; ++i)
          each_candidate<T>(x[i], 0, lane + 64 * i, least, [&](bool is, auto key_at) { list.insert_lanes(key_at(), is, n); });
        if (lane < n) write_top<T>(out, r, lane, list.key, f);
      }
    }
  }
}

// What a part of a row leaves for the join: its sums and n_top keys, best first.
typedef float Part __attribute__((ext_vector_type(4)));

template <uint32_t kTeam>
struct Shared {
  Sums sums[kTeam / 64];
  float token[kTeam / 64];
  Room<kTeam> room;
  uint64_t key[kTeam < 64 ? 64 : kTeam];
  uint64_t list[kTeam / 64 * VL_MAX_TOP];   // (a multiple of four long)
  uint64_t least;
  uint32_t n_hot, hot[kTeam];
};

// The n best of `found` different keys, no more than there are threads, best first: entry k in thread k < n, 0 where there are fewer.  (Lists
// for rank_of: the wavefronts' lists are 4 n or 16 n keys, a single one n and zeros.)
__device__ inline uint64_t in_order(const uint64_t *keys, uint32_t found, uint64_t *out, uint32_t n) {
  const uint64_t mine = threadIdx.x < found ? keys[threadIdx.x] : 0ull;
  if (threadIdx.x < found && mine) {
    const uint32_t rank = rank_of(keys, found, mine);
    if (rank < n) out[rank] = mine;
  }
  __syncthreads();
  return threadIdx.x < n && threadIdx.x < found ? out[threadIdx.x] : 0ull;
}
// the same of the wavefronts' lists
template <uint32_t kTeam>
__device__ inline uint64_t join_lists(Shared<kTeam> &sh, const List &list, uint32_t n) {
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
  if (lane < n) sh.list[wave * n + lane] = list.key;
  if (kTeam == 64 && lane >= n && lane < VL_MAX_TOP) sh.list[lane] = 0;
  if (threadIdx.x < n) sh.key[threadIdx.x] = 0;   // (done with by now)
  __syncthreads();
  return in_order(sh.list, kTeam / 64 * n, sh.key, n);
}
// A key that n of the threads' best, `mine`, reach, and not many more
template <class T, uint32_t kTeam>
__device__ inline uint64_t least_of_interest(Shared<kTeam> &sh, uint64_t mine, uint32_t place_bits, uint32_t n) {
  sh.key[threadIdx.x] = mine;
  if (threadIdx.x < sh.room.kMost) sh.room.key[threadIdx.x] = 0;
  if (threadIdx.x == 0) sh.n_hot = sh.room.n = 0;
  __syncthreads();
  if (threadIdx.x < 64) {   // of several threads' best the best one: a key that n of these 64 reach serves as well
    uint64_t k = 0;
#pragma unroll
    for (uint32_t i = 0; i < kTeam / 64; ++i) k = sh.key[threadIdx.x + 64 * i] > k ? sh.key[threadIdx.x + 64 * i] : k;
    const uint64_t least = nth_key<T::kBits>(k, place_bits, n, n + kMoreHot);
    if (threadIdx.x == 0) sh.least = least;
  }
  __syncthreads();
  return sh.least;
}

// The sums of all of a workgroup's threads.  With kOne `token`, of each thread the first token of its largest logit, becomes the first of
// the largest of all.  (Tokens are below 2^24: floats hold them.)
constexpr float kBehind = 0x1p24f;
template <uint32_t kTeam, bool kOne = false>
__device__ inline Sums join_sums(Shared<kTeam> &sh, Sums mine, float scale2, float *token = nullptr) {
  auto add = [](float u, float v) { return u + v; };
  auto lower = [](float u, float v) { return fminf(u, v); };
  const float most = wave_max(mine.m);
  if (kOne) *token = wave_fold(mine.m == most ? *token : kBehind, kBehind, lower);
  mine = rebase(mine, most, scale2);
  mine.s = wave_sum(mine.s);
  mine.y = wave_sum(mine.y);
  if constexpr (kTeam == 64) return mine;
  if ((threadIdx.x & 63u) == 0) {
    sh.sums[threadIdx.x >> 6] = mine;
    if (kOne) sh.token[threadIdx.x >> 6] = *token;
  }
  __syncthreads();
  const uint32_t w = threadIdx.x & 15u;   // (16 wavefronts at most)
  mine = w < kTeam / 64 ? sh.sums[w] : Sums{kNoLogit, 0.0f, 0.0f};
  const float best = quarter_fold(mine.m, [](float u, float v) { return fmaxf(u, v); });
  if (kOne) *token = quarter_fold(w < kTeam / 64 && mine.m == best ? sh.token[w] : kBehind, lower);
  mine = rebase(mine, best, scale2);
  mine.s = quarter_fold(mine.s, add);
  mine.y = quarter_fold(mine.y, add);
  return mine;
}


// what is asked for: alternatives too, just one, or sums alone; and whether nothing of the logits is kept in the caches
enum Kind { kWithTop, kWithTopOnce, kWithOne, kWithOneOnce, kSums, kSumsOnce };
constexpr uint32_t kFewChunks = 4;

// Long rows: a workgroup of kTeam threads per row or part of a row.  Thread t takes the part's chunks t, t + kTeam, t + 2 kTeam, ...
// kN chunks of a lane are on their way at once.  If one alternative is asked for, a lane keeps its best chunk in registers.
template <class T, uint32_t kTeam, uint32_t kN, bool kMask, Kind kKind>
__global__ __launch_bounds__(kTeam, kTeam == 1024 && kN == 2 ? 8 : 1) void k_scores_long(Rows a, Scores out, uint32_t part_chunks, Part VL_GLOBAL *parts, uint64_t VL_GLOBAL *part_keys) {
  __shared__ Shared<kTeam> sh;
  constexpr bool kTop = kKind == kWithTop || kKind == kWithTopOnce, kOne = kKind == kWithOne || kKind == kWithOneOnce;
  constexpr bool kOnce = kKind == kWithTopOnce || kKind == kWithOneOnce || kKind == kSumsOnce;
  const uint32_t c0 = blockIdx.x * part_chunks, n_top = kTop ? out.n_top : 0;
  for (uint32_t r = blockIdx.y; r < a.n_row; r += gridDim.y) {
    const uint8_t VL_GLOBAL *row = a.logits + (uint64_t)r * a.ld;
    const uint8_t VL_GLOBAL *mask = kMask ? a.mask + (uint64_t)r * a.mask_ld : nullptr;
    const int32_t token = a.token ? a.token[r] : 0;
    if (token < 0) {
      if (!parts) write_padding(out, r, threadIdx.x);
      continue;
    }
    const uint32_t lead = lead_of<T>(row), n_full = (a.n_vocab + lead) / T::kElems, n_chunk = (a.n_vocab + lead + T::kElems - 1) / T::kElems;
    const uint32_t c1 = min(n_chunk, c0 + part_chunks), c1_full = min(n_full, c1);
    const Given<T> given = parts ? Given<T>{} : given_logit<T>(a, r, token);
    Sums sums = {kNoLogit, 0.0f, 0.0f};
    uint32_t place = 0;        // the chunk that sums.m came from
    float second = kNoLogit;   // the largest logit of the other chunks
    u32x4 kept = {T::kNone, T::kNone, T::kNone, T::kNone};   // that chunk
    uint32_t kept_bits = 0;
    // kHere chunks of this lane from c on, kTeam apart
    auto add = [&](auto n_of, const float (*x)[T::kElems], uint32_t c, const u32x4 *w, const uint32_t *bits) {
      constexpr uint32_t kHere = decltype(n_of)::value;
      float b[kHere], m = kNoLogit;
#pragma unroll
      for (uint32_t u = 0; u < kHere; ++u) {
        b[u] = x[u][0];
#pragma unroll
        for (uint32_t j = 1; j < T::kElems; ++j) b[u] = fmaxf(b[u], x[u][j]);
        m = fmaxf(m, b[u]);
      }
      if (kTop || kOne) {
        float best = sums.m;
#pragma unroll
        for (uint32_t u = 0; u < kHere; ++u) {
          if (kTop) second = __builtin_amdgcn_fmed3f(best, second, b[u]);   // (second <= best)
          place = b[u] > best ? c + u * kTeam : place;
          if (kOne) {
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) kept[j] = b[u] > best ? w[u][j] : kept[j];
            if (kMask) kept_bits = b[u] > best ? bits[u] : kept_bits;
          }
          best = fmaxf(best, b[u]);
        }
      }
      sums = rebase(sums, fmaxf(sums.m, m), a.scale2);
      const float ref = ref_of(sums.m);
      float s = 0.0f, y = 0.0f;   // (of these chunks, so that long rows are not added up one by one)
#pragma unroll
      for (uint32_t u = 0; u < kHere; ++u)
#pragma unroll
        for (uint32_t j = 0; j < T::kElems; ++j) {
          const float z = (x[u][j] - ref) * a.scale2, e = __builtin_amdgcn_exp2f(z);
          s += e;
          y += e * fmaxf(z, kFar);
        }
      sums.s += s;
      sums.y += y;
    };
    for (uint32_t c = c0 + threadIdx.x; c - threadIdx.x < c1_full; c += kN * kTeam) {
      u32x4 w[kN];
      uint32_t bits[kN];
      if (c - threadIdx.x + kN * kTeam <= c1_full) {
#pragma unroll
        for (uint32_t u = 0; u < kN; ++u) w[u] = kOnce ? load_once<T>(row, lead, c + u * kTeam) : load_even<T>(row, lead, c + u * kTeam);
        if (kMask) {
#pragma unroll
          for (uint32_t u = 0; u < kN; ++u) bits[u] = mask_bits<T>(mask, lead, c + u * kTeam);
        }
      } else {
#pragma unroll
        for (uint32_t u = 0; u < kN; ++u) {
          const bool in = c + u * kTeam < c1_full;
          w[u] = u32x4{T::kNone, T::kNone, T::kNone, T::kNone};
          bits[u] = 0;
          if (in) w[u] = load_even<T>(row, lead, c + u * kTeam);
          if (kMask && in) bits[u] = mask_bits<T>(mask, lead, c + u * kTeam);
        }
      }
      float x[kN][T::kElems];
#pragma unroll
      for (uint32_t u = 0; u < kN; ++u) {
        T::unpack(w[u], x[u]);
        if (kMask) keep_allowed<T>(x[u], bits[u]);
      }
      if (lead > c) x[0][0] = kNoLogit;
      add(std::integral_constant<uint32_t, kN>{}, x, c, w, bits);
    }
    if (c0 <= n_full && n_full < c1 && threadIdx.x == (n_full - c0) % kTeam) {   // the chunk that the row's end cuts
      float x[1][T::kElems];
      load_any<T>(a, row, mask, lead, n_full, x[0]);
      const u32x4 w = kOne ? T::pack(x[0]) : u32x4{};   // (as it was: these are the type's own values)
      const uint32_t bits = ~0u;
      add(std::integral_constant<uint32_t, 1>{}, x, n_full, &w, &bits);
    }
    const float mine = sums.m;
    float first = kBehind;
    if constexpr (kOne) {
      float x[T::kElems];
      T::unpack(kept, x);
      if (kMask) keep_allowed<T>(x, kept_bits);
      if (lead > place) x[0] = kNoLogit;
      uint32_t at = 0;
#pragma unroll
      for (int32_t j = T::kElems - 1; j >= 0; --j) at = x[j] == mine ? j : at;
      first = (float)(int32_t)(place * T::kElems - lead + at);
    }
    sums = join_sums<kTeam, kOne>(sh, sums, a.scale2, &first);
    Final f = {};
    if (!parts) f = finish(a, out, r, sums, given.logit(), threadIdx.x == 0);
    else if (threadIdx.x == 0) parts[(uint64_t)r * gridDim.x + blockIdx.x] = Part{sums.m, sums.s, sums.y, 0.0f};
    if (kOne && threadIdx.x == 0) {
      const uint64_t best = sums.m == kNoLogit ? 0ull : key_of(ordered<T>(sums.m), (uint32_t)first);
      if (!parts) write_top<T>(out, r, 0, best, f);
      else part_keys[(uint64_t)r * gridDim.x + blockIdx.x] = best;
    }
    if (n_top) {
      const uint64_t key = mine == kNoLogit ? 0ull : key_of(ordered<T>(mine), place), least = least_of_interest<T>(sh, key, bits_for(n_chunk), n_top);
      const bool hot = key >= least;
      const uint32_t each = (c1 - c0 + kTeam - 1) / kTeam;
      const bool own = each > kFewChunks;   // (fewer: all chunks of all hot threads at once)
      if (hot && !own) sh.hot[atomicAdd(&sh.n_hot, 1u)] = threadIdx.x;
      if (hot && own) {
        float x[T::kElems];
        load_any<T>(a, row, mask, lead, place, x);
        each_candidate<T>(x, lead, place, least, [&](bool is, auto key_at) { if (is) gather(sh.room, key_at()); });
        if (second != kNoLogit && ordered<T>(second) >= (uint32_t)(least >> 32)) sh.hot[atomicAdd(&sh.n_hot, 1u)] = threadIdx.x;
      }
      __syncthreads();
      // the (other) chunks of hot threads that have more to offer, dealt out to all
      const uint32_t n_hot = sh.n_hot;
      for (uint32_t i = threadIdx.x; i < n_hot * each; i += kTeam) {
        const uint32_t turn = i / n_hot, who = sh.hot[i - turn * n_hot], at = c0 + who + turn * kTeam;
        if (at >= c1 || (own && at == (uint32_t)~sh.key[who])) continue;
        float x[T::kElems];
        load_any<T>(a, row, mask, lead, at, x);
        each_candidate<T>(x, lead, at, least, [&](bool is, auto key_at) { if (is) gather(sh.room, key_at()); });
      }
      if (n_hot) __syncthreads();
      uint64_t best;
      if (sh.room.n <= sh.room.kMost) {
        best = in_order(sh.room.key, sh.room.n, sh.key, n_top);
      } else {
        const uint32_t lane = threadIdx.x & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        List list;
        for (uint64_t all = __ballot(hot); all; all &= all - 1) {   // this wavefront's hot threads, all their chunks
          const uint32_t from = c0 + wave * 64 + (uint32_t)__builtin_ctzll(all);
          for (uint32_t base = from; base < c1; base += 64 * kTeam) {
            const uint32_t at = base + lane * kTeam;
            float x[T::kElems];
            if (at < c1) {
              load_any<T>(a, row, mask, lead, at, x);
            } else {
#pragma unroll
              for (uint32_t j = 0; j < T::kElems; ++j) x[j] = kNoLogit;
            }
            each_candidate<T>(x, lead, at, least, [&](bool is, auto key_at) { list.insert_lanes(key_at(), is, n_top); });
          }
        }
        best = join_lists(sh, list, n_top);
      }
      if (threadIdx.x < n_top) {
        if (!parts) write_top<T>(out, r, threadIdx.x, best, f);
        else part_keys[((uint64_t)r * gridDim.x + blockIdx.x) * n_top + threadIdx.x] = best;
      }
    }
    __syncthreads();   // (sh is used again)
  }
}

// The parts of a row as one: a workgroup per row.
template <class T>
__global__ __launch_bounds__(kThreads) void k_scores_join(Rows a, Scores out, uint32_t n_part, const Part VL_GLOBAL *parts, const uint64_t VL_GLOBAL *part_keys) {
  __shared__ Shared<kThreads> sh;
  const uint32_t lane = threadIdx.x & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n_top = out.n_top;
  for (uint32_t r = blockIdx.x; r < a.n_row; r += gridDim.x) {
    const int32_t token = a.token ? a.token[r] : 0;
    if (token < 0) {
      write_padding(out, r, threadIdx.x);
      continue;
    }
    const Given<T> given = given_logit<T>(a, r, token);
    const uint64_t VL_GLOBAL *keys = part_keys + (uint64_t)r * n_part * n_top;
    uint64_t mine = 0;   // this thread's best of the parts' keys
    for (uint32_t i = threadIdx.x; i < n_part * n_top; i += kThreads) mine = keys[i] > mine ? keys[i] : mine;
    float first = (float)~(uint32_t)mine;   // (if there is one key per part)
    Sums sums = {kNoLogit, 0.0f, 0.0f};
    if (threadIdx.x < n_part) {   // (never more than there are threads)
      const Part p = parts[(uint64_t)r * n_part + threadIdx.x];
      sums = Sums{p.x, p.y, p.z};
    }
    sums = join_sums<kThreads, true>(sh, sums, a.scale2, &first);
    const Final f = finish(a, out, r, sums, given.logit(), threadIdx.x == 0);
    if (n_top == 1) {
      if (threadIdx.x == 0) write_top<T>(out, r, 0, sums.m == kNoLogit ? 0ull : key_of(ordered<T>(sums.m), (uint32_t)first), f);
    } else if (n_top) {
      // the keys that n of the threads' best reach
      const uint64_t least = least_of_interest<T>(sh, mine, bits_for(a.n_vocab), n_top);
      if (mine >= least) {
        for (uint32_t i = threadIdx.x; i < n_part * n_top; i += kThreads) {
          const uint64_t k = keys[i];
          if (k >= least) gather(sh.room, k);
        }
      }
      __syncthreads();
      // (The bound is one of columns of kWaves threads: n_top + kMoreHot of the 64 reach `least`, so up to kWaves times as many threads, each
      // with n_part * n_top / kThreads keys or one more.  Where that is more than there is room for, insertion finds the best.)
      uint64_t best;
      if (sh.room.n <= sh.room.kMost) {
        best = in_order(sh.room.key, sh.room.n, sh.key, n_top);
      } else {
        List list;
        for (uint32_t p = wave; p < n_part; p += kWaves) {
          const uint64_t k = lane < n_top ? keys[(uint64_t)p * n_top + lane] : 0ull;
          list.insert_lanes(k, k >= least, n_top);
        }
        best = join_lists(sh, list, n_top);
      }
      if (threadIdx.x < n_top) write_top<T>(out, r, threadIdx.x, best, f);
    }
    __syncthreads();
  }
}

// ---- the gradient
struct Grad {
  const float VL_GLOBAL *stat, *entropy, *g_logprob, *g_entropy;
  uint8_t VL_GLOBAL *grad;
  uint64_t ld;   // in bytes
};
// What a row's elements need: with t = log2 p, d = p (t * slope + level), and `hot` more at the given token.
struct GradRow { float ref, log2_sum, slope, level, hot; uint32_t token; bool idle; };
__device__ inline GradRow grad_row(const Rows &a, const Grad &b, uint32_t r) {
  GradRow g = {};
  const int32_t token = a.token ? a.token[r] : 0;
  const float m = b.stat[2ull * r], log_sum = b.stat[2ull * r + 1];
  g.idle = token < 0 || m == kNoLogit;
  if (g.idle) return g;
  g.ref = m;
  g.log2_sum = log_sum * kLog2e;
  const float gl = b.g_logprob ? b.g_logprob[r] : 0.0f, e = b.g_entropy ? b.g_entropy[r] : 0.0f;
  const float h = b.g_entropy ? b.entropy[r] : 0.0f;
  g.slope = -a.scale * e * kLn2;
  g.level = -a.scale * (gl + e * h);
  g.hot = b.g_logprob ? gl * a.scale : 0.0f;
  g.token = b.g_logprob ? (uint32_t)token : kNone;
  return g;
}
template <class T>
__device__ inline void grad_chunk(const Rows &a, const GradRow &g, uint32_t lead, uint32_t c, float *x, uint32_t bits, bool masked) {
#pragma unroll
  for (uint32_t j = 0; j < T::kElems; ++j) {
    const float t = __builtin_fmaf(x[j] - g.ref, a.scale2, -g.log2_sum), p = __builtin_amdgcn_exp2f(t);
    x[j] = p * __builtin_fmaf(fmaxf(t, kFar), g.slope, g.level);
  }
  const uint32_t place = g.token + lead;
  if (place / T::kElems == c) {
#pragma unroll
    for (uint32_t j = 0; j < T::kElems; ++j) x[j] += place % T::kElems == j ? g.hot : 0.0f;
  }
  if (masked) {   // 0 where not allowed, whatever stood there
#pragma unroll
    for (uint32_t j = 0; j < T::kElems; ++j)
      x[j] = as_float(as_word(x[j]) & (uint32_t)((int32_t)(bits << (31 - j)) >> 31));
  }
}
// (not kept in the caches of a die, which others could not use: 25,600 rows of 1,024 25.8 -> 22.4 us, 400 of 80,000 28.1 -> 22.3, 8,192 of
// 131,072 745 -> 733; but 100 of 2,900 3.7 -> 4.0)
template <class T>
__device__ inline void store_any(const Rows &a, uint8_t VL_GLOBAL *to, uint32_t c, const float *x) {
  const uint32_t from = c * T::kElems;
  if (from + T::kElems <= a.n_vocab) {
    __builtin_nontemporal_store(T::pack(x), (typename T::chunk VL_GLOBAL *)(to + (uint64_t)c * 16));
  } else {
#pragma unroll
    for (uint32_t j = 0; j < T::kElems; ++j)
      if (from + j < a.n_vocab) ((typename T::type VL_GLOBAL *)to)[from + j] = T::narrow(x[j]);
  }
}

// Short rows: kTeam lanes per row, eight workgroups per compute unit.  (25,600 rows of 512 logits, 64 chunks: 16 and 32 lanes 12.7 us, 64
// 14.5; as many workgroups as it takes 13.3.)
template <class T, uint32_t kTeam, uint32_t kChunks>
__global__ __launch_bounds__(kThreads) void k_grad_short(Rows a, Grad b) {
  constexpr uint32_t kTeams = kThreads / kTeam;
  const uint32_t lane = threadIdx.x % kTeam, team = kTeam == 64 ? (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x / kTeam) : threadIdx.x / kTeam;
  for (uint32_t first = blockIdx.x * kTeams; first < a.n_row; first += gridDim.x * kTeams) {
    const uint32_t r = first + team;
    if (r >= a.n_row) break;
    const uint8_t VL_GLOBAL *row = a.logits + (uint64_t)r * a.ld;
    uint8_t VL_GLOBAL *to = b.grad + (uint64_t)r * b.ld;
    const uint8_t VL_GLOBAL *mask = a.mask ? a.mask + (uint64_t)r * a.mask_ld : nullptr;
    float x[kChunks][T::kElems];
    uint32_t bits[kChunks];
    load_row<T, kTeam, kChunks>(a, row, mask, lane, x, bits);
    const GradRow g = grad_row(a, b, r);
#pragma unroll
    for (uint32_t i = 0; i < kChunks; ++i) {
      grad_chunk<T>(a, g, 0, lane + kTeam * i, x[i], bits[i], mask != nullptr);
#pragma unroll
      for (uint32_t j = 0; j < T::kElems; ++j) x[i][j] = g.idle ? 0.0f : x[i][j];
      store_any<T>(a, to, lane + kTeam * i, x[i]);
    }
  }
}

// Long rows: a workgroup per piece of a row, of kBatch chunks for each thread, all on their way at once.  kOnce: the logits are not kept in the caches.
template <class T, bool kMask, bool kOnce, uint32_t kBatch>
__global__ __launch_bounds__(kThreads) void k_grad_long(Rows a, Grad b) {
  constexpr uint32_t piece_chunks = kBatch * kThreads;
  typedef typename T::chunk chunk;
  const uint32_t c0 = blockIdx.x * piece_chunks, c = c0 + threadIdx.x;
  for (uint32_t r = blockIdx.y; r < a.n_row; r += gridDim.y) {
    const uint8_t VL_GLOBAL *row = a.logits + (uint64_t)r * a.ld;
    uint8_t VL_GLOBAL *to = b.grad + (uint64_t)r * b.ld;
    const uint8_t VL_GLOBAL *mask = kMask ? a.mask + (uint64_t)r * a.mask_ld : nullptr;
    const GradRow g = grad_row(a, b, r);
    // (chunks from the even place in front, if that suits both: 4,096 bf16 rows of 50,001 151 -> 142 us, 25,600 of 20,011 392 -> 359)
    const uint32_t lead = lead_of<T>(row) == lead_of<T>(to) ? lead_of<T>(row) : 0u;
    const uint32_t n_full = (a.n_vocab + lead) / T::kElems, n_chunk = (a.n_vocab + lead + T::kElems - 1) / T::kElems;
    const uint32_t c1 = min(n_chunk, c0 + piece_chunks), c1_full = min(n_full, c1);
    if (g.idle) {
      float x[T::kElems] = {};
      for (uint32_t at = c; at < c1; at += kThreads) store_any<T>(a, to, at, x);
      continue;
    }
    row -= lead * 2;
    to -= lead * 2;
    u32x4 w[kBatch];
    uint32_t bits[kBatch];
    const bool all = c0 + piece_chunks <= c1_full;
#pragma unroll
    for (uint32_t u = 0; u < kBatch; ++u) {
      w[u] = u32x4{};
      if (all || c + u * kThreads < c1_full) w[u] = kOnce ? load_once<T>(row, c + u * kThreads) : load_chunk<T>(row, c + u * kThreads);
    }
#pragma unroll
    for (uint32_t u = 0; u < kBatch; ++u) {
      bits[u] = 0;
      if (kMask && (all || c + u * kThreads < c1_full)) bits[u] = mask_bits<T>(mask, lead, c + u * kThreads);
    }
#pragma unroll
    for (uint32_t u = 0; u < kBatch; ++u) {
      const uint32_t at = c + u * kThreads;
      if (!all && at >= c1_full) break;
      float x[T::kElems];
      T::unpack(w[u], x);
      grad_chunk<T>(a, g, lead, at, x, bits[u], kMask);
      if (lead > at) {   // (what stands in front of the row stays)
        for (uint32_t j = 1; j < T::kElems; ++j) ((typename T::type VL_GLOBAL *)to)[j] = T::narrow(x[j]);
      } else {
        __builtin_nontemporal_store(T::pack(x), (chunk VL_GLOBAL *)(to + (uint64_t)at * 16));
      }
    }
    if (c0 <= n_full && n_full < c1 && threadIdx.x == (n_full - c0) % kThreads) {   // the chunk that the row's end cuts
      float x[T::kElems];
      load_any<T>(a, row + lead * 2, nullptr, lead, n_full, x);
      grad_chunk<T>(a, g, lead, n_full, x, 0, false);
#pragma unroll
      for (uint32_t j = 0; j < T::kElems; ++j) {
        const uint32_t t = n_full * T::kElems + j - lead;
        if (t >= a.n_vocab) continue;   // (behind the row, or in front of it)
        const bool allowed = !kMask || ((mask[t >> 3] >> (t & 7)) & 1);
        ((typename T::type VL_GLOBAL *)(to + lead * 2))[t] = T::narrow(allowed ? x[j] : 0.0f);
      }
    }
  }
}

// ---- host

constexpr uint32_t kMostRows = 0x7FFFFFFFu;
constexpr uint32_t kShortGradChunks = 256;
constexpr uint32_t kMostGridY = 65535;

uint32_t size_of(uint32_t type) { return type == VL_F32 ? 4u : 2u; }
uint32_t chunks_of(const vl_token_rows *a, bool lead = false) { const uint32_t e = 16u / size_of(a->type); return (a->n_vocab + lead + e - 1) / e; }
bool has_lead(const vl_token_rows *a) {   // some row starts at an odd place
  return a->type != VL_F32 && (((uintptr_t)a->logits & 2) || (a->n_row > 1 && (a->ld & 1)));
}

int32_t check_rows(const vl_token_rows *a) {
  if (!a || !a->logits) return VL_E_NULL;
  if (a->type > VL_BF16) return VL_E_RANGE;
  if (a->n_vocab == 0 || a->n_vocab > VL_MAX_VOCAB || !(a->scale >= VL_MIN_SCALE) || a->scale > 1.0f / VL_MIN_SCALE) return VL_E_RANGE;
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
  return Rows{(const uint8_t VL_GLOBAL *)a->logits, a->ld * size_of(a->type), (const uint8_t VL_GLOBAL *)a->mask, a->mask_ld * 4,
              (const int32_t VL_CONSTANT *)a->token, a->n_row, a->n_vocab, a->scale, (float)((double)a->scale * 1.4426950408889634)};
}

// How many threads a workgroup has, how many workgroups share a row, and how many chunks each takes.  A wavefront per row where it is short
// or there are rows for all wavefronts (with alternatives, which are found in a share of the row that falls with the threads, not if
// it is very long); more threads the longer the row and the fewer rows there are; and parts, which a second launch joins, where few
// rows are too long for one workgroup.  Measured, us (this choice / the others), bf16 logits:
//   1,000 x 2,000: 64 threads 3.9 / 256 5.2, 1,024 8.8; five alternatives 6.1 / 8.4, 16.3
//   600 x 4,000: 64 4.5 / 256 4.8, 1,024 7.3;                          1 x 4,000: 256 3.4 / 64 3.8
//   3,000 x 5,000: 64 10.5 / 256 13.2;                                 4,096 x 20,000, twenty: 64 46 / 256 48
//   (4,096 x 50,001 in 32 bits, five, 12,501 chunks: 256 73.7 / 64 77.4)
//   1,000 x 16,000, five: 256 12.8 / 64 15.0, 1,024 17.9;              1 x 16,000: 256 4.2 / 1,024 4.6
//   500 x 32,000 in 32 bits, one: 256 14.8 / 1,024 15.9;               500 x 100,000: 1,024 24.2 / 256 26.9
//   150 x 32,000: 1,024 5.9 / 256 7.2, in 3 parts 9.2;                 1 x 32,000: 1,024 4.7 / 256 5.6
//   1 x 131,072, twenty: 256 in 21 parts 10.2 / in 32 10.6, 1,024 15.3; 60: 256 in 21 parts 15.0 / 1,024 16.5, 128: 1,024 16.7 / in 16 parts 19.6
// (between 60 rows and 128 neither side is measured)
struct Split { uint32_t team, parts, chunks; bool few; };   // few: a compute unit has one workgroup at most, which may use twice the registers
Split split_of(const vl_token_rows *a, uint32_t n_top, bool lead) {
  const uint32_t n = chunks_of(a, lead), rows = a->n_row;
  const bool few = rows <= 256;
  uint32_t team = 1024, parts = 1;
  if (n <= 256 || (n <= 512 && rows >= 600) || (rows >= 2048 && (n_top == 0 || n <= 8192))) team = 64;
  else if (n <= 2048 || rows > 512 || (!few && n <= 8192)) team = 256;
  else if (rows < 96 && n > 8192) { team = 256; parts = std::min({2048 / rows, n / 768, 256u}); }
  if (parts == 1) return Split{team, 1, n, few};
  const uint32_t chunks = ((n + parts - 1) / parts + team - 1) / team * team;
  return Split{team, (n + chunks - 1) / chunks, chunks, few};
}
uint64_t work_of(const vl_token_rows *a, const vl_token_scores *o) {
  if (chunks_of(a) <= kShortChunks) return 0;
  // enough wherever the rows start
  const uint32_t parts = std::max(split_of(a, o->n_top, false).parts, split_of(a, o->n_top, a->type != VL_F32).parts);
  return parts == 1 ? 0 : (uint64_t)a->n_row * parts * (sizeof(Part) + 8ull * o->n_top);
}

template <class T, uint32_t kTeam, uint32_t kN>
void launch_long(const Rows &a, const Scores &out, Split split, Part VL_GLOBAL *parts, uint64_t VL_GLOBAL *keys, hipStream_t stream) {
  const dim3 grid(split.parts, std::min(a.n_row, kMostGridY));
  // Logits beyond what the Infinity Cache holds (256 MB) are not kept in the caches: 1,500 rows of 131,072 77 -> 69 us,
  // 8,000 of 20,000 65 -> 56, with five alternatives 4,096 of 50,001 85 -> 82; but 64 MB that the program before has just written
  // 17.7 -> 19.9.
  auto launch = [&](auto with_top, auto with_one, auto sums) {
    constexpr Kind kTop = decltype(with_top)::value, kOne = decltype(with_one)::value, kNone = decltype(sums)::value;
    (a.mask ? out.n_top > 1 ? k_scores_long<T, kTeam, kN, true, kTop> : out.n_top ? k_scores_long<T, kTeam, kN, true, kOne> : k_scores_long<T, kTeam, kN, true, kNone>
            : out.n_top > 1 ? k_scores_long<T, kTeam, kN, false, kTop> : out.n_top ? k_scores_long<T, kTeam, kN, false, kOne> : k_scores_long<T, kTeam, kN, false, kNone>)
        <<<grid, kTeam, 0, stream>>>(a, out, split.chunks, parts, keys);
  };
  if constexpr (kTeam != 1024 || kN != 4) {   // (256 rows or fewer are seldom that much)
    if ((uint64_t)a.n_row * a.n_vocab * sizeof(typename T::type) > (256ull << 20)) {
      launch(std::integral_constant<Kind, kWithTopOnce>{}, std::integral_constant<Kind, kWithOneOnce>{}, std::integral_constant<Kind, kSumsOnce>{});
      return;
    }
  }
  launch(std::integral_constant<Kind, kWithTop>{}, std::integral_constant<Kind, kWithOne>{}, std::integral_constant<Kind, kSums>{});
}
template <class T>
void launch_scores(const Rows &a, const Scores &out, uint32_t n_chunk, Split split, void *work, hipStream_t stream) {
  // Short rows, few lanes each: no alternatives, or few enough.  25,600 bf16 rows, us this way / with a wavefront each and its search: of 512,
  // one alternative 10.3 / 16.8, two 12.7 / 17.2, four 17.6 / 17.8; of 128, one 4.8 / 15.0, eight 12.1 / 17.6; in 32 bits of
  // 256, four 12.8 / 15.9, eight 19.0 / 16.7.  An alternative more takes 0.35 to 0.85 us even of few rows, where the search's take
  // 0.05 (one alternative of 500 rows of 512 3.95 / 3.92, two 4.8 / 4.0; of 4,000 rows two 4.86 / 4.86; four of rows of 256, 4,000 of
  // them 5.0 / 5.0, 8,000 5.6 / 7.2; eight of rows of 128, 4,000 of them 5.6 / 5.3, 8,000 6.1 / 7.6).
  // (16 at most, as many as a row has lanes)
  const uint32_t held = (n_chunk <= 16 ? 1u : n_chunk <= 32 ? 2u : 4u) * T::kElems;   // logits of a lane
  if (n_chunk <= kShortChunks && (out.n_top <= 1 || (out.n_top * held <= 64 && a.n_row >= 512 * (out.n_top + 5)))) {
    // 16 lanes per row while a lane has at most 4 chunks, then 32.  25,600 bf16 rows of 512: 9.6 us with 16 lanes, 10.1 with
    // 32; rows of 1,024: 15.5 us with 16 lanes of 8 chunks, 12.5 with 32 of 4.
    const uint32_t teams = kThreads / (n_chunk <= 64 ? 16 : 32), blocks = std::min((a.n_row + teams - 1) / teams, 1u << 20);
    auto launch = [&](auto top) {
      constexpr bool kTop = decltype(top)::value;
      (n_chunk <= 16 ? k_scores_few_lanes<T, 16, 1, kTop> : n_chunk <= 32 ? k_scores_few_lanes<T, 16, 2, kTop> : n_chunk <= 64 ? k_scores_few_lanes<T, 16, 4, kTop> : k_scores_few_lanes<T, 32, 4, kTop>)
          <<<blocks, kThreads, 0, stream>>>(a, out);
    };
    if (out.n_top) launch(std::true_type{});
    else launch(std::false_type{});
    return;
  }
  if (n_chunk <= kShortChunks) {
    const uint32_t blocks = std::min((a.n_row + kWaves - 1) / kWaves, 1u << 20);
    (n_chunk <= 64 ? k_scores_short<T, 1> : k_scores_short<T, 2>)<<<blocks, kThreads, 0, stream>>>(a, out);
    return;
  }
  Part VL_GLOBAL *parts = split.parts > 1 ? (Part VL_GLOBAL *)work : nullptr;
  uint64_t VL_GLOBAL *keys = parts ? (uint64_t VL_GLOBAL *)((uint8_t *)work + (uint64_t)a.n_row * split.parts * sizeof(Part)) : nullptr;
  (split.team == 64 ? launch_long<T, 64, 4> : split.team == 256 ? launch_long<T, 256, 4> : split.few ? launch_long<T, 1024, 4> : launch_long<T, 1024, 2>)(a, out, split, parts, keys, stream);
  if (parts) k_scores_join<T><<<a.n_row, kThreads, 0, stream>>>(a, out, split.parts, parts, keys);
}

template <class T>
void launch_grad(const Rows &a, const Grad &b, uint32_t n_chunk, hipStream_t stream) {
  // (rows of 1,500 bf16 logits, us this way / in pieces: 100 rows 4.7 / 3.5, 1,000 5.1 / 4.6, 2,500 6.9 / 7.5, 25,600 34 / 59)
  if (n_chunk <= 128 || (n_chunk <= kShortGradChunks && a.n_row >= 2048)) {
    const uint32_t team = n_chunk <= 32 ? 16 : n_chunk <= 64 ? 32 : 64, teams = kThreads / team;
    (n_chunk <= 16 ? k_grad_short<T, 16, 1> : n_chunk <= 32 ? k_grad_short<T, 16, 2> : n_chunk <= 64 ? k_grad_short<T, 32, 2>
     : n_chunk <= 128 ? k_grad_short<T, 64, 2> : k_grad_short<T, 64, 4>)<<<std::min((a.n_row + teams - 1) / teams, 2048u), kThreads, 0, stream>>>(a, b);
    return;
  }
  // Two chunks per thread, four where a row is one piece then (us, this way / the other): 8,192 bf16 rows of 5,000 26.6 / 30.1, of 8,200 53.8 / 61.3, of
  // 131,072 670 / 735.  One chunk 930 there, three 783, eight 781.
  // Logits that with their gradient are more than the Infinity Cache holds (256 MB) are not kept in the caches: 4,096 rows of 50,001
  // in 32 bits 284 -> 269, 8,192 bf16 rows of 12,000 69.6 -> 67.7; but 2,000 of 20,000 (160 MB) 26.9 -> 30.4.
  const bool lead = T::kElems == 8 && (((uintptr_t)a.logits | (a.n_row > 1 ? a.ld : 0)) & 2);   // some row starts at an odd place
  const uint32_t n_most = (a.n_vocab + lead + T::kElems - 1) / T::kElems;
  const bool once = 2ull * a.n_row * a.n_vocab * sizeof(typename T::type) > (256ull << 20);
  auto launch = [&](auto batch) {
    constexpr uint32_t kBatch = decltype(batch)::value;
    const dim3 grid((n_most + kBatch * kThreads - 1) / (kBatch * kThreads), std::min(a.n_row, kMostGridY));
    (a.mask ? once ? k_grad_long<T, true, true, kBatch> : k_grad_long<T, true, false, kBatch> : once ? k_grad_long<T, false, true, kBatch> : k_grad_long<T, false, false, kBatch>)
        <<<grid, kThreads, 0, stream>>>(a, b);
  };
  if (n_chunk > 2 * kThreads && n_chunk <= 4 * kThreads) launch(std::integral_constant<uint32_t, 4>{});
  else launch(std::integral_constant<uint32_t, 2>{});
}

}  // namespace

extern "C" int32_t vl_token_logprobs_work(const vl_token_rows *rows, const vl_token_scores *out, uint64_t *bytes) {
  if (!bytes) return VL_E_NULL;
  const int32_t rc = check_scores(rows, out);
  if (rc == VL_OK) *bytes = work_of(rows, out);
  return rc;
}

extern "C" int32_t vl_token_logprobs(const vl_token_rows *rows, const vl_token_scores *out, void *work, uint64_t work_bytes, vl_stream stream_) {
  const int32_t rc = check_scores(rows, out);
  if (rc != VL_OK) return rc;
  if (const uint64_t need = work_of(rows, out)) {
    if (!work) return VL_E_NULL;
    if (work_bytes < need || (uintptr_t)work & 15) return VL_E_SHAPE;
  }
  hipStream_t stream = (hipStream_t)stream_;
  const Scores o = {(float VL_GLOBAL *)out->logprob, (float VL_GLOBAL *)out->entropy, (float VL_GLOBAL *)out->stat, (float VL_GLOBAL *)out->top_logprob,
                    (int32_t VL_GLOBAL *)out->top_token, out->n_top};
  (rows->type == VL_F32 ? launch_scores<F32> : rows->type == VL_F16 ? launch_scores<F16> : launch_scores<BF16>)(
      device_rows(rows), o, chunks_of(rows), split_of(rows, out->n_top, has_lead(rows)), work, stream);
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
  const Grad b = {(const float VL_GLOBAL *)stat, (const float VL_GLOBAL *)entropy, (const float VL_GLOBAL *)g_logprob, (const float VL_GLOBAL *)g_entropy,
                  (uint8_t VL_GLOBAL *)grad, grad_ld * size_of(rows->type)};
  (rows->type == VL_F32 ? launch_grad<F32> : rows->type == VL_F16 ? launch_grad<F16> : launch_grad<BF16>)(device_rows(rows), b, chunks_of(rows), stream);
  VL_HIP(hipGetLastError());
  return VL_OK;
}
