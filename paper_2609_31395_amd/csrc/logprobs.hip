// logprobs.hip -- log probabilities of given tokens, the entropy of each row of logits and its top
// alternatives (actkv_token_logprobs).
//
// Per row, with m = max x, S = sum e^(x - m) and U = sum e^(x - m) (x - m):
//   LSE = m + log S,   log p_v = x_v - LSE,   -sum p log p = log S - U / S.
// Bound by reading the logits once.  A row is cut into chunks, one workgroup each, which holds its
// chunk in registers: the maximum, then the two sums, then the chunk's top_k in order.  A second kernel
// joins a row's chunks in fp64 and ranks their candidates.
// Chunks of 16,384 logits (64 to a thread); of 4,096 for so few rows that the CUs would hold fewer than
// two of the large ones each, as long as a row's candidates stay at most 1,024.
//
// An entry's order is its 64-bit key: the order key of its value, then the complement of its token,
// so that keys differ and the larger one goes first.
#include <type_traits>

#include "device_common.hpp"

namespace actkv {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kCand = kLogprobsCand;      // candidates ranked in LDS, of a chunk or of a row

typedef unsigned long long u64;

__device__ __forceinline__ uint32_t order_key(float v) {   // -0 as +0
  const uint32_t u = __float_as_uint(v == 0.0f ? 0.0f : v);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k);
}

// How many of the C keys of `cand` (LDS) are larger than `key`.  cand[C ..] up to a multiple of
// kRankPad keys are 0, which no key is larger than; the reads of a batch are in flight together (one by
// one they cost 35 ns each).
constexpr int kRankPad = 16;
__device__ __forceinline__ int rank_of(u64 key, const u64* cand, int C) {
  int rank = 0;
  for (int x = 0; x < C; x += kRankPad) {
    u64 v[kRankPad];
#pragma unroll
    for (int y = 0; y < kRankPad; ++y) v[y] = cand[x + y];
#pragma unroll
    for (int y = 0; y < kRankPad; ++y) rank += v[y] > key ? 1 : 0;
  }
  return rank;
}

template <typename T>
__device__ __forceinline__ float widen(T v) {
  if constexpr (std::is_same<T, uint16_t>::value) return __uint_as_float((uint32_t)v << 16);   // bf16
  else return (float)v;
}

// One DPP step of a reduction over the wave: lanes with no source take `none`.
template <int kCtrl, int kRowMask, typename Join>
__device__ __forceinline__ float dpp_join(float v, float none, Join join) {
  const int o = __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, v), kCtrl,
                                            kRowMask, 0xf, false);
  return join(v, __builtin_bit_cast(float, o));
}
// join over the wave's 64 lanes, in a fixed order (every lane gets it): within rows of 16, then rows.
template <typename Join>
__device__ __forceinline__ float wave_join(float v, float none, Join join) {
  v = dpp_join<0x111, 0xf>(v, none, join);   // row_shr:1, 2, 4, 8
  v = dpp_join<0x112, 0xf>(v, none, join);
  v = dpp_join<0x114, 0xf>(v, none, join);
  v = dpp_join<0x118, 0xf>(v, none, join);
  v = dpp_join<0x142, 0xa>(v, none, join);   // row_bcast:15 into rows 1 and 3
  v = dpp_join<0x143, 0xc>(v, none, join);   // row_bcast:31 into rows 2 and 3
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
__device__ __forceinline__ float wave_max(float v) {
  return wave_join(v, -__builtin_inff(), [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_sum(float v) {
  return wave_join(v, 0.f, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float block_max(float v, float* red) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}

// The chunk's kk largest keys of u (register j of the thread: token of(j)), kk >= 1, into out[0 .. kk).
// Few candidates: those at or above the kk-th largest of the threads' own maxima, ranked by counting.
// Too many of them (equal values): the kk-th value by bisection, then the entries above it and the
// first of those equal to it.
template <int kPer, typename Of>
__device__ __forceinline__ void chunk_top(const uint32_t (&u)[kPer], Of of, int vec, int kk, u64* out,
                                          u64* cand, uint32_t* lmax, uint32_t* cnt, int64_t* scan_s) {
  const int tid = threadIdx.x, lane = tid & 63;
  uint32_t mine = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) mine = max(mine, u[j]);
  lmax[tid] = mine;
  if (tid == 0) *cnt = 0;
  __syncthreads();
  // A value that at least kk threads' maxima reach: the largest such in its upper 20 bits (the lower
  // ones would save a candidate now and then).  By one wave: four doing the same would keep the vector
  // units of all from the other workgroups.
  if (tid < 64) {
    uint32_t x[kWaves], t0 = 0;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) x[k] = lmax[k * 64 + lane];
#pragma unroll 4
    for (int b = 31; b >= 12; --b) {
      const uint32_t t = t0 | (1u << b);
      int c = 0;
#pragma unroll
      for (int k = 0; k < kWaves; ++k) c += __popcll(__ballot(x[k] >= t));
      if (c >= kk) t0 = t;
    }
    if (tid == 0) lmax[0] = max(t0, 1u);   // (0: fewer threads than kk hold an entry: all entries)
  }
  __syncthreads();
  const uint32_t lo = lmax[0];
#pragma unroll
  for (int j = 0; j < kPer; ++j)
    if (u[j] >= lo) {
      const uint32_t at = atomicAdd(cnt, 1u);
      if (at < (uint32_t)kCand) cand[at] = ((u64)u[j] << 32) | (0xFFFFFFFFu - (uint32_t)of(j));
    }
  __syncthreads();
  const int C = (int)*cnt;
  if (C <= kCand) {
    if (tid < kRankPad) cand[C + tid] = 0;
    __syncthreads();
    for (int i = tid; i < C; i += kThreads) {
      const int rank = rank_of(cand[i], cand, C);
      if (rank < kk) out[rank] = cand[i];
    }
    return;
  }
  uint32_t tau = 0;
  for (int b = 31; b >= 0; --b) {
    const uint32_t t = tau | (1u << b);
    int c = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) c += u[j] >= t ? 1 : 0;
    int64_t all;
    block_excl_scan_i64(c, scan_s, &all);
    if (all >= kk) tau = t;
  }
  int above = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) above += u[j] > tau ? 1 : 0;
  int64_t all;
  int64_t at = block_excl_scan_i64(above, scan_s, &all);
  // (the chosen ones, in LDS, then in order)
#pragma unroll
  for (int j = 0; j < kPer; ++j)
    if (u[j] > tau) cand[at++] = ((u64)u[j] << 32) | (0xFFFFFFFFu - (uint32_t)of(j));
  // equal entries in the order of their tokens: groups of `vec` registers, threads, registers
  int64_t taken = all;
  for (int g = 0; g < kPer / vec && taken < kk; ++g) {
    int equal = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) equal += j / vec == g && u[j] == tau ? 1 : 0;
    int64_t place = taken + block_excl_scan_i64(equal, scan_s, &all);
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (j / vec == g && u[j] == tau) {
        if (place < kk) cand[place] = ((u64)tau << 32) | (0xFFFFFFFFu - (uint32_t)of(j));
        ++place;
      }
    taken += all;
  }
  if (tid < kRankPad) cand[kk + tid] = 0;
  __syncthreads();
  if (tid < kk) out[rank_of(cand[tid], cand, kk)] = cand[tid];
}

}  // namespace

// Workgroup (row, chunk).  Register j of thread t holds token ((j / V) * 256 + t) * V + j % V of the
// chunk, V = 16 bytes of logits: 16-byte loads where the rows allow them, else one logit at a time.
template <typename T, bool kTop, int kPer>
__global__ __launch_bounds__(kThreads) void logprobs_chunk_kernel(
    const T* __restrict__ logits, int64_t vocab, int64_t row_stride, int k, int splits, int aligned,
    float* __restrict__ stats, u64* __restrict__ top) {
  constexpr int V = 16 / (int)sizeof(T), kChunk = kPer * kThreads;
  __shared__ float red[3][kWaves];
  __shared__ __align__(16) u64 cand[kTop ? kCand + kRankPad : 1];
  __shared__ uint32_t lmax[kTop ? kThreads : 1], cnt;
  __shared__ int64_t scan_s[17];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int64_t slot = blockIdx.x, row = slot / splits;
  const int c0 = (int)(slot % splits) * kChunk;
  const int n = (int)(vocab - c0 < kChunk ? vocab - c0 : kChunk);
  const T* base = logits + row * row_stride + c0;
  auto of = [&](int j) { return ((j / V) * kThreads + tid) * V + j % V; };
  float x[kPer];
  if (aligned) {
    // (up to the 4 bytes that hold the last logit: the rest reads as 0)
    const __amdgpu_buffer_rsrc_t rs = buffer_over(base, (n * (int)sizeof(T) + 3) & ~3);
#pragma unroll
    for (int g = 0; g < kPer / V; ++g) {
      const u32x4 raw = __builtin_amdgcn_raw_buffer_load_b128(rs, (g * kThreads + tid) * 16, 0, 0);
      T e[V];
      __builtin_memcpy(e, &raw, 16);
#pragma unroll
      for (int y = 0; y < V; ++y) x[g * V + y] = widen(e[y]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < kPer; ++j) x[j] = of(j) < n ? widen(base[of(j)]) : 0.f;
  }
  if (n < kChunk) {
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (of(j) >= n) x[j] = -__builtin_inff();
  }
  float m = x[0];
#pragma unroll
  for (int j = 1; j < kPer; ++j) m = fmaxf(m, x[j]);
  m = block_max(m, red[0]);
  float s = 0.f, u = 0.f;
  if (m != -__builtin_inff()) {
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const float d = fmaxf(x[j] - m, -1e30f);   // a masked token: e^d is 0, and so is e^d d
      const float e = fast_exp2(d * kLog2e);
      s += e;
      u = __builtin_fmaf(e, d, u);
    }
  }
  s = wave_sum(s);
  u = wave_sum(u);
  if (lane == 0) {
    red[1][w] = s;
    red[2][w] = u;
  }
  __syncthreads();
  if (tid == 0) {
    stats[slot * 3] = m;
    stats[slot * 3 + 1] = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
    stats[slot * 3 + 2] = (red[2][0] + red[2][1]) + (red[2][2] + red[2][3]);
  }
  if constexpr (kTop) {
    const int kk = k < n ? k : n;
    uint32_t key[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) key[j] = of(j) < n ? max(order_key(x[j]), 1u) : 0u;
    u64* out = top + slot * k;
    for (int i = kk + tid; i < k; i += kThreads) out[i] = 0;
    chunk_top<kPer>(key, [&](int j) { return c0 + of(j); }, V, kk, out, cand, lmax, &cnt, scan_s);
  }
}

// A wave per row: its chunks joined, the given token.  With alternatives a workgroup per row, whose
// candidates all its threads rank.
template <typename T, bool kTop>
__global__ __launch_bounds__(kThreads) void logprobs_row_kernel(
    const T* __restrict__ logits, int64_t rows, int64_t vocab, int64_t row_stride,
    const int64_t* __restrict__ tokens, int k, int splits, const float* __restrict__ stats,
    const u64* __restrict__ top, float* __restrict__ logprobs, float* __restrict__ entropy,
    int64_t* __restrict__ top_tokens, float* __restrict__ top_logprobs) {
  __shared__ __align__(16) u64 cand[kTop ? kCand + kRankPad : 1];
  __shared__ uint32_t count;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int64_t row = kTop ? blockIdx.x : (int64_t)blockIdx.x * kWaves + w;
  if (row >= rows) return;
  const bool asks = logprobs && (kTop ? tid == 0 : lane == 0);
  const int64_t given = asks ? tokens[row] : 0;
  const float x_given = asks && given >= 0 && given < vocab ? widen(logits[row * row_stride + given]) : 0.f;
  // a chunk to a lane (splits <= 64); the sums by a fixed tree
  const float* st = stats + row * splits * 3;
  const float mc = lane < splits ? st[3 * lane] : -__builtin_inff();
  const float sc = lane < splits ? st[3 * lane + 1] : 0.f, uc = lane < splits ? st[3 * lane + 2] : 0.f;
  // the first two candidates of each chunk, and its last (a bound: see below)
  uint32_t first = 0, second = 0, least = 0;
  if constexpr (kTop) {
    if (tid == 0) count = 0;
    if (lane < splits) {
      const u64* c = top + (row * splits + lane) * k;
      first = (uint32_t)(c[0] >> 32);
      second = k > 1 ? (uint32_t)(c[1] >> 32) : 0;
      least = (uint32_t)(c[k - 1] >> 32);
    }
  }
  float m = mc;
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
  const bool none = m == -__builtin_inff();   // every token is masked
  double s = 0.0, u = 0.0;
  if (mc != -__builtin_inff()) {
    const double d = (double)mc - (double)m, f = exp(d);
    s = f * sc;
    u = f * (uc + d * sc);
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) {
    s += __shfl_xor(s, d, 64);
    u += __shfl_xor(u, d, 64);
  }
  const double ls = none ? 0.0 : log(s), lse = (double)m + ls;
  auto logprob = [&](float x) { return none ? -__builtin_inff() : (float)((double)x - lse); };
  if (kTop ? tid == 0 : lane == 0) {
    if (entropy) entropy[row] = none ? 0.f : (float)(ls - u / s);
    if (logprobs) logprobs[row] = given < 0 ? 0.f : (given >= vocab ? __builtin_nanf("") : logprob(x_given));
  }
  if constexpr (kTop) {
    // The row's k-th value is no smaller than the largest of the chunks' k-th, nor than the k-th of the
    // chunks' first two (0, no bound, where they are fewer than k).
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) least = max(least, (uint32_t)__shfl_xor((int)least, d, 64));
    uint32_t lo = 0;
    for (int b = 31; b >= 0; --b) {
      const uint32_t t = lo | (1u << b);
      if ((int)(__popcll(__ballot(first >= t)) + __popcll(__ballot(second >= t))) >= k) lo = t;
    }
    lo = max(max(lo, least), 1u);   // (key 0: a chunk of fewer than k logits)
    __syncthreads();
    const int N = splits * k;
    for (int i = tid; i < N; i += kThreads) {
      const u64 key = top[row * N + i];
      if ((uint32_t)(key >> 32) >= lo) cand[atomicAdd(&count, 1u)] = key;
    }
    __syncthreads();
    const int C = (int)count;
    if (tid < kRankPad) cand[C + tid] = 0;
    __syncthreads();
    for (int i = tid; i < C; i += kThreads) {
      const u64 key = cand[i];
      const int rank = rank_of(key, cand, C);
      if (rank < k) {
        top_tokens[row * k + rank] = (int64_t)(0xFFFFFFFFu - (uint32_t)key);
        top_logprobs[row * k + rank] = logprob(key_value((uint32_t)(key >> 32)));
      }
    }
    for (int64_t i = vocab + tid; i < k; i += kThreads) {
      top_tokens[row * k + i] = -1;
      top_logprobs[row * k + i] = -__builtin_inff();
    }
  }
}

hipError_t launch_token_logprobs(const void* logits, int type, int64_t rows, int64_t vocab,
                                 int64_t row_stride, const int64_t* tokens, int k, float* logprobs,
                                 float* entropy, int64_t* top_tokens, float* top_logprobs,
                                 float* stats, unsigned long long* top, hipStream_t s) {
  const int splits = logprobs_splits(rows, vocab, k);
  const bool small = splits > logprobs_large(vocab);
  auto run = [&](auto zero) {
    using T = decltype(zero);
    const T* x = static_cast<const T*>(logits);
    const int aligned = (reinterpret_cast<uintptr_t>(x) & 15) == 0 &&
                        (rows == 1 || (row_stride * sizeof(T)) % 16 == 0);
    const dim3 grid((unsigned)(rows * splits));
    auto chunks = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, x, vocab, row_stride, k, splits, aligned, stats, top);
    };
    constexpr int kLarge = kLogprobsChunk / kThreads, kSmall = kLogprobsSmallChunk / kThreads;
    if (k > 0) small ? chunks(logprobs_chunk_kernel<T, true, kSmall>) : chunks(logprobs_chunk_kernel<T, true, kLarge>);
    else small ? chunks(logprobs_chunk_kernel<T, false, kSmall>) : chunks(logprobs_chunk_kernel<T, false, kLarge>);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    auto join = [&](auto kernel, int64_t wgs) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(kThreads), 0, s, x, rows, vocab, row_stride, tokens, k,
                         splits, stats, top, logprobs, entropy, top_tokens, top_logprobs);
    };
    if (k > 0) join(logprobs_row_kernel<T, true>, rows);
    else join(logprobs_row_kernel<T, false>, (rows + kWaves - 1) / kWaves);
    return hipGetLastError();
  };
  return type == ACTKV_LOGITS_F32 ? run(0.0f) : type == ACTKV_LOGITS_BF16 ? run((uint16_t)0) : run((_Float16)0);
}

}  // namespace actkv
