// logprobs.hip -- log probabilities of given tokens, the entropy of each row of logits and its top
// alternatives (actkv_token_logprobs).
//
// Per row, with m = max x, S = sum e^(x - m) and U = sum e^(x - m) (x - m):
//   LSE = m + log S,   log p_v = x_v - LSE,   -sum p log p = log S - U / S.
// Bound by reading the logits once.  A row is cut into chunks of 16,384 logits, one workgroup each,
// which holds its chunk in registers: the maximum, then the two sums, then the chunk's top_k.  A
// second kernel joins a row's chunks in fp64 and ranks their candidates.
//
// An entry's order is its 64-bit key: the order key of its value, then the complement of its token,
// so that keys differ and the larger one goes first.
#include <type_traits>

#include "device_common.hpp"

namespace actkv {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kChunk = kConfChunkLogits;
constexpr int kPer = kChunk / kThreads;   // 64 logits per thread
constexpr int kCand = 1024;               // candidates of a chunk ranked in LDS

typedef unsigned long long u64;

__device__ __forceinline__ uint32_t order_key(float v) {   // -0 as +0
  const uint32_t u = __float_as_uint(v == 0.0f ? 0.0f : v);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k);
}

template <typename T>
__device__ __forceinline__ float widen(T v) {
  if constexpr (std::is_same<T, uint16_t>::value) return __uint_as_float((uint32_t)v << 16);   // bf16
  else return (float)v;
}

__device__ __forceinline__ float block_max(float v, float* red) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v = fmaxf(v, __shfl_xor(v, d, 64));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
  return v;
}

// The chunk's kk largest keys of u (register j of the thread: token of(j)), kk >= 1, into out[0 .. kk).
// Few candidates: those at or above the kk-th largest of the threads' own maxima, ranked by counting.
// Too many of them (equal values): the kk-th value by bisection, then the entries above it and the
// first of those equal to it.
template <typename Of>
__device__ __forceinline__ void chunk_top(const uint32_t (&u)[kPer], Of of, int vec, int kk, u64* out,
                                          u64* cand, uint32_t* lmax, uint32_t* cnt, int64_t* scan_s) {
  const int tid = threadIdx.x, lane = tid & 63;
  uint32_t mine = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) mine = max(mine, u[j]);
  lmax[tid] = mine;
  if (tid == 0) *cnt = 0;
  __syncthreads();
  uint32_t lo = 0;   // the largest t with at least kk threads whose maximum is >= t
  {
    uint32_t x[kWaves];
#pragma unroll
    for (int k = 0; k < kWaves; ++k) x[k] = lmax[k * 64 + lane];
    for (int b = 31; b >= 0; --b) {
      const uint32_t t = lo | (1u << b);
      int c = 0;
#pragma unroll
      for (int k = 0; k < kWaves; ++k) c += __popcll(__ballot(x[k] >= t));
      if (c >= kk) lo = t;
    }
  }
  if (lo == 0) lo = 1;   // fewer threads than kk hold an entry: all entries
#pragma unroll
  for (int j = 0; j < kPer; ++j)
    if (u[j] >= lo) {
      const uint32_t at = atomicAdd(cnt, 1u);
      if (at < (uint32_t)kCand) cand[at] = ((u64)u[j] << 32) | (0xFFFFFFFFu - (uint32_t)of(j));
    }
  __syncthreads();
  const int C = (int)*cnt;
  if (C <= kCand) {
    for (int i = tid; i < C; i += kThreads) {
      const u64 key = cand[i];
      int rank = 0;
      for (int x = 0; x < C; ++x) rank += cand[x] > key ? 1 : 0;
      if (rank < kk) out[rank] = key;
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
#pragma unroll
  for (int j = 0; j < kPer; ++j)
    if (u[j] > tau) out[at++] = ((u64)u[j] << 32) | (0xFFFFFFFFu - (uint32_t)of(j));
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
        if (place < kk) out[place] = ((u64)tau << 32) | (0xFFFFFFFFu - (uint32_t)of(j));
        ++place;
      }
    taken += all;
  }
}

}  // namespace

// Workgroup (row, chunk).  Register j of thread t holds token ((j / V) * 256 + t) * V + j % V of the
// chunk, V = 16 bytes of logits: 16-byte loads where the rows allow them, else one logit at a time.
template <typename T, bool kTop>
__global__ __launch_bounds__(kThreads) void logprobs_chunk_kernel(
    const T* __restrict__ logits, int64_t vocab, int64_t row_stride, int k, int splits, int aligned,
    float* __restrict__ stats, u64* __restrict__ top) {
  constexpr int V = 16 / (int)sizeof(T);
  __shared__ float red[3][kWaves];
  __shared__ u64 cand[kTop ? kCand : 1];
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
    chunk_top(key, [&](int j) { return c0 + of(j); }, V, kk, out, cand, lmax, &cnt, scan_s);
  }
}

// One workgroup per row: its chunks joined, the given token, the candidates ranked.
template <typename T>
__global__ __launch_bounds__(kThreads) void logprobs_row_kernel(
    const T* __restrict__ logits, int64_t vocab, int64_t row_stride, const int64_t* __restrict__ tokens,
    int k, int splits, const float* __restrict__ stats, const u64* __restrict__ top,
    float* __restrict__ logprobs, float* __restrict__ entropy, int64_t* __restrict__ top_tokens,
    float* __restrict__ top_logprobs) {
  __shared__ u64 cand[kConfMaxSplits * kConfMaxTopK];
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;
  const float* st = stats + row * splits * 3;
  float m = st[0];
  for (int i = 1; i < splits; ++i) m = fmaxf(m, st[3 * i]);
  const bool none = m == -__builtin_inff();   // every token is masked
  double s = 0.0, u = 0.0;
  for (int i = 0; i < splits; ++i)
    if (st[3 * i] != -__builtin_inff()) {
      const double d = (double)st[3 * i] - (double)m, f = exp(d);
      s += f * st[3 * i + 1];
      u += f * (st[3 * i + 2] + d * st[3 * i + 1]);
    }
  const double ls = none ? 0.0 : log(s), lse = (double)m + ls;
  auto logprob = [&](float x) { return none ? -__builtin_inff() : (float)((double)x - lse); };
  if (tid == 0) {
    if (entropy) entropy[row] = none ? 0.f : (float)(ls - u / s);
    if (logprobs) {
      const int64_t t = tokens[row];
      logprobs[row] = t < 0 ? 0.f
                            : (t >= vocab ? __builtin_nanf("") : logprob(widen(logits[row * row_stride + t])));
    }
  }
  if (k == 0) return;
  const int N = splits * k;
  for (int i = tid; i < N; i += kThreads) cand[i] = top[row * N + i];
  __syncthreads();
  for (int i = tid; i < N; i += kThreads) {
    const u64 key = cand[i];
    if (key == 0) continue;   // a chunk of fewer than k logits
    int rank = 0;
    for (int x = 0; x < N; ++x) rank += cand[x] > key ? 1 : 0;
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

hipError_t launch_token_logprobs(const void* logits, int type, int64_t rows, int64_t vocab,
                                 int64_t row_stride, const int64_t* tokens, int k, float* logprobs,
                                 float* entropy, int64_t* top_tokens, float* top_logprobs,
                                 float* stats, unsigned long long* top, hipStream_t s) {
  const int splits = conf_splits(vocab);
  auto run = [&](auto zero) {
    using T = decltype(zero);
    const T* x = static_cast<const T*>(logits);
    const int aligned = (reinterpret_cast<uintptr_t>(x) & 15) == 0 &&
                        (rows == 1 || (row_stride * sizeof(T)) % 16 == 0);
    const dim3 grid((unsigned)(rows * splits));
    if (k > 0)
      hipLaunchKernelGGL((logprobs_chunk_kernel<T, true>), grid, dim3(kThreads), 0, s, x, vocab, row_stride,
                         k, splits, aligned, stats, top);
    else
      hipLaunchKernelGGL((logprobs_chunk_kernel<T, false>), grid, dim3(kThreads), 0, s, x, vocab, row_stride,
                         k, splits, aligned, stats, top);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(logprobs_row_kernel<T>, dim3((unsigned)rows), dim3(k > 0 ? kThreads : 64), 0, s, x,
                       vocab, row_stride, tokens, k, splits, stats, top, logprobs, entropy, top_tokens,
                       top_logprobs);
    return hipGetLastError();
  };
  return type == ACTKV_LOGITS_F32 ? run(0.0f) : type == ACTKV_LOGITS_BF16 ? run((uint16_t)0) : run((_Float16)0);
}

}  // namespace actkv
