// pages.hip -- pages shared by several requests: counts of holders (actkv_acquire_pages,
// actkv_release_pages) and forks of requests (actkv_fork_pages).
//
// A fork moves what it copies (a page is read and written once) and touches one table entry per page; a
// release reads the entries.  An atomic on a count for each entry would bound both (25 a nanosecond over
// the card), so one is made for several: the forks of a parent that follow each other count its pages
// once, and a release takes off at once what a column of its list names in a run, as the branches' rows
// of one parent do (32 x 8 branches of 30,000-35,000 entries, 560,000 of them: fork 24 -> 10.5 us, counts of
// the release 22 -> 7.5; with the workgroups numbered by rows, then copies, the fork takes 8.7).  What is
// left of these is 70,000 atomics each, 2.8 us, and chains of dependent loads.  The pages a release frees
// are listed by page id through a bitmap of the pool, so the list does not depend on the order in which
// the counts' atomics land.
#include "device_common.hpp"

namespace actkv {

namespace {

constexpr int kThreads = 256;
constexpr int kRowEntries = 1024;   // table entries a workgroup of a fork writes

__device__ __forceinline__ bool in_pool(int64_t page, int64_t num_pages) {
  return page >= 0 && page < num_pages;
}

// The sum of v over the wave, in its last lane.  (32 bits: a fork has 2^23 pages at most.)
__device__ __forceinline__ int32_t wave_last_sum(int32_t v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);   // row_shr:1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // row_bcast:15 into rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);   // row_bcast:31 into rows 2 and 3
  return v;
}

// Where the parent of fresh page x is entered in the block table (-1: x is behind the last): the forks are
// added up in chunks of 64, as many as a lane each can hold, until x lies in one of these, and every wave
// then has a chunk's forks in its lanes.  For the whole workgroup; up to 64 forks take no barrier.
constexpr int kForkChunks = 64;
__device__ __forceinline__ int64_t parent_entry(const actkv_fork* forks, int num_forks, int64_t x, int32_t bt_stride,
                                                int32_t* chunk_s) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  auto fresh_of = [&](int f) { return f < num_forks ? forks[f].pages - forks[f].shared : 0; };
  // the lanes that x is behind, and what the pages of all of these come to
  auto behind = [&](int64_t incl, int* lanes) {
    *lanes = __popcll(__ballot(incl <= x));
    return *lanes > 0 ? readlane_i64(incl, *lanes - 1) : 0;
  };
  int64_t before = 0;   // pages of the forks before `first`
  int first = 0, k;
  if (num_forks > 64)
    for (;; first += 64 * kForkChunks) {
      constexpr int kWaves = kThreads / 64, kPer = kForkChunks / kWaves;
      int32_t n[kPer];   // a lane's forks of the wave's chunks, all loads in flight
#pragma unroll
      for (int c = 0; c < kPer; ++c) n[c] = fresh_of(first + 64 * (kWaves * c + w) + lane);
#pragma unroll
      for (int c = 0; c < kPer; ++c) {
        n[c] = wave_last_sum(n[c]);
        if (lane == 63) chunk_s[kWaves * c + w] = n[c];
      }
      __syncthreads();
      const int64_t incl = before + wave_incl_scan_i64(chunk_s[lane]);
      const int64_t all = readlane_i64(incl, 63);
      if (x < all) {
        const int64_t b = behind(incl, &k);
        if (k > 0) before = b;
        first += 64 * k;
        break;
      }
      before = all;
      if (first + 64 * kForkChunks >= num_forks) return -1;
      __syncthreads();   // chunk_s is written again
    }
  const int64_t incl = before + wave_incl_scan_i64(fresh_of(first + lane));
  const int64_t b = behind(incl, &k);
  if (k == 64) return -1;
  const actkv_fork fk = forks[first + k];
  return (int64_t)fk.parent * bt_stride + fk.shared + (x - (k > 0 ? b : before));
}

}  // namespace

// Workgroups: row_wgs for the row of each fork, which write kRowEntries of the child's row each and count
// the shared pages; then, by `each`, that many for each fork, or (0) one for each page that is copied
// (`fresh` of them, numbered as the fresh pages are), which copy a page, K and V.
__global__ __launch_bounds__(kThreads) void fork_kernel(
    const actkv_fork* forks, int num_forks, int row_wgs, int each, uint32_t fresh, int32_t bt_stride,
    int64_t num_pages, int64_t page_vecs, u32x4* kv, int32_t* bt, const int32_t* free_pages, int32_t* refs) {
  __shared__ int64_t scan_s[17];
  __shared__ int32_t chunk_s[kForkChunks];
  const int tid = threadIdx.x;
  const uint32_t rows = (uint32_t)num_forks * (uint32_t)row_wgs, wg = blockIdx.y * gridDim.x + blockIdx.x;
  // fresh pages of the forks before f
  auto fresh_before = [&](int f) {
    int64_t mine = 0, all;
    for (int x = tid; x < f; x += kThreads) mine += forks[x].pages - forks[x].shared;
    block_excl_scan_i64(mine, scan_s, &all);
    return all;
  };
  if (wg >= rows) {
    int64_t x = wg - rows, entry;
    if (each > 0) {
      const int f = (int)((uint32_t)x / (uint32_t)each), i = (int)((uint32_t)x - (uint32_t)f * each);
      if (f >= num_forks) return;
      const actkv_fork fk = forks[f];
      if (i >= fk.pages - fk.shared) return;
      x = fresh_before(f) + i;
      entry = (int64_t)fk.parent * bt_stride + fk.shared + i;
    } else {
      if (x >= fresh) return;
      entry = parent_entry(forks, num_forks, x, bt_stride, chunk_s);
      if (entry < 0) return;
    }
    const int64_t src = bt[entry], dst = free_pages[x];
    if (!in_pool(src, num_pages) || !in_pool(dst, num_pages)) return;
    for (int64_t i = tid; i < page_vecs; i += kThreads) {
      kv[dst * page_vecs + i] = kv[src * page_vecs + i];
      kv[(num_pages + dst) * page_vecs + i] = kv[(num_pages + src) * page_vecs + i];
    }
    return;
  }
  const int f = (int)(wg / (uint32_t)row_wgs), row_wg = (int)(wg - (uint32_t)f * row_wgs);
  const actkv_fork fk = forks[f];
  const int64_t off = fresh_before(f);
  const int32_t* parent = bt + (int64_t)fk.parent * bt_stride;
  // the shared pages of the forks of this parent in this fork's group of 64: a run of them counts a
  // page once
  __shared__ int32_t shared_s[64];
  if (tid < 64) {
    const int x = (f & ~63) + tid;
    shared_s[tid] = x < num_forks && forks[x].parent == fk.parent ? forks[x].shared : 0;
  }
  int32_t* child = bt + (int64_t)fk.child * bt_stride;
  constexpr int kPer = kRowEntries / kThreads;
  int32_t page[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = row_wg * kRowEntries + k * kThreads + tid;
    page[k] = i < fk.shared ? parent[i] : i < fk.pages ? free_pages[off + i - fk.shared] : -1;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = row_wg * kRowEntries + k * kThreads + tid;
    if (i >= bt_stride) continue;
    child[i] = page[k];
    if (!refs || !in_pool(page[k], num_pages)) continue;
    if (i >= fk.shared) {
      refs[page[k]] = 1;
    } else if ((f & 63) == 0 || shared_s[(f & 63) - 1] <= i) {   // the first of its run
      int x = (f & 63) + 1;
      while (x < 64 && shared_s[x] > i) ++x;
      atomicAdd(refs + page[k], x - (f & 63));
    }
  }
}

__global__ __launch_bounds__(kThreads) void acquire_kernel(const int32_t* pages, int64_t n,
                                                           int64_t num_pages, int32_t* refs) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads)
    if (in_pool(pages[i], num_pages)) atomicAdd(refs + pages[i], 1);
}

__global__ __launch_bounds__(kThreads) void release_clear_kernel(uint32_t* words, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads)
    words[i] = 0;
}

// After `off` was counted off a page that had `old`: whether that brought it to 0.  What was not there
// is put back: the count can't pass 0 again on the way, so of all that count a page off the one that
// sees a positive count and takes the last of it is the one that frees the page.
__device__ __forceinline__ bool came_to_zero(int32_t* ref, int32_t old, int off) {
  if (old < off) atomicAdd(ref, off - max(old, 0));
  return old > 0 && old <= off;
}

// A thread: kRows entries of one column of the list, [rows][row_len] (the last row may be short).
// A freed page sets its bit.
template <int kRows>
__global__ __launch_bounds__(kThreads) void release_kernel(const int32_t* pages, int64_t n, int64_t row_len,
                                                           int64_t num_pages, int32_t* refs,
                                                           uint32_t* bits) {
  const int64_t col_wgs = (row_len + kThreads - 1) / kThreads;
  const int64_t col = blockIdx.x % col_wgs * kThreads + threadIdx.x;
  const int64_t first = blockIdx.x / col_wgs * kRows * row_len + col;
  if (col >= row_len) return;
  int32_t page[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r) page[r] = first + r * row_len < n ? pages[first + r * row_len] : -1;
  // off[r]: what the run that ends at r counts off (0: none ends there); all counts set out first
  int off[kRows], old[kRows], run = 0;
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    ++run;
    const bool ends = r + 1 == kRows || page[r + 1] != page[r];
    off[r] = ends && in_pool(page[r], num_pages) ? run : 0;
    if (ends) run = 0;
  }
#pragma unroll
  for (int r = 0; r < kRows; ++r) old[r] = off[r] > 0 ? atomicSub(refs + page[r], off[r]) : 0;
#pragma unroll
  for (int r = 0; r < kRows; ++r)
    if (off[r] > 0 && came_to_zero(refs + page[r], old[r], off[r]))
      atomicOr(bits + (page[r] >> 5), 1u << (page[r] & 31));
}

// counts[b]: the freed pages of block b, kReleaseBlock pages, a word of the bitmap per thread.  (Counted
// here and not as they are freed: atomics on so few counters cost 13 us for 17,500 pages.)
__global__ __launch_bounds__(kThreads) void release_count_kernel(int64_t num_words, const uint32_t* bits,
                                                                 uint32_t* counts) {
  __shared__ int64_t scan_s[17];
  const int64_t word = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  int64_t all;
  block_excl_scan_i64(word < num_words ? __popc(bits[word]) : 0, scan_s, &all);
  if (threadIdx.x == 0) counts[blockIdx.x] = (uint32_t)all;
}

// Workgroup b lists the freed pages of block b (behind the bitmap's end: none); the entries of `freed`
// behind the list are filled by all of them.  kCounts: the blocks' counts are there; otherwise every
// workgroup counts the whole bitmap, which is short.
template <bool kCounts>
__global__ __launch_bounds__(kThreads) void release_list_kernel(int64_t n, int64_t num_words,
                                                                const uint32_t* bits,
                                                                const uint32_t* counts,
                                                                int32_t* freed, int32_t* num_freed) {
  __shared__ int64_t scan_s[17];
  const int64_t b = blockIdx.x, wgs = gridDim.x;
  const int tid = threadIdx.x;
  const int64_t word = b * kThreads + tid;
  uint32_t w = word < num_words ? bits[word] : 0u;
  int64_t sums = 0, all;   // pages of the blocks before, and of all of them in the upper half
  const int64_t entries = kCounts ? (num_words + kThreads - 1) / kThreads : num_words;
  const int64_t here_from = kCounts ? b : b * kThreads;
#pragma unroll 8
  for (int64_t x = tid; x < entries; x += kThreads) {
    const int64_t v = kCounts ? (int64_t)counts[x] : (int64_t)__popc(bits[x]);
    sums += (v << 32) + (x < here_from ? v : 0);
  }
  block_excl_scan_i64(sums, scan_s, &all);
  const int64_t before = all & 0xFFFFFFFF, total = all >> 32;
  int64_t here;
  int64_t at = before + block_excl_scan_i64(__popc(w), scan_s, &here);
  for (; w; w &= w - 1) freed[at++] = (int32_t)(word * 32 + __builtin_ctz(w));
  for (int64_t i = total + b * kThreads + tid; i < n; i += wgs * kThreads) freed[i] = -1;
  if (b == 0 && tid == 0) *num_freed = (int32_t)total;
}

// The same for at most kReleaseSmall entries, in one workgroup without the bitmap: the freed pages
// listed in LDS, then each at its rank among them.
__global__ __launch_bounds__(kReleaseSmall) void release_small_kernel(const int32_t* pages, int n,
                                                                      int64_t num_pages, int32_t* refs,
                                                                      int32_t* freed, int32_t* num_freed) {
  __shared__ int32_t gone[kReleaseSmall];
  __shared__ int count;
  const int tid = threadIdx.x;
  if (tid == 0) count = 0;
  __syncthreads();
  if (tid < n) {
    const int32_t page = pages[tid];
    if (in_pool(page, num_pages) && came_to_zero(refs + page, atomicSub(refs + page, 1), 1))
      gone[atomicAdd(&count, 1)] = page;
  }
  __syncthreads();
  const int total = count;
  if (tid < total) {
    int rank = 0;
    for (int x = 0; x < total; ++x) rank += gone[x] < gone[tid] ? 1 : 0;
    freed[rank] = gone[tid];
  } else if (tid < n) {
    freed[tid] = -1;
  }
  if (tid == 0) *num_freed = total;
}

static_assert(kReleaseBlock == kThreads * 32, "a word of the bitmap per thread");

namespace {
unsigned blocks_for(int64_t n) {
  const int64_t b = (n + kThreads - 1) / kThreads;
  return (unsigned)(b < 1 ? 1 : b > 4096 ? 4096 : b);
}
}  // namespace

hipError_t launch_fork(const actkv_fork* forks, int num_forks, int64_t fresh, int32_t max_copied,
                       int32_t bt_stride, int64_t num_pages, int64_t page_bytes, void* kv, int32_t* bt,
                       const int32_t* free_pages, int32_t* refs, hipStream_t s) {
  const int row_wgs = (bt_stride + kRowEntries - 1) / kRowEntries;
  // As many workgroups for each fork's copies while at most half of them are idle: a fork that is known
  // needs no search (4,096 forks of 4 pages: 43 against 63 us, 16,384 of one 145 against 174; 256 of one 7.3
  // and 7.4).  By page for unequal copies (256 forks of which one copies 2,188 pages: 2,956 workgroups in
  // place of 560,896).
  const int64_t even = (int64_t)num_forks * max_copied;
  const int each = even <= 2 * fresh && even <= INT32_MAX ? max_copied : 0;
  // (at most 2^29 for the rows and 2^31 for the pages: numbered in 32 bits, in rows of at most 2^20)
  const int64_t wgs = (int64_t)num_forks * row_wgs + (each > 0 ? even : fresh), wide = wgs < (1 << 20) ? wgs : 1 << 20;
  hipLaunchKernelGGL(fork_kernel, dim3((unsigned)wide, (unsigned)((wgs + wide - 1) / wide)), dim3(kThreads), 0, s,
                     forks, num_forks, row_wgs, each, (uint32_t)fresh, bt_stride, num_pages, page_bytes / 16,
                     static_cast<u32x4*>(kv), bt, free_pages, refs);
  return hipGetLastError();
}

hipError_t launch_acquire(const int32_t* pages, int64_t n, int64_t num_pages, int32_t* refs,
                          hipStream_t s) {
  hipLaunchKernelGGL(acquire_kernel, dim3(blocks_for(n)), dim3(kThreads), 0, s, pages, n, num_pages, refs);
  return hipGetLastError();
}

hipError_t launch_release(const int32_t* pages, int64_t n, int64_t row_len, int64_t num_pages,
                          int32_t* refs, int32_t* freed, int32_t* num_freed, uint32_t* bits,
                          uint32_t* counts, hipStream_t s) {
  const int64_t num_words = (num_pages + 31) / 32;
  if (n <= kReleaseSmall) {
    hipLaunchKernelGGL(release_small_kernel, dim3(1), dim3(kReleaseSmall), 0, s, pages, (int)n, num_pages, refs,
                       freed, num_freed);
    return hipGetLastError();
  }
  // (a fill kernel: a memset node of a captured graph is not to be relied on)
  hipLaunchKernelGGL(release_clear_kernel, dim3(blocks_for(num_words)), dim3(kThreads), 0, s, bits, num_words);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // several rows to a thread once that leaves 64 workgroups (8 x 2,188 entries: 13.7 us with 9 of them)
  const bool deep = n >= 64 * kThreads * kReleaseRows;
  const int64_t rows = (n + row_len - 1) / row_len, per = deep ? kReleaseRows : 1;
  const dim3 grid((unsigned)((row_len + kThreads - 1) / kThreads * ((rows + per - 1) / per)));
  if (deep)
    hipLaunchKernelGGL(release_kernel<kReleaseRows>, grid, dim3(kThreads), 0, s, pages, n, row_len, num_pages,
                       refs, bits);
  else
    hipLaunchKernelGGL(release_kernel<1>, grid, dim3(kThreads), 0, s, pages, n, row_len, num_pages, refs, bits);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t blocks = release_blocks(num_pages);
  const int64_t fill_wgs = n / (8 * kThreads) < 512 ? n / (8 * kThreads) : 512;
  const dim3 list_grid((unsigned)(blocks > fill_wgs ? blocks : fill_wgs));
  // (64 KB of bitmap to each of at most 512 workgroups: no more than a launch costs)
  if (num_words <= 16384) {
    hipLaunchKernelGGL(release_list_kernel<false>, list_grid, dim3(kThreads), 0, s, n, num_words, bits, counts,
                       freed, num_freed);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(release_count_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, s, num_words, bits, counts);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(release_list_kernel<true>, list_grid, dim3(kThreads), 0, s, n, num_words, bits, counts, freed,
                     num_freed);
  return hipGetLastError();
}

}  // namespace actkv
