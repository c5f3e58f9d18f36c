// pages.hip -- pages shared by several requests: counts of holders (actkv_acquire_pages,
// actkv_release_pages) and forks of requests (actkv_fork_pages).
//
// A fork moves what it copies (a page is read and written once) and touches one count and one table
// entry per shared page; a release touches one count per entry.  The pages a release frees are
// listed by page id through a bitmap of the pool, so the list does not depend on the order in which
// the counts' atomics land.
#include "device_common.hpp"

namespace actkv {

namespace {

constexpr int kThreads = 256;
constexpr int kRowEntries = 1024;   // table entries a workgroup of a fork writes

__device__ __forceinline__ bool in_pool(int64_t page, int64_t num_pages) {
  return page >= 0 && page < num_pages;
}

}  // namespace

// Grid: (row workgroups + the most pages one fork copies, forks).  The first write kRowEntries of the
// child's row and count the shared pages; each of the others copies a page, K and V.
__global__ __launch_bounds__(kThreads) void fork_kernel(
    const actkv_fork* forks, int row_wgs, int32_t bt_stride, int64_t num_pages, int64_t page_vecs,
    u32x4* kv, int32_t* bt, const int32_t* free_pages, int32_t* refs) {
  __shared__ int64_t scan_s[17];
  const int f = blockIdx.y, tid = threadIdx.x;
  const actkv_fork fk = forks[f];
  int64_t mine = 0, off;   // off: fresh pages of the forks before
  for (int x = tid; x < f; x += kThreads) mine += forks[x].pages - forks[x].shared;
  block_excl_scan_i64(mine, scan_s, &off);
  const int32_t* parent = bt + (int64_t)fk.parent * bt_stride;
  if ((int)blockIdx.x >= row_wgs) {
    const int x = (int)blockIdx.x - row_wgs;
    if (x >= fk.pages - fk.shared) return;
    const int64_t src = parent[fk.shared + x], dst = free_pages[off + x];
    if (!in_pool(src, num_pages) || !in_pool(dst, num_pages)) return;
    for (int64_t i = tid; i < page_vecs; i += kThreads) {
      kv[dst * page_vecs + i] = kv[src * page_vecs + i];
      kv[(num_pages + dst) * page_vecs + i] = kv[(num_pages + src) * page_vecs + i];
    }
    return;
  }
  int32_t* child = bt + (int64_t)fk.child * bt_stride;
  for (int i = blockIdx.x * kRowEntries + tid; i < bt_stride && i < (int)(blockIdx.x + 1) * kRowEntries;
       i += kThreads) {
    int32_t page = -1;
    if (i < fk.shared) {
      page = parent[i];
      if (refs && in_pool(page, num_pages)) atomicAdd(refs + page, 1);
    } else if (i < fk.pages) {
      page = free_pages[off + i - fk.shared];
      if (refs && in_pool(page, num_pages)) refs[page] = 1;
    }
    child[i] = page;
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

// One count off per entry; a page whose count comes to 0 sets its bit and is counted in its block of
// kReleaseBlock pages.  A count that was not positive is put back: it can't pass 0 again on the way,
// so the one entry that sees 1 is the one that frees the page.
__global__ __launch_bounds__(kThreads) void release_kernel(const int32_t* pages, int64_t n,
                                                           int64_t num_pages, int32_t* refs,
                                                           uint32_t* bits, uint32_t* counts) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) {
    const int32_t page = pages[i];
    if (!in_pool(page, num_pages)) continue;
    const int32_t old = atomicSub(refs + page, 1);
    if (old == 1) {
      atomicOr(bits + (page >> 5), 1u << (page & 31));
      atomicAdd(counts + page / kReleaseBlock, 1u);
    } else if (old <= 0) {
      atomicAdd(refs + page, 1);
    }
  }
}

// Workgroup b lists the freed pages of block b, a word of the bitmap per thread; the entries of
// `freed` behind the list are filled by all of them.
__global__ __launch_bounds__(kThreads) void release_list_kernel(int64_t n, int64_t num_pages,
                                                                const uint32_t* bits,
                                                                const uint32_t* counts,
                                                                int32_t* freed, int32_t* num_freed) {
  __shared__ int64_t scan_s[17];
  const int b = blockIdx.x, blocks = gridDim.x, tid = threadIdx.x;
  int64_t sums = 0, all;   // pages of the blocks before, and of all of them in the upper half
  for (int x = tid; x < blocks; x += kThreads)
    sums += ((int64_t)counts[x] << 32) + (x < b ? counts[x] : 0u);
  block_excl_scan_i64(sums, scan_s, &all);
  const int64_t before = all & 0xFFFFFFFF, total = all >> 32;
  const int64_t word = (int64_t)b * kThreads + tid;
  uint32_t w = word < (num_pages + 31) / 32 ? bits[word] : 0u;
  int64_t here;
  int64_t at = before + block_excl_scan_i64(__popc(w), scan_s, &here);
  for (; w; w &= w - 1) freed[at++] = (int32_t)(word * 32 + __builtin_ctz(w));
  for (int64_t i = total + (int64_t)b * kThreads + tid; i < n; i += (int64_t)blocks * kThreads) freed[i] = -1;
  if (b == 0 && tid == 0) *num_freed = (int32_t)total;
}

static_assert(kReleaseBlock == kThreads * 32, "a word of the bitmap per thread");

namespace {
unsigned blocks_for(int64_t n) {
  const int64_t b = (n + kThreads - 1) / kThreads;
  return (unsigned)(b < 1 ? 1 : b > 4096 ? 4096 : b);
}
}  // namespace

hipError_t launch_fork(const actkv_fork* forks, int num_forks, int64_t max_copied, int32_t bt_stride,
                       int64_t num_pages, int64_t page_bytes, void* kv, int32_t* bt,
                       const int32_t* free_pages, int32_t* refs, hipStream_t s) {
  const int row_wgs = (bt_stride + kRowEntries - 1) / kRowEntries;
  hipLaunchKernelGGL(fork_kernel, dim3((unsigned)(row_wgs + max_copied), (unsigned)num_forks),
                     dim3(kThreads), 0, s, forks, row_wgs, bt_stride, num_pages, page_bytes / 16,
                     static_cast<u32x4*>(kv), bt, free_pages, refs);
  return hipGetLastError();
}

hipError_t launch_acquire(const int32_t* pages, int64_t n, int64_t num_pages, int32_t* refs,
                          hipStream_t s) {
  hipLaunchKernelGGL(acquire_kernel, dim3(blocks_for(n)), dim3(kThreads), 0, s, pages, n, num_pages, refs);
  return hipGetLastError();
}

hipError_t launch_release(const int32_t* pages, int64_t n, int64_t num_pages, int32_t* refs,
                          int32_t* freed, int32_t* num_freed, uint32_t* bits, uint32_t* counts,
                          int64_t words, hipStream_t s) {
  // (a fill kernel: a memset node of a captured graph is not to be relied on)
  hipLaunchKernelGGL(release_clear_kernel, dim3(blocks_for(words)), dim3(kThreads), 0, s, bits, words);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (n > 0) {
    hipLaunchKernelGGL(release_kernel, dim3(blocks_for(n)), dim3(kThreads), 0, s, pages, n, num_pages,
                       refs, bits, counts);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(release_list_kernel, dim3((unsigned)release_blocks(num_pages)), dim3(kThreads), 0,
                     s, n, num_pages, bits, counts, freed, num_freed);
  return hipGetLastError();
}

}  // namespace actkv
