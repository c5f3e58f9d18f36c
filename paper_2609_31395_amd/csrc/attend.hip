// attend.hip -- decode attention over the paged cache (actkv_attend): the newest tokens' queries
// against their request's entries, one length per (request, KV head).
//
// Bound by reading K and V: 4 D bytes per entry and KV head for 4 D flop per query row, of which
// there are G (8, say) per new token.  So the work is split over the cache's length into equal
// shares of 32-key steps, one per workgroup, whatever the lengths; each wave streams its steps of K
// and V from global memory straight into MFMA operands, and the pieces of a (request, head) that
// several workgroups hold are joined by a second kernel.  Short requests have a workgroup per item
// instead, which needs neither the plan nor the join (attend_direct has the rule and the figures).
//
// The mathematics of a piece, per query row: a shift m, l = sum 2^(x_t - m) and o = sum 2^(x_t - m) v_t
// over its entries, x_t = sm_scale log2(e) q.k_t.  Two pieces join as m = max(m1, m2),
// l = l1 2^(m1 - m) + l2 2^(m2 - m) and the same for o; out = o / l, LSE = (m + log2 l) ln 2.
//
// The newest tokens' own K and V, where the call brings them, are read from where the call has them,
// by the wave that also writes them to the cache, where nobody reads them in this call.
#include <type_traits>

#include "device_common.hpp"

namespace actkv {

namespace {

constexpr int kStep = kAttendStep;   // keys of a wave's step: two pages
static_assert(kStep == 2 * kPageSize, "a step is two pages");

// A row's shift is raised only when a logit passes it by this much (in powers of two): any shift
// gives the same sums to rounding while nothing overflows, and a rescaling costs a pass over o.
constexpr float kLazy = 8.0f;
constexpr float kNegInf = -__builtin_inff();
constexpr int kItemCost = 6;         // see item_cost
constexpr float kLn2 = 0.6931471805599453f;

// Waves of a workgroup: two on every SIMD, or one where the rows' registers leave no room for two.
// With equal shares it has a CU to itself; with a workgroup per item several may share one or follow each
// other.  A wave has one step in flight; two or four of them, or two workgroups to a CU, were no faster
// with equal shares (attend_batch the same; 64-element heads 78 against 73.5 us).
template <int D, int kRowTiles>
struct Shape {
  static constexpr int kWaves = attend_waves(D, 16 * kRowTiles);
  static constexpr int kThreads = kWaves * 64;
};

// A work item: a request, or, with kv_lens, a (request, KV head) pair.  Its new tokens, its entries
// that lie in the cache already and those that the call brings, and its steps: those of the cached
// entries, of which the last takes the others as well (none without a new token).
struct Item {
  int n, cached, fresh;
  __device__ __forceinline__ int cached_steps() const { return n > 0 ? ceil_div(cached, kStep) : 0; }
  __device__ __forceinline__ int steps() const { return max(cached_steps(), n > 0 && fresh > 0 ? 1 : 0); }
};
__device__ __forceinline__ Item item_of(const AttendArgs& a, int x) {
  const int r = a.kv_lens ? x / a.Hkv : x;
  Item it;
  it.n = a.q_lens[r];
  it.cached = a.seq_lens[r];
  if (a.kv_lens) it.cached = min(max(a.kv_lens[x], 0), it.cached);
  it.fresh = a.k_new ? min(it.n, it.cached) : 0;
  it.cached -= it.fresh;
  return it;
}

// What an item costs a workgroup beside its steps (its queries, page ids and the join of the waves'
// pieces, about 4 us), in steps of a workgroup of `hw` heads side by side (0.6 us of one).
__device__ __forceinline__ int item_cost(int hw) { return kItemCost / hw; }

// Equal shares of `total` cost for at most `grid` workgroups, the first `more` of them larger by one
// (no more workgroups than units of cost: each of them holds one at least).
struct Shares {
  int wgs, each, more;
  __device__ __forceinline__ Shares(int total, int grid) {
    wgs = min(total, grid);
    each = wgs > 0 ? total / wgs : 1;
    more = total - wgs * each;
  }
  __device__ __forceinline__ int begin(int b) const { return b * each + min(b, more); }
  __device__ __forceinline__ int holder(int unit) const {   // the workgroup whose share it is in
    const int large = more * (each + 1);
    return unit < large ? unit / (each + 1) : more + (unit - large) / each;
  }
};

// v, from where the compiler cannot trace it back: what is computed from it is computed there, and not
// held in registers across a loop before it.
__device__ __forceinline__ int opaque(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

__device__ __forceinline__ float xor_max(float v, int d) { return fmaxf(v, __shfl_xor(v, d, 64)); }
__device__ __forceinline__ float xor_sum(float v, int d) { return v + __shfl_xor(v, d, 64); }

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Operands of one step (32 keys of two pages), as loaded: lane l = 16 c + i holds, of K, 16 bytes
// of entry i of either page per 32 elements, and of V the 16th i of entries 4 c .. 4 c + 3 of either
// page.  The first is the A operand of S^T = K Q^T; its result leaves lane l with the logits of query
// row i for exactly the entries 4 c .. 4 c + 3 of either page, which is the B operand of
// O^T = V^T P^T for V in this order: the probabilities never change lanes.
template <int D>
struct Operands {
  static constexpr int kSteps = D / 32;         // MFMAs of a product over the head dimension
  static constexpr int kVWords = D / 32;        // 4-byte words of V per lane and entry
  u32x4 k[2][kSteps];
  uint32_t v[8][kVWords];
};

// A page's operands: `bytes` of K or V rows from p on; the lane's places in them.
template <int D>
__device__ __forceinline__ void load_k(Operands<D>& op, int sub, const char* p, int bytes, uint32_t off) {
  const __amdgpu_buffer_rsrc_t rs = buffer_over(p, bytes);
#pragma unroll
  for (int ks = 0; ks < Operands<D>::kSteps; ++ks)
    op.k[sub][ks] = __builtin_amdgcn_raw_buffer_load_b128(rs, off + 64 * ks, 0, 0);
}
template <int D>
__device__ __forceinline__ void load_v(Operands<D>& op, int sub, const char* p, int bytes,
                                       const uint32_t (&off)[4]) {
  const __amdgpu_buffer_rsrc_t rs = buffer_over(p, bytes);
#pragma unroll
  for (int y = 0; y < 4; ++y) {
    if constexpr (D == 128) {
      const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(rs, off[y], 0, 0);
#pragma unroll
      for (int z = 0; z < 4; ++z) op.v[4 * sub + y][z] = v[z];
    } else {
      const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(rs, off[y], 0, 0);
      op.v[4 * sub + y][0] = v[0];
      op.v[4 * sub + y][1] = v[1];
    }
  }
}

// Element e of the lane's 8 V rows as an MFMA operand: 16-bit halves of words e / 2.
template <int D>
__device__ __forceinline__ bf16x8 v_column(const Operands<D>& x, int e) {
  const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
  u32x4 r;
#pragma unroll
  for (int w = 0; w < 4; ++w)
    r[w] = __builtin_amdgcn_perm(x.v[2 * w + 1][e / 2], x.v[2 * w][e / 2], sel);
  return as_bf16x8(r);
}

template <int D, int kRowTiles>
struct Rows {
  static constexpr int kE = D / 16;   // columns of V a lane holds: o of row i, d = kE (4 c + v) + e
  bf16x8 q[kRowTiles][D / 32];
  f32x4 o[kRowTiles][kE];
  float m[kRowTiles], l[kRowTiles];   // l: over the lane's own entries
  int last[kRowTiles];                // entries below it are seen by the row
};

// Row `mrow` of a piece, `kN` elements of it from d on: the output (and, d = 0, the LSE) if the piece is
// the whole segment, else the workgroup's partial.
template <int D, int kN>
__device__ __forceinline__ void put_row(const AttendArgs& a, bool whole, int64_t slot, int q_off, int h,
                                        int mrow, int d, const float (&o)[kN], float m, float l) {
  if (whole) {
    const int j = mrow / a.G, g = mrow - j * a.G;
    const int64_t at = (int64_t)(q_off + j) * a.Hq + h * a.G + g;
    const float inv = l > 0.f ? 1.0f / l : 0.f;
    __bf16* out = reinterpret_cast<__bf16*>(a.out) + at * D + d;
#pragma unroll
    for (int e = 0; e < kN; ++e) out[e] = (__bf16)(o[e] * inv);
    if (a.lse && d == 0) a.lse[at] = m == kNegInf ? kNegInf : (m + __log2f(l)) * kLn2;
  } else {
    float* out = a.part_o + (slot * a.max_rows + mrow) * D + d;
#pragma unroll
    for (int e = 0; e < kN; ++e) out[e] = o[e];
    if (d == 0) a.part_ml[slot * a.max_rows + mrow] = make_float2(m, l);
  }
}

}  // namespace

// Waves of a workgroup: a.head_waves KV heads side by side (without kv_lens; their rows of a page
// alternate in memory, so that its reads arrive together), and the rest take every key_waves-th step
// of the workgroup's share each.
template <int D, int kRowTiles>
__global__ __launch_bounds__((Shape<D, kRowTiles>::kThreads), (Shape<D, kRowTiles>::kWaves / 4))
void attend_kernel(AttendArgs a) {
  using Op = Operands<D>;
  using Sh = Shape<D, kRowTiles>;
  constexpr int kE = D / 16, kWaves = Sh::kWaves, kThreads = Sh::kThreads;
  constexpr int kOStride = D + 4;
  __shared__ __align__(16) float o_s[kWaves][16][kOStride];
  __shared__ float m_s[kWaves][16], l_s[kWaves][16];
  __shared__ int64_t scan_s[17];
  __shared__ int first_s[6];
  const int tid = threadIdx.x, lane = tid & 63, c = lane >> 4, i16 = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hw = a.head_waves, kw = kWaves / hw;
  const int groups = a.kv_lens ? 1 : a.Hkv / hw;   // workgroups on one share, for the heads of a request
  const int items = a.kv_lens ? a.R * a.Hkv : a.R;
  const int b = blockIdx.x / groups;
  const int h_wave = a.kv_lens ? 0 : (int)(blockIdx.x % groups) * hw + w % hw, k_wave = w / hw;

  // a.direct: workgroup b has item b, all of it, and there is nothing to join.  Otherwise the plan: cost
  // and new tokens before each item (every workgroup finds its own share).
  const int fixed = item_cost(hw);
  auto cost_of = [&](const Item& i) { const int n_steps = i.steps(); return n_steps > 0 ? n_steps + fixed : 0; };
  Item it = {0, 0, 0};
  int c0 = 0, c1 = 1 << 30;
  if (a.direct) {
    const int r = a.kv_lens ? b / a.Hkv : b;
    int64_t own = 0, all;
    for (int x = tid; x < r; x += kThreads) own += a.q_lens[x];
    it = item_of(a, b);
    block_excl_scan_i64(own, scan_s, &all);
    if (tid == 0) {
      first_s[0] = b;
      first_s[1] = -fixed;
      first_s[2] = (int)all;
      first_s[3] = it.n;
      first_s[4] = it.cached;
      first_s[5] = it.fresh;
    }
    if (it.steps() == 0) {   // rows that see no entry, of every head of the workgroup
      const int rows = it.n * a.G, heads = a.kv_lens ? 1 : hw, h0 = a.kv_lens ? b % a.Hkv : (int)(blockIdx.x % groups) * hw;
      for (int y = tid; y < rows * heads * D; y += kThreads) {
        const int row = y / D, m = row % rows, j = m / a.G;
        const int64_t at = (all + j) * a.Hq + (h0 + row / rows) * a.G + (m - j * a.G);
        a.out[at * D + y % D] = 0;
        if (a.lse && y % D == 0) a.lse[at] = kNegInf;
      }
      return;
    }
    __syncthreads();
  } else {
    const int per = ceil_div(items, kThreads);
    int64_t own = 0;
    for (int x = tid * per; x < items && x < (tid + 1) * per; ++x) {
      it = item_of(a, x);
      own += ((int64_t)cost_of(it) << 32) + (!a.kv_lens || x % a.Hkv == 0 ? it.n : 0);
    }
    int64_t all;
    const int64_t before = block_excl_scan_i64(own, scan_s, &all);
    const int total = (int)(all >> 32);
    const Shares shares(total, gridDim.x / groups);
    c0 = b < shares.wgs ? shares.begin(b) : 0;
    c1 = b < shares.wgs ? shares.begin(b + 1) : 0;
    const int t_before = (int)(before >> 32);
    const bool mine = c0 < c1 && t_before <= c0 && c0 < t_before + (int)(own >> 32);
    if (mine || blockIdx.x == 0) {
      int t = t_before, q = (int)before;
      for (int x = tid * per; x < items && x < (tid + 1) * per; ++x) {
        if (per > 1) it = item_of(a, x);
        const int h = a.kv_lens ? x % a.Hkv : 0, cost = cost_of(it);
        if (blockIdx.x == 0) {
          a.start[x] = t;
          if (h == 0) a.q_off[a.kv_lens ? x / a.Hkv : x] = q;
        }
        if (mine && t <= c0 && c0 < t + cost) {
          first_s[0] = x;
          first_s[1] = t;
          first_s[2] = h == 0 ? q : q - it.n;
          first_s[3] = it.n;
          first_s[4] = it.cached;
          first_s[5] = it.fresh;
        }
        t += cost;
        if (h == 0) q += it.n;
      }
      if (blockIdx.x == 0 && tid == 0) a.start[items] = total;
    }
    if (c0 >= c1) return;
    __syncthreads();
  }
  int x = __builtin_amdgcn_readfirstlane(first_s[0]);
  int start = __builtin_amdgcn_readfirstlane(first_s[1]);
  int q_off = __builtin_amdgcn_readfirstlane(first_s[2]);
  it.n = __builtin_amdgcn_readfirstlane(first_s[3]);
  it.cached = __builtin_amdgcn_readfirstlane(first_s[4]);
  it.fresh = __builtin_amdgcn_readfirstlane(first_s[5]);

  const int64_t page_bytes = (int64_t)kPageSize * a.Hkv * D * 2;
  const int64_t v_plane = a.num_pages * page_bytes;
  const int row_bytes = a.Hkv * D * 2;
  const int32_t num_pages32 = (int32_t)(a.num_pages < INT32_MAX ? a.num_pages : INT32_MAX);

  for (;;) {
    const int r = a.kv_lens ? x / a.Hkv : x, h = a.kv_lens ? x % a.Hkv : h_wave;
    const int n = it.n, n_steps = it.steps(), cached_steps = it.cached_steps();
    // the workgroup's steps of the item (none where its share ends in the item's fixed cost)
    const int t0 = max(c0 - start - fixed, 0), t1 = min(c1 - start - fixed, n_steps);
    if (t0 < t1) {
      const bool whole = t0 == 0 && t1 == n_steps;
      // a workgroup leaves at most one piece that starts its item, and one that does not
      const int64_t slot = (int64_t)(2 * b + (t0 == 0 ? 1 : 0)) * a.Hkv_slots + (a.kv_lens ? 0 : h);
      const int rows = n * a.G, len = it.cached + it.fresh;

      Rows<D, kRowTiles> st;
#pragma unroll
      for (int rt = 0; rt < kRowTiles; ++rt) {
        const int m = rt * 16 + i16, j = m / a.G, gq = m - j * a.G;
        const bool real = m < rows;
        const uint16_t* src = a.q + (int64_t)(q_off + j) * a.q_stride + (h * a.G + gq) * D + 8 * c;
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks)
          st.q[rt][ks] = as_bf16x8(real ? *reinterpret_cast<const u32x4*>(src + 32 * ks)
                                        : u32x4{0u, 0u, 0u, 0u});
        st.last[rt] = a.causal && real ? len - n + j + 1 : len;
        st.m[rt] = kNegInf;
        st.l[rt] = 0.f;
#pragma unroll
        for (int e = 0; e < kE; ++e) st.o[rt][e] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      const int all_see = a.causal ? len - n + 1 : len;   // entries below it are seen by every row

      const int32_t* bt_row = a.bt + (int64_t)r * a.bt_stride;
      const int pages = ceil_div(len, kPageSize);
      const char* k_head = a.kv + h * D * 2;
      const uint32_t k_off = (uint32_t)(i16 * row_bytes + 16 * c);
      uint32_t v_off[4];   // (in the lane's offset: the bounds check takes a scalar one off the size)
#pragma unroll
      for (int y = 0; y < 4; ++y) v_off[y] = (uint32_t)((4 * c + y) * row_bytes + 2 * kE * i16);
      Op op;
      // this wave's steps: t_first and every kw-th from there, `steps` of them in the cache
      const int t_first = t0 + k_wave;
      const int steps = max(ceil_div(min(t1, cached_steps) - t_first, kw), 0);
      // Their pages, 32 steps at a time: lane l holds the id of page l % 2 of step l / 2 and how many
      // bytes of it, from this head's first row on, hold entries.  Loads past those bytes read as
      // zero and move nothing: the slots behind the entries (which may hold anything, and 0 times a
      // NaN of theirs would be one), and pages outside the pool.
      int32_t page_next = 0, page_now = 0, bytes_now = 0;
      auto fetch_pages = [&](int y) {
        page_next = bt_row[max(min(2 * (t_first + (y + (lane >> 1)) * kw) + (lane & 1), pages - 1), 0)];
      };
      auto take_pages = [&](int y) {
        const int step = y + (lane >> 1);
        const int held = min(it.cached - kPageSize * (2 * (t_first + step * kw) + (lane & 1)), kPageSize);
        const bool ok = step < steps && held > 0 && page_next >= 0 && page_next < num_pages32;
        page_now = ok ? page_next : 0;
        bytes_now = ok ? (held - 1) * row_bytes + 2 * D : 0;
      };
      auto issue = [&](int step) {
        if ((step & 31) == 0) {
          take_pages(step);
          fetch_pages(step + 32);
        }
        const char* at[2];
        int bytes[2];
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
          at[sub] = k_head + __builtin_amdgcn_readlane(page_now, 2 * (step & 31) + sub) * page_bytes;
          bytes[sub] = __builtin_amdgcn_readlane(bytes_now, 2 * (step & 31) + sub);
        }
        load_k<D>(op, 0, at[0], bytes[0], k_off);
        load_k<D>(op, 1, at[1], bytes[1], k_off);
        load_v<D>(op, 0, at[0] + v_plane, bytes[0], v_off);
        load_v<D>(op, 1, at[1] + v_plane, bytes[1], v_off);
      };
      // the new tokens of a step, as loaded, to their places in the cache
      auto write_new = [&](int j0, int c, int i16) {
        char* kv = const_cast<char*>(k_head);
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
          const int j = j0 + sub * kPageSize + i16, t = it.cached + j;
          if (j < it.fresh) {
            const int64_t page = bt_row[t / kPageSize];
            if (page >= 0 && page < a.num_pages)
#pragma unroll
              for (int ks = 0; ks < Op::kSteps; ++ks)
                *reinterpret_cast<u32x4*>(kv + page * page_bytes + t % kPageSize * row_bytes + 16 * c + 64 * ks) =
                    op.k[sub][ks];
          }
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const int jv = j0 + sub * kPageSize + 4 * c + y, tv = it.cached + jv;
            if (jv < it.fresh) {
              const int64_t page = bt_row[tv / kPageSize];
              char* dst = kv + v_plane + page * page_bytes + tv % kPageSize * row_bytes + 2 * kE * i16;
              if (page >= 0 && page < a.num_pages) {
                if constexpr (D == 128)
                  *reinterpret_cast<u32x4*>(dst) = u32x4{op.v[4 * sub + y][0], op.v[4 * sub + y][1],
                                                         op.v[4 * sub + y][2], op.v[4 * sub + y][3]};
                else
                  *reinterpret_cast<u32x2*>(dst) = u32x2{op.v[4 * sub + y][0], op.v[4 * sub + y][1]};
              }
            }
          }
        }
      };
      f32x4 acc[kRowTiles][2];
      auto scores = [&]() {
#pragma unroll
        for (int rt = 0; rt < kRowTiles; ++rt)
#pragma unroll
          for (int sub = 0; sub < 2; ++sub) {
            acc[rt][sub] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < Op::kSteps; ++ks)
              acc[rt][sub] = mfma16(as_bf16x8(op.k[sub][ks]), st.q[rt][ks], acc[rt][sub]);
          }
      };
      // 32 entries from key0 on, of which those below `end` count
      auto add = [&](int key0, int end) {
        const bool tail = key0 + kStep > min(all_see, end);
        bf16x8 hi[kRowTiles], lo[kRowTiles];
#pragma unroll
        for (int rt = 0; rt < kRowTiles; ++rt) {
          float y[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) y[k] = acc[rt][k / 4][k % 4];
          if (tail) {
            const int last = min(st.last[rt], end);
#pragma unroll
            for (int k = 0; k < 8; ++k)
              if (key0 + 16 * (k / 4) + 4 * c + k % 4 >= last) y[k] = kNegInf;
          }
          float mx = y[0];
#pragma unroll
          for (int k = 1; k < 8; ++k) mx = fmaxf(mx, y[k]);
          mx *= a.alpha;   // alpha > 0 keeps the order
          if (__ballot(mx > st.m[rt] + kLazy) != 0ull) {
            mx = xor_max(xor_max(mx, 16), 32);   // the row's, over its four lanes
            const float m = fmaxf(st.m[rt], mx), mf = m == kNegInf ? 0.f : m;
            const float f = fast_exp2(st.m[rt] - mf);
            st.m[rt] = m;
            st.l[rt] *= f;
#pragma unroll
            for (int e = 0; e < kE; ++e) st.o[rt][e] *= f;
          }
          const float m = st.m[rt] == kNegInf ? 0.f : st.m[rt];
          float p[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) p[k] = fast_exp2(__builtin_fmaf(y[k], a.alpha, -m));
          st.l[rt] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
          // p as the sum of two bf16 values: the rounding of p alone would add an error as large
          // as the output's own, and the kernel has matrix time to spare
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            hi[rt][k] = (__bf16)p[k];
            lo[rt][k] = (__bf16)(p[k] - (float)hi[rt][k]);
          }
        }
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          const bf16x8 v = v_column<D>(op, e);
#pragma unroll
          for (int rt = 0; rt < kRowTiles; ++rt) {
            st.o[rt][e] = mfma16(v, hi[rt], st.o[rt][e]);
            st.o[rt][e] = mfma16(v, lo[rt], st.o[rt][e]);
          }
        }
      };
      if (steps > 0) fetch_pages(0);
      // the newest tokens' own rows, by the wave that has (or would have) the last cached step
      if (it.fresh > 0 && t1 == n_steps && t0 < t1 && (t1 - 1 - t0) % kw == k_wave)
        for (int j0 = 0; j0 < it.fresh; j0 += kStep) {
          const int new_bytes = (int)(a.new_stride * 2);
          const int l2 = opaque(lane), c = l2 >> 4, i16 = l2 & 15;
          uint32_t off[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) off[y] = (uint32_t)((4 * c + y) * new_bytes + 2 * kE * i16);
#pragma unroll
          for (int sub = 0; sub < 2; ++sub) {
            const int j = j0 + sub * kPageSize, held = min(it.fresh - j, kPageSize);
            const int64_t at = ((int64_t)q_off + n - it.fresh + j) * a.new_stride + h * D;
            const int bytes = held > 0 ? (held - 1) * new_bytes + 2 * D : 0;
            load_k<D>(op, sub, reinterpret_cast<const char*>(a.k_new + at), bytes,
                      (uint32_t)(i16 * new_bytes + 16 * c));
            load_v<D>(op, sub, reinterpret_cast<const char*>(a.v_new + at), bytes, off);
          }
          write_new(j0, c, i16);
          scores();
          add(it.cached + j0, len);
        }
      for (int step = 0; step < steps; ++step) {
        issue(step);
        scores();
        add((t_first + step * kw) * kStep, it.cached);
      }
      const int tid2 = opaque(tid), lane2 = tid2 & 63, c2 = lane2 >> 4, i2 = lane2 & 15;
      // the pieces of a head's key waves joined, 16 rows at a time
      auto join_waves = [&](auto key_waves) {
        constexpr int kW = decltype(key_waves)::value, kH = kWaves / kW;
        static_assert(kW * kH == kWaves, "the waves of a workgroup, by keys and heads");
#pragma unroll
        for (int rt = 0; rt < kRowTiles; ++rt) {
          const float l = xor_sum(xor_sum(st.l[rt], 16), 32);
          if (lane2 < 16) {
            m_s[w][lane2] = st.m[rt];
            l_s[w][lane2] = l;
          }
          __syncthreads();
          float m = m_s[w % kH][i2];
#pragma unroll
          for (int k = 1; k < kW; ++k) m = fmaxf(m, m_s[w % kH + k * kH][i2]);
          const float f = st.m[rt] == kNegInf ? 0.f : fast_exp2(st.m[rt] - m);
#pragma unroll
          for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int e = 0; e < kE; e += 4)
              *reinterpret_cast<f32x4*>(&o_s[w][i2][kE * (4 * c2 + v) + e]) =
                  f32x4{st.o[rt][e][v], st.o[rt][e + 1][v], st.o[rt][e + 2][v], st.o[rt][e + 3][v]} * f;
          __syncthreads();
          // a row's kE elements at a time, 16 threads to a row, 16 rows of each head
          for (int y = tid2; y < 256 * kH; y += kThreads) {
            const int hh = y >> 8, row = (y >> 4) & 15, d = (y & 15) * kE, mrow = rt * 16 + row;
            if (mrow >= rows) continue;
            float mk[kW], mm = kNegInf, ll = 0.f, o[kE];
#pragma unroll
            for (int k = 0; k < kW; ++k) {
              mk[k] = m_s[hh + k * kH][row];
              mm = fmaxf(mm, mk[k]);
            }
#pragma unroll
            for (int k = 0; k < kW; ++k)
              ll += mk[k] == kNegInf ? 0.f : l_s[hh + k * kH][row] * fast_exp2(mk[k] - mm);
#pragma unroll
            for (int e = 0; e < kE; ++e) o[e] = 0.f;
#pragma unroll 1
            for (int k0 = 0; k0 < kW; k0 += 2)   // (two at a time: more would not fit the registers)
#pragma unroll
              for (int k = k0; k < k0 + 2; ++k)
#pragma unroll
                for (int e = 0; e < kE; e += 4) {
                  const f32x4 v = *reinterpret_cast<const f32x4*>(&o_s[hh + k * kH][row][d + e]);
                  o[e] += v[0]; o[e + 1] += v[1]; o[e + 2] += v[2]; o[e + 3] += v[3];
                }
            const int head = a.kv_lens ? h : h_wave - w % kH + hh;
            put_row<D>(a, whole, a.kv_lens ? slot : slot - h + head, q_off, head, mrow, d, o, mm, ll);
          }
          __syncthreads();   // o_s and m_s are written again
        }
      };
      if (kw == 1) {
        // the wave's rows are the piece's: register v of lane 16 c + i holds elements kE (4 c + v) .. of row i
#pragma unroll
        for (int rt = 0; rt < kRowTiles; ++rt) {
          const float l = xor_sum(xor_sum(st.l[rt], 16), 32);
          if (rt * 16 + i2 < rows) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              float o[kE];
#pragma unroll
              for (int e = 0; e < kE; ++e) o[e] = st.o[rt][e][v];
              put_row<D>(a, whole, slot, q_off, h, rt * 16 + i2, kE * (4 * c2 + v), o, st.m[rt], l);
            }
          }
        }
      } else if (kw == 2) {
        join_waves(std::integral_constant<int, 2>());
      } else if constexpr (kWaves == 8) {
        if (kw == 4) join_waves(std::integral_constant<int, 4>());
        else join_waves(std::integral_constant<int, 8>());
      } else {
        join_waves(std::integral_constant<int, 4>());
      }
    }
    start += cost_of(it);
    if (!a.kv_lens || h == a.Hkv - 1) q_off += n;
    if (a.direct || start >= c1) break;   // (there is cost left, so there is another item)
    const Item next = item_of(a, ++x);
    it.n = __builtin_amdgcn_readfirstlane(next.n);
    it.cached = __builtin_amdgcn_readfirstlane(next.cached);
    it.fresh = __builtin_amdgcn_readfirstlane(next.fresh);
  }
}

// The pieces of a segment (request and KV head) that several workgroups hold, and the rows of an empty
// one.  kWide: a workgroup per row, for long segments in many pieces; otherwise a wave per row
// (attend_draft, 5,120 rows of 2 or 3 pieces: 8 against 15.6 us).
constexpr int kJoinThreads = 256, kJoinWaves = kJoinThreads / 64;

template <int D, bool kWide>
__global__ __launch_bounds__(kJoinThreads) void attend_join_kernel(AttendArgs a, int grid) {
  constexpr int kLanes = D / 4, kBatch = 8;                      // lanes of a row of D
  constexpr int kSpan = kWide ? kJoinThreads : 64, kGroups = kSpan / kLanes;   // threads of a row
  __shared__ float weight[kWide ? kJoinThreads : 1];
  __shared__ float red[2][kJoinWaves];
  __shared__ __align__(16) float o_s[kWide ? kGroups : 1][D];
  const int s = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int mrow = kWide ? (int)blockIdx.y : (int)blockIdx.y * kJoinWaves + w;
  const int t = kWide ? tid : lane;   // within the row's threads
  const int r = s / a.Hkv, h = s % a.Hkv, n = a.q_lens[r];
  const int x = a.kv_lens ? s : r, groups = a.kv_lens ? 1 : a.Hkv / a.head_waves;
  const int cs = a.start[x], ce = a.start[x + 1], total = a.start[a.kv_lens ? a.R * a.Hkv : a.R];
  const int q_off = a.q_off[r];
  if (mrow >= n * a.G) return;
  const int j = mrow / a.G, gq = mrow - j * a.G;
  const int64_t at = (int64_t)(q_off + j) * a.Hq + h * a.G + gq;
  if (cs == ce) {
    for (int d = t; d < D; d += kSpan) reinterpret_cast<uint16_t*>(a.out)[at * D + d] = 0;
    if (t == 0 && a.lse) a.lse[at] = kNegInf;
    return;
  }
  const Shares shares(total, grid / groups);
  const int first = shares.holder(cs + item_cost(a.head_waves)), last = shares.holder(ce - 1);
  if (first == last) return;   // written by that workgroup
  const int pieces = last - first + 1;
  auto slot_of = [&](int p) {   // the first piece starts the item
    return ((int64_t)(2 * (first + p) + (p == 0 ? 1 : 0)) * a.Hkv_slots + (a.kv_lens ? 0 : h)) * a.max_rows + mrow;
  };
  float m = kNegInf;
  const int grp = t / kLanes, d4 = (t % kLanes) * 4;
  float l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  // kSpan pieces at a time: the first kBatch rows of a group's set out before the pieces' weights (in
  // LDS, or one per lane) are known
  for (int p0 = 0; p0 < pieces; p0 += kSpan) {
    const int here = min(pieces - p0, kSpan);
    f32x4 v[kBatch];
    auto load_rows = [&](int k0) {
#pragma unroll
      for (int k = 0; k < kBatch; ++k)
        v[k] = *reinterpret_cast<const f32x4*>(
            a.part_o + slot_of(p0 + min(k0 + k * kGroups + grp, here - 1)) * D + d4);
    };
    const float2 ml = t < here ? a.part_ml[slot_of(p0 + t)] : make_float2(kNegInf, 0.f);
    load_rows(0);
    if (p0 == 0) {   // the row's shift; past kSpan pieces, from all of them
      m = ml.x;
      for (int p = t + kSpan; p < pieces; p += kSpan) m = fmaxf(m, a.part_ml[slot_of(p)].x);
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) m = xor_max(m, d);
      if constexpr (kWide) {
        if (lane == 0) red[0][w] = m;
        __syncthreads();
        m = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
      }
    }
    const float f = ml.x == kNegInf ? 0.f : fast_exp2(ml.x - m);
    l += ml.y * f;
    if constexpr (kWide) {
      weight[t] = f;
      __syncthreads();
    }
    for (int k0 = 0; k0 < here; k0 += kGroups * kBatch) {
      if (k0 > 0) load_rows(k0);
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int p = k0 + k * kGroups + grp;
        float g;
        if constexpr (kWide) g = weight[min(p, kSpan - 1)];
        else g = __shfl(f, p & 63, 64);
        o += v[k] * (p < here ? g : 0.f);
      }
    }
    if constexpr (kWide) __syncthreads();   // weight is written again
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) l = xor_sum(l, d);
  if constexpr (kWide) {
    if (lane == 0) red[1][w] = l;
    *reinterpret_cast<f32x4*>(&o_s[grp][d4]) = o;
    __syncthreads();
    l = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
    if (t >= kLanes) return;
    o = *reinterpret_cast<const f32x4*>(&o_s[0][d4]);
#pragma unroll
    for (int k = 1; k < kGroups; ++k) o += *reinterpret_cast<const f32x4*>(&o_s[k][d4]);
  } else {
#pragma unroll
    for (int d = 32; d >= kLanes; d >>= 1)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = xor_sum(o[e], d);
    if (t >= kLanes) return;
  }
  const float inv = l > 0.f ? 1.0f / l : 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) reinterpret_cast<__bf16*>(a.out)[at * D + d4 + e] = (__bf16)(o[e] * inv);
  if (t == 0 && a.lse) a.lse[at] = m == kNegInf ? kNegInf : (m + __log2f(l)) * kLn2;
}

hipError_t launch_attend(AttendArgs a, int64_t steps, hipStream_t s) {
  int64_t wgs = 0;
  auto run = [&](auto d, auto tiles) {
    constexpr int D = decltype(d)::value, kTiles = decltype(tiles)::value;
    using Sh = Shape<D, kTiles>;
    // a workgroup per CU, at most one per step
    const int groups = a.kv_lens ? 1 : a.Hkv / a.head_waves;
    wgs = device_cus();
    if (wgs > kAttendMaxWgs) wgs = kAttendMaxWgs;
    wgs /= groups;
    const int64_t shared_steps = a.kv_lens ? steps * a.Hkv : steps;
    if (wgs > shared_steps) wgs = shared_steps;
    wgs = (wgs < 1 ? 1 : wgs) * groups;
    if (a.direct) wgs = (int64_t)groups * (a.kv_lens ? a.R * a.Hkv : a.R);
    hipLaunchKernelGGL((attend_kernel<D, kTiles>), dim3((unsigned)wgs), dim3(Sh::kThreads), 0, s, a);
  };
  auto run_d = [&](auto d) {
    switch ((a.max_rows + 15) / 16) {
      case 1: run(d, std::integral_constant<int, 1>()); break;
      case 2: run(d, std::integral_constant<int, 2>()); break;
      case 3: run(d, std::integral_constant<int, 3>()); break;
      default: run(d, std::integral_constant<int, 4>()); break;
    }
  };
  if (a.D == 128) run_d(std::integral_constant<int, 128>());
  else run_d(std::integral_constant<int, 64>());
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.direct) return e;
  // more than 16 pieces to a segment in the mean: a workgroup per row
  const int64_t gangs = a.kv_lens ? wgs : wgs / (a.Hkv / a.head_waves);
  const bool wide = gangs > 16 * (int64_t)(a.kv_lens ? a.R * a.Hkv : a.R);
  const dim3 grid((unsigned)(a.R * a.Hkv), (unsigned)(wide ? a.max_rows : (a.max_rows + kJoinWaves - 1) / kJoinWaves));
  auto join = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kJoinThreads), 0, s, a, (int)wgs);
  };
  if (a.D == 128) wide ? join(attend_join_kernel<128, true>) : join(attend_join_kernel<128, false>);
  else wide ? join(attend_join_kernel<64, true>) : join(attend_join_kernel<64, false>);
  return hipGetLastError();
}

}  // namespace actkv
