// attend.hip -- decode attention over the paged cache (actkv_attend): the newest tokens' queries
// against their request's entries, one length per (request, KV head).
//
// Bound by reading K and V: 4 D bytes per entry and KV head for 4 D flop per query row, of which
// there are G (8, say) per new token.  So the work is split over the cache's length into equal
// shares of 128-key units, one per workgroup, whatever the lengths; each wave streams 32-key steps
// of K and V from global memory straight into MFMA operands, and the pieces of a (request, head)
// that several workgroups hold are joined by a second kernel.
//
// The mathematics of a piece, per query row: a shift m, l = sum 2^(x_t - m) and o = sum 2^(x_t - m) v_t
// over its entries, x_t = sm_scale log2(e) q.k_t.  Two pieces join as m = max(m1, m2),
// l = l1 2^(m1 - m) + l2 2^(m2 - m) and the same for o; out = o / l, LSE = (m + log2 l) ln 2.
#include <type_traits>

#include "device_common.hpp"

namespace actkv {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kStep = 32;                  // keys of a wave's step: two pages
constexpr int kUnit = kStep * kWaves;      // keys of a work unit
static_assert(kUnit == kAttendUnit, "the host counts the same units");

// A row's shift is raised only when a logit passes it by this much (in powers of two): any shift
// gives the same sums to rounding while nothing overflows, and a rescaling costs a pass over o.
constexpr float kLazy = 8.0f;
constexpr float kNegInf = -__builtin_inff();

// Segment s = request * Hkv + head: its entries, and its work units (none without a new token).
struct Segment {
  int len, n;
};
__device__ __forceinline__ Segment segment(const AttendArgs& a, int s) {
  const int r = s / a.Hkv;
  Segment g;
  g.n = a.q_lens[r];
  g.len = a.seq_lens[r];
  if (a.kv_lens) g.len = min(max(a.kv_lens[s], 0), g.len);
  return g;
}
__device__ __forceinline__ int units_of(const Segment& g) {
  return g.n > 0 ? ceil_div(g.len, kUnit) : 0;
}

// Equal shares of `total` units for at most `grid` workgroups, the first `more` of them a unit larger
// (no more workgroups than units: each of them holds one at least).
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

__device__ __forceinline__ float xor_max(float v, int d) { return fmaxf(v, __shfl_xor(v, d, 64)); }
__device__ __forceinline__ float xor_sum(float v, int d) { return v + __shfl_xor(v, d, 64); }

// Steps of K and V a wave has in flight, and workgroups per CU (a wave of each on every SIMD), by what
// fits the registers.
template <int D, int kRowTiles>
struct Shape {
  static constexpr int kRing = (D == 128 ? kRowTiles == 1 : kRowTiles <= 2) ? 2 : 1;
  static constexpr int kWgs = D == 128 ? (kRowTiles <= 2 ? 2 : 1) : (kRowTiles == 1 ? 3 : 2);
};

// Operands of one step (32 keys of two pages), as loaded: lane l = 16 c + i holds, of K, 16 bytes
// of entry i of either page per 32 elements, and of V the 16th i of entries 4 c .. 4 c + 3 of either
// page.  The first is the A operand of S^T = K Q^T; its result leaves lane l with the logits of query
// row i for exactly the entries 4 c .. 4 c + 3 of either page, which is the B operand of
// O^T = V^T P^T for V in this order: the probabilities never change lanes.
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

template <int D>
struct Operands {
  static constexpr int kSteps = D / 32;         // MFMAs of a product over the head dimension
  static constexpr int kVWords = D / 32;        // 4-byte words of V per lane and entry
  u32x4 k[2][kSteps];
  uint32_t v[8][kVWords];
};

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

}  // namespace

template <int D, int kRowTiles>
__global__ __launch_bounds__(kThreads, (Shape<D, kRowTiles>::kWgs)) void attend_kernel(AttendArgs a) {
  using Op = Operands<D>;
  constexpr int kE = D / 16, kRing = Shape<D, kRowTiles>::kRing;
  constexpr int kOStride = D + 4;
  __shared__ __align__(16) float o_s[kWaves][16][kOStride];
  __shared__ float m_s[kWaves][16], l_s[kWaves][16];
  __shared__ int64_t scan_s[17];
  __shared__ int first_s[5];
  const int tid = threadIdx.x, lane = tid & 63, c = lane >> 4, i16 = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int S = a.R * a.Hkv, b = blockIdx.x;

  // the plan: units and new tokens before each segment (every workgroup finds its own share)
  const int per = ceil_div(S, kThreads);
  int64_t own = 0;
  Segment g = {0, 0};   // this thread's (last) segment
  for (int x = tid * per; x < S && x < (tid + 1) * per; ++x) {
    g = segment(a, x);
    own += ((int64_t)units_of(g) << 32) + (x % a.Hkv == 0 ? g.n : 0);
  }
  int64_t all;
  const int64_t before = block_excl_scan_i64(own, scan_s, &all);
  const int total = (int)(all >> 32);
  const Shares shares(total, gridDim.x);
  const int c0 = b < shares.wgs ? shares.begin(b) : 0, c1 = b < shares.wgs ? shares.begin(b + 1) : 0;
  const int u_before = (int)(before >> 32);
  const bool mine = c0 < c1 && u_before <= c0 && c0 < u_before + (int)(own >> 32);
  if (mine || b == 0) {
    int u = u_before, q = (int)before;
    for (int x = tid * per; x < S && x < (tid + 1) * per; ++x) {
      if (per > 1) g = segment(a, x);
      const int h = x % a.Hkv, n_units = units_of(g);
      if (b == 0) {
        a.seg_start[x] = u;
        if (h == 0) a.q_off[x / a.Hkv] = q;
      }
      if (mine && u <= c0 && c0 < u + n_units) {
        first_s[0] = x;
        first_s[1] = u;
        first_s[2] = h == 0 ? q : q - g.n;
        first_s[3] = g.len;
        first_s[4] = g.n;
      }
      u += n_units;
      if (h == 0) q += g.n;
    }
    if (b == 0 && tid == 0) a.seg_start[S] = total;
  }
  if (c0 >= c1) return;
  __syncthreads();
  int s = __builtin_amdgcn_readfirstlane(first_s[0]);
  int start = __builtin_amdgcn_readfirstlane(first_s[1]);
  int q_off = __builtin_amdgcn_readfirstlane(first_s[2]);
  int len = __builtin_amdgcn_readfirstlane(first_s[3]);
  int n = __builtin_amdgcn_readfirstlane(first_s[4]);

  const int64_t page_bytes = (int64_t)kPageSize * a.Hkv * D * 2;
  const int64_t v_plane = a.num_pages * page_bytes;
  const int row_bytes = a.Hkv * D * 2;
  const int32_t num_pages32 = (int32_t)(a.num_pages < INT32_MAX ? a.num_pages : INT32_MAX);

  for (;;) {
    const int r = s / a.Hkv, h = s % a.Hkv;
    const int n_units = n > 0 ? ceil_div(len, kUnit) : 0;
    if (n_units > 0) {
      const int u0 = max(c0 - start, 0), u1 = min(c1 - start, n_units);
      const bool whole = u0 == 0 && u1 == n_units;
      const int rows = n * a.G;
      const int keys_end = min(u1 * kUnit, len);
      const int pages = ceil_div(len, kPageSize);

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
      const char* k_head = a.kv + h * D * 2;
      const uint32_t k_off = (uint32_t)(i16 * row_bytes + 16 * c);
      uint32_t v_off[4];   // (in the lane's offset: the bounds check takes a scalar one off the size)
#pragma unroll
      for (int y = 0; y < 4; ++y) v_off[y] = (uint32_t)((4 * c + y) * row_bytes + 2 * kE * i16);
      Op ring[kRing];
      // this wave's steps: u0 * kWaves + w, and every kWaves-th from there
      const int i_first = u0 * kWaves + w;
      const int steps = max(ceil_div(ceil_div(keys_end, kStep) - i_first, kWaves), 0);
      // Their pages, 32 steps at a time: lane l holds the id of page l % 2 of step l / 2 and how many
      // bytes of it, from this head's first row on, hold entries.  Loads past those bytes read as
      // zero and move nothing: the slots behind the entries (which may hold anything, and 0 times a
      // NaN of theirs would be one), pages outside the pool, and steps past the wave's last, which
      // are issued like the others so that every wait counts the same loads.
      int32_t page_next = 0, page_now = 0, bytes_now = 0;
      auto fetch_pages = [&](int x) {
        page_next = bt_row[min(2 * (i_first + (x + (lane >> 1)) * kWaves) + (lane & 1), pages - 1)];
      };
      auto take_pages = [&](int x) {
        const int step = x + (lane >> 1);
        const int held = min(len - kPageSize * (2 * (i_first + step * kWaves) + (lane & 1)), kPageSize);
        const bool ok = step < steps && held > 0 && page_next >= 0 && page_next < num_pages32;
        page_now = ok ? page_next : 0;
        bytes_now = ok ? (held - 1) * row_bytes + 2 * D : 0;
      };
      auto issue = [&](int slot, int x) {   // step x of the wave
        if ((x & 31) == 0) {
          take_pages(x);
          fetch_pages(x + 32);
        }
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
          const int64_t page = __builtin_amdgcn_readlane(page_now, 2 * (x & 31) + sub);
          const int bytes = __builtin_amdgcn_readlane(bytes_now, 2 * (x & 31) + sub);
          const char* kp = k_head + page * page_bytes;
          const __amdgpu_buffer_rsrc_t kr = buffer_over(kp, bytes), vr = buffer_over(kp + v_plane, bytes);
#pragma unroll
          for (int ks = 0; ks < Op::kSteps; ++ks)
            ring[slot].k[sub][ks] = __builtin_amdgcn_raw_buffer_load_b128(kr, k_off + 64 * ks, 0, 0);
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            if constexpr (D == 128) {
              const u32x4 t = __builtin_amdgcn_raw_buffer_load_b128(vr, v_off[y], 0, 0);
#pragma unroll
              for (int z = 0; z < 4; ++z) ring[slot].v[4 * sub + y][z] = t[z];
            } else {
              const u32x2 t = __builtin_amdgcn_raw_buffer_load_b64(vr, v_off[y], 0, 0);
              ring[slot].v[4 * sub + y][0] = t[0];
              ring[slot].v[4 * sub + y][1] = t[1];
            }
          }
        }
      };
      auto compute = [&](int slot, int step) {
        Op& x = ring[slot];
        const int key0 = (i_first + step * kWaves) * kStep;
        const bool tail = key0 + kStep > all_see;
        bf16x8 hi[kRowTiles], lo[kRowTiles];
#pragma unroll
        for (int rt = 0; rt < kRowTiles; ++rt) {
          f32x4 acc[2];
#pragma unroll
          for (int sub = 0; sub < 2; ++sub) {
            acc[sub] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < Op::kSteps; ++ks)
              acc[sub] = mfma16(as_bf16x8(x.k[sub][ks]), st.q[rt][ks], acc[sub]);
          }
          float y[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) y[k] = acc[k / 4][k % 4];
          if (tail) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
              if (key0 + 16 * (k / 4) + 4 * c + k % 4 >= st.last[rt]) y[k] = kNegInf;
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
          const bf16x8 v = v_column<D>(x, e);
#pragma unroll
          for (int rt = 0; rt < kRowTiles; ++rt) {
            st.o[rt][e] = mfma16(v, hi[rt], st.o[rt][e]);
            st.o[rt][e] = mfma16(v, lo[rt], st.o[rt][e]);
          }
        }
      };
      if (steps > 0) {
        fetch_pages(0);
#pragma unroll
        for (int j = 0; j < kRing; ++j) issue(j, j);
        for (int x = 0; x < steps; x += kRing) {
#pragma unroll
          for (int j = 0; j < kRing; ++j) {
            if (j == 0 || x + j < steps) compute(j, x + j);
            issue(j, x + j + kRing);
          }
        }
      }
      // the four waves' pieces joined, 16 rows at a time
#pragma unroll
      for (int rt = 0; rt < kRowTiles; ++rt) {
        const float l = xor_sum(xor_sum(st.l[rt], 16), 32);
        if (lane < 16) {
          m_s[w][lane] = st.m[rt];
          l_s[w][lane] = l;
        }
        __syncthreads();
        float m = m_s[0][i16];
#pragma unroll
        for (int k = 1; k < kWaves; ++k) m = fmaxf(m, m_s[k][i16]);
        const float f = st.m[rt] == kNegInf ? 0.f : fast_exp2(st.m[rt] - m);
#pragma unroll
        for (int v = 0; v < 4; ++v)
#pragma unroll
          for (int e = 0; e < kE; e += 4)
            *reinterpret_cast<f32x4*>(&o_s[w][i16][kE * (4 * c + v) + e]) =
                f32x4{st.o[rt][e][v], st.o[rt][e + 1][v], st.o[rt][e + 2][v], st.o[rt][e + 3][v]} * f;
        __syncthreads();
        // 16 threads to a row, kE elements each
        const int row = tid >> 4, d = (tid & 15) * kE, mrow = rt * 16 + row;
        if (mrow < rows) {
          float mm = m_s[0][row], ll = 0.f;
#pragma unroll
          for (int k = 1; k < kWaves; ++k) mm = fmaxf(mm, m_s[k][row]);
#pragma unroll
          for (int k = 0; k < kWaves; ++k)
            ll += m_s[k][row] == kNegInf ? 0.f : l_s[k][row] * fast_exp2(m_s[k][row] - mm);
          float o[kE];
#pragma unroll
          for (int e = 0; e < kE; ++e) o[e] = 0.f;
#pragma unroll
          for (int k = 0; k < kWaves; ++k)
#pragma unroll
            for (int e = 0; e < kE; ++e) o[e] += o_s[k][row][d + e];
          if (whole) {
            const int j = mrow / a.G, gq = mrow - j * a.G;
            const int64_t at = (int64_t)(q_off + j) * a.Hq + h * a.G + gq;
            const float inv = ll > 0.f ? 1.0f / ll : 0.f;
#pragma unroll
            for (int e = 0; e < kE; ++e)
              reinterpret_cast<__bf16*>(a.out)[at * D + d + e] = (__bf16)(o[e] * inv);
            if (a.lse && d == 0)
              a.lse[at] = mm == kNegInf ? kNegInf : (mm + __log2f(ll)) * 0.6931471805599453f;
          } else {
            const int64_t slot = (2 * (int64_t)b + (start > c0 ? 1 : 0)) * a.max_rows + mrow;
#pragma unroll
            for (int e = 0; e < kE; ++e) a.part_o[slot * D + d + e] = o[e];
            if (d == 0) a.part_ml[slot] = make_float2(mm, ll);
          }
        }
        __syncthreads();   // o_s and m_s are written again
      }
    }
    start += n_units;
    if (h == a.Hkv - 1) q_off += n;
    if (start >= c1) break;   // (there are units left, so there is another segment)
    const Segment next = segment(a, ++s);
    len = __builtin_amdgcn_readfirstlane(next.len);
    n = __builtin_amdgcn_readfirstlane(next.n);
  }
}

// One workgroup per (segment, query row): the pieces of a segment that several workgroups hold, and
// the rows of an empty segment.
template <int D>
__global__ __launch_bounds__(kThreads) void attend_join_kernel(AttendArgs a, int grid) {
  constexpr int kLanes = D / 4, kGroups = kThreads / kLanes;
  __shared__ float weight[kAttendMaxWgs];
  __shared__ float red[2][kWaves];
  __shared__ __align__(16) float o_s[kGroups][D];
  const int s = blockIdx.x, mrow = blockIdx.y, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int r = s / a.Hkv, h = s % a.Hkv, n = a.q_lens[r];
  if (mrow >= n * a.G) return;
  const int S = a.R * a.Hkv;
  const int cs = a.seg_start[s], ce = a.seg_start[s + 1], total = a.seg_start[S];
  const int j = mrow / a.G, gq = mrow - j * a.G;
  const int64_t at = (int64_t)(a.q_off[r] + j) * a.Hq + h * a.G + gq;
  if (cs == ce) {
    if (tid < D) reinterpret_cast<uint16_t*>(a.out)[at * D + tid] = 0;
    if (tid == 0 && a.lse) a.lse[at] = kNegInf;
    return;
  }
  const Shares shares(total, grid);
  const int first = shares.holder(cs), last = shares.holder(ce - 1);
  if (first == last) return;   // written by that workgroup
  const int pieces = last - first + 1;
  // only the first piece can be its workgroup's second
  const int second = shares.begin(first) < cs ? 1 : 0;
  auto slot_of = [&](int p) {
    return (int64_t)(2 * (first + p) + (p == 0 ? second : 0)) * a.max_rows + mrow;
  };
  float m = kNegInf;
  for (int p = tid; p < pieces; p += kThreads) m = fmaxf(m, a.part_ml[slot_of(p)].x);
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) m = xor_max(m, d);
  if (lane == 0) red[0][w] = m;
  __syncthreads();
  m = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  float l = 0.f;
  for (int p = tid; p < pieces; p += kThreads) {
    const float2 ml = a.part_ml[slot_of(p)];
    const float f = ml.x == kNegInf ? 0.f : fast_exp2(ml.x - m);
    weight[p] = f;
    l += ml.y * f;
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) l = xor_sum(l, d);
  if (lane == 0) red[1][w] = l;
  __syncthreads();
  l = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
  const int grp = tid / kLanes, d4 = (tid % kLanes) * 4;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int p = grp; p < pieces; p += kGroups)
    o += *reinterpret_cast<const f32x4*>(a.part_o + slot_of(p) * D + d4) * weight[p];
  *reinterpret_cast<f32x4*>(&o_s[grp][d4]) = o;
  __syncthreads();
  if (tid < D) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kGroups; ++k) v += o_s[k][tid];
    reinterpret_cast<__bf16*>(a.out)[at * D + tid] = (__bf16)(l > 0.f ? v / l : 0.f);
    if (tid == 0 && a.lse)
      a.lse[at] = m == kNegInf ? kNegInf : (m + __log2f(l)) * 0.6931471805599453f;
  }
}

// The newest tokens' K and V rows into the entries kv_lens - n + j.  One thread per 16 bytes of both;
// grid: (ceil(most rows of a request * pieces of a row / 256), requests).
__global__ __launch_bounds__(kThreads) void append_kernel(AttendArgs a, const uint16_t* k_new,
                                                          const uint16_t* v_new, int64_t stride) {
  __shared__ int64_t scan_s[17];
  const int r = blockIdx.y, n = a.q_lens[r];
  int64_t q_off = 0, mine = 0;
  for (int x = threadIdx.x; x < r; x += kThreads) mine += a.q_lens[x];
  block_excl_scan_i64(mine, scan_s, &q_off);
  const int per_row = a.Hkv * a.D / 8;
  const int64_t x = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (x >= (int64_t)n * per_row) return;
  const int j = (int)(x / per_row), piece = (int)(x % per_row), h = piece / (a.D / 8);
  const Segment g = segment(a, r * a.Hkv + h);
  const int t = g.len - n + j;
  if (t < 0) return;
  const int64_t page = a.bt[(int64_t)r * a.bt_stride + t / kPageSize];
  if (page < 0 || page >= a.num_pages) return;
  const int64_t plane = a.num_pages * kPageSize * a.Hkv * a.D;
  uint16_t* dst = reinterpret_cast<uint16_t*>(const_cast<char*>(a.kv)) +
                  (page * kPageSize + t % kPageSize) * a.Hkv * a.D + piece * 8;
  const int64_t src = (q_off + j) * stride + piece * 8;
  *reinterpret_cast<u32x4*>(dst) = *reinterpret_cast<const u32x4*>(k_new + src);
  *reinterpret_cast<u32x4*>(dst + plane) = *reinterpret_cast<const u32x4*>(v_new + src);
}

hipError_t launch_append(const AttendArgs& a, int64_t max_n, const void* k_new, const void* v_new,
                         int64_t stride, hipStream_t s) {
  const int64_t pieces = max_n * a.Hkv * a.D / 8;
  hipLaunchKernelGGL(append_kernel, dim3((unsigned)((pieces + kThreads - 1) / kThreads), (unsigned)a.R),
                     dim3(kThreads), 0, s, a, static_cast<const uint16_t*>(k_new),
                     static_cast<const uint16_t*>(v_new), stride);
  return hipGetLastError();
}

hipError_t launch_attend(const AttendArgs& a, int64_t units, hipStream_t s) {
  int64_t wgs = 0;
  auto run = [&](auto d, auto tiles) {
    constexpr int D = decltype(d)::value, kTiles = decltype(tiles)::value;
    wgs = (int64_t)Shape<D, kTiles>::kWgs * device_cus();
    if (wgs > kAttendMaxWgs) wgs = kAttendMaxWgs;
    if (wgs > units) wgs = units;
    if (wgs < 1) wgs = 1;
    hipLaunchKernelGGL((attend_kernel<D, kTiles>), dim3((unsigned)wgs), dim3(kThreads), 0, s, a);
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
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)(a.R * a.Hkv), (unsigned)a.max_rows);
  if (a.D == 128)
    hipLaunchKernelGGL(attend_join_kernel<128>, grid, dim3(kThreads), 0, s, a, (int)wgs);
  else
    hipLaunchKernelGGL(attend_join_kernel<64>, grid, dim3(kThreads), 0, s, a, (int)wgs);
  return hipGetLastError();
}

}  // namespace actkv
