// The key/value cache in pages: rows appended to it (with the rotary
// embedding), the attention of new rows over a sequence's cached ones, and
// the same where all sequences of a batch share their first rows.
//
// Layout: a pool of pages, each of page_size (a power of two, from 16 on) rows
// [k | v], kvd = kv_heads * head_dim elements each; row r of sequence b is row
// r % page_size of page table[b][r / page_size]. A page id outside the pool
// stands for a page of zeros, and nothing is written to it.
//
//   append:    x'_i = x_i cos - x_{i + hd/2} sin, x'_{i + hd/2} = x_{i + hd/2} cos + x_i sin
//              with the angle pos theta^(-2i/hd), for k and q; v as it is
//   attention: s_j = scale q . k_j for the keys j that the row sees,
//              out = sum_j exp(s_j) v_j / sum_j exp(s_j),  lse = log sum_j exp(s_j);
//              a row that sees no key: out = 0, lse = -inf
//
// New row r of sequence b, of its n, is the cached row len - n + r; under the
// causal mask it sees the rows up to itself, else all len.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "zsa_internal.h"

namespace zsa {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kNoReference = -3.402823466e38f;  // a reference maximum of no key: the lowest number, from which an infinite score is infinitely far

// ---------------------------------------------------------------------------
// append
// ---------------------------------------------------------------------------
constexpr int kAppendRows = 8;  // most rows of a workgroup

// sequence of row t: cu[b] <= t < cu[b + 1] (t below cu[B]). One row per
// sequence, as in generation, needs no search.
__device__ __forceinline__ int sequence_of(const int32_t* __restrict__ cu, int B, int t) {
  if (t < B && cu[t] <= t && t < cu[t + 1]) return t;
  int lo = 0, hi = B - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (t < cu[mid + 1])
      hi = mid;
    else
      lo = mid + 1;
  }
  return lo;
}

// past the L2, which the next launch's readers on other XCDs cannot use anyway
template <typename T>
__device__ __forceinline__ void store16(T* p, const uint4& v) {
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), reinterpret_cast<u32x4*>(p));
}

// A workgroup takes `rows` rows: where each goes and its angles' (cos, sin) are
// found once for all its heads, then every thread moves 16 bytes at a time (a
// rotation's two halves together). Bound by the bytes: every row is read and
// written once. 16384 rows, 32 heads of 128 on 8, two rows a workgroup: 76.2 us
// (5.29 TB/s); with ordinary stores 79.7; with eight rows 81.8, with both 84.0;
// with two items' loads ahead of their stores 84.8.
template <typename T>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedAppend a, int rows) {
  constexpr int V = Vec16<T>::N;
  __shared__ float2 cs[kAppendRows][kMaxHalfHead];
  __shared__ int64_t dst[kAppendRows];  // element in the pool, or -1
  const int t0 = blockIdx.x * rows, nt = min(rows, a.T - t0);
  const int tid = threadIdx.x, half = a.hd / 2;
  if (tid < nt) {
    const int t = t0 + tid, b = sequence_of(a.cu, a.B, t);
    const int lo = a.cu[b], n = a.cu[b + 1] - lo;
    const int64_t row = static_cast<int64_t>(a.kv_len[b]) - n + (t - lo);
    int64_t d = -1;
    if (row >= 0 && (row >> a.at.shift) < a.at.max_pages) {
      const int page = a.at.table[b * a.at.table_stride + (row >> a.at.shift)];
      if (page >= 0 && page < a.at.n_pages)
        d = page * a.at.page_stride + (row & ((1 << a.at.shift) - 1)) * 2 * a.at.kvd;
    }
    dst[tid] = d;
  }
  if (a.pos != nullptr)
    for (int i = tid; i < nt * half; i += 256) {
      float s, c;
      rope_angle(a.pos[t0 + i / half], a.inv_freq[i % half], &s, &c);
      cs[i / half][i % half] = make_float2(c, s);
    }
  __syncthreads();
  // a row's items: pairs of 16 bytes of the rotated heads, then 16 bytes of the others
  const int hc = half / V, nq = a.q != nullptr ? a.H * hc : 0;
  const int nrot = a.pos != nullptr ? nq + a.Hkv * hc : 0;
  const int nk = a.pos != nullptr ? 0 : a.at.kvd / V, items = nrot + nk + a.at.kvd / V;
  T* pool = static_cast<T*>(a.at.pool);
  for (int i = tid; i < nt * items; i += 256) {
    const int r = i / items, e = i - r * items;
    const int64_t t = t0 + r, d = dst[r];
    if (e < nrot) {
      const bool isq = e < nq;
      const int f = isq ? e : e - nq, h = f / hc, c = (f - h * hc) * V;
      if (!isq && d < 0) continue;
      const T* src = (isq ? static_cast<const T*>(a.q) + t * a.q_stride : static_cast<const T*>(a.k) + t * a.k_stride) + h * a.hd + c;
      T* to = (isq ? static_cast<T*>(a.q_out) + t * a.q_out_stride : pool + d) + h * a.hd + c;
      float x0[V], x1[V], y0[V], y1[V];
      unpack16(*reinterpret_cast<const uint4*>(src), x0, T());
      unpack16(*reinterpret_cast<const uint4*>(src + half), x1, T());
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float2 w = cs[r][c + j];
        y0[j] = fmaf(x0[j], w.x, -(x1[j] * w.y));
        y1[j] = fmaf(x1[j], w.x, x0[j] * w.y);
      }
      store16(to, pack16(y0, T()));
      store16(to + half, pack16(y1, T()));
    } else if (d >= 0) {
      const int f = e - nrot;
      const bool isk = f < nk;
      const int c = (isk ? f : f - nk) * V;
      const T* src = isk ? static_cast<const T*>(a.k) + t * a.k_stride + c : static_cast<const T*>(a.v) + t * a.v_stride + c;
      store16(pool + d + (isk ? 0 : a.at.kvd) + c, *reinterpret_cast<const uint4*>(src));
    }
  }
}

// ---------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------
struct Span {     // what a workgroup works on
  int lo;         // first row of the sequence, in the packed batch
  int rows;       // its packed rows (new rows * G)
  int len;        // cached rows that can be read
  int first;      // keys that new row 0 sees under the mask: row r sees first + r (below len)
  const int32_t* table;
};

__device__ __forceinline__ Span span_of(const PagedAttention& a, int b) {
  Span s;
  s.lo = a.cu != nullptr ? a.cu[b] : 0;
  const int n = a.cu != nullptr ? a.cu[b + 1] - s.lo : a.T;
  const int len = a.kv_len != nullptr ? max(a.kv_len[b], 0) : a.max_len;
  s.rows = n * a.G;
  s.len = static_cast<int>(min(static_cast<int64_t>(min(len, a.max_len)),
                               static_cast<int64_t>(a.at.max_pages) << a.at.shift));
  s.first = len - n + 1;
  s.table = a.at.table + (a.cu != nullptr ? b * a.at.table_stride : 0);
  return s;
}

// the maximum and the sum over the lanes l % 16 (half_swap_max goes on from
// rows of 16 lanes swapped in pairs)
__device__ __forceinline__ float quarter_swap_max(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return half_swap_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float quarter_swap_sum(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return half_swap_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// A launch's work: the common prefix's and the sequences' own, if both are of
// one kind. The prefix's workgroups, which have more to do, come first.
struct PagedJobs {
  PagedAttention job[2];
  uint32_t first, blocks;  // workgroups of the first, and of both
};

// The parts of a row: (maximum, sum) in ml and the sums of values in o, one of
// each split. A sum of kDone in the first says that the row is finished.
constexpr float kDone = -1.0f;

// the parts that another launch of the call has and this one has not
__device__ __forceinline__ void empty_parts(const PagedAttention& a, int64_t at) {
  for (int p = a.splits; p < a.parts; ++p) a.ml[at + static_cast<int64_t>(p) * a.T * a.H] = make_float2(-INFINITY, 0.f);
}

// lds_load16 of rows that no other workgroup reads, too many to stay in the
// last-level cache: they do not displace what is there. One row of 64 sequences
// of up to 4096, 32 heads of 128 on 8, 102.9 us (5.4 TB/s), with lds_load16
// 117.9. Where other workgroups read them too it loses (63 rows over 4000 common
// ones, 32 heads of 64, 36.2 / 31.1), and where the next call finds them in the
// cache (52 MB of fp32 rows 20.5 / 19.3).
__device__ __forceinline__ void lds_load16_once(uint32_t lds, uint32_t off, const u32x4& res) {
  asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"{m0}"(lds), "v"(off), "s"(res) : "memory");
}

// the page ids and lengths, read as scalars: loads that would wait in line
// with a wave's tile loads otherwise
typedef const __attribute__((address_space(4))) int32_t* scalar_ids;
__device__ __forceinline__ scalar_ids scalar(const int32_t* p) {
  return reinterpret_cast<scalar_ids>(reinterpret_cast<uintptr_t>(p));
}

// The values, but 2^120 in the place of larger ones, infinities and NaN (-2^120
// of those below zero): as signed integers their bits are above the positive
// numbers', as unsigned ones above the negative numbers'.
__device__ __forceinline__ bf16x8_t bounded(bf16x8_t v) {
  typedef int16_t i16x8 __attribute__((ext_vector_type(8)));
  typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
  const i16x8 x = __builtin_elementwise_min(__builtin_bit_cast(i16x8, v), i16x8(int16_t{0x7b80}));
  return __builtin_bit_cast(bf16x8_t, __builtin_elementwise_min(__builtin_bit_cast(u16x8, x), u16x8(uint16_t{0xfb80})));
}

// Workgroups of the few-row kernels: the (key/value head, sequence) pairs
// vary fastest, then the blocks of rows, then the splits. Workgroup L runs on
// XCD L % 8: with the splits fastest and 2, 4 or 8 of them a ragged batch's
// last splits, mostly empty, were all on the same XCDs.

// bf16, heads of 32, 64 and 128, 16 packed rows at a time: bound by the
// cached rows' bytes. A workgroup takes 16 packed rows of one (sequence,
// key/value head) and a split of its keys; its four waves take 32-key tiles in
// turn, each through its own K and V buffer in LDS, without barriers: the next
// tile's K is under way as soon as S^T = K Q^T has read the last one, its V
// after O^T += V^T P^T has. A load instruction covers whole rows of a head (4
// of 128, 8 of 64, 16 of 32) of one page, through a buffer resource that ends with the
// sequence, so what lies behind its last row reads as zeros, and so does a
// page outside the pool. The transposed products leave a lane eight scores of
// one row, keys 4 (l / 16) + r and those + 16, which are its operand of the
// second product; V is read in that same order of keys. P meets V as two bf16
// numbers whose sum has 16 bits: the matrix cores have the time. The second,
// which is zero or below it as often as not, meets bounded values: an infinite
// one is the first's to pass on (the second is up to 1 in size, and 32 of 2^120
// stay a number). 32 packed rows
// at a time (the 32-wide products) took as long where the bytes bound it and
// longer elsewhere (8 of 128 on 1, 16 of up to 10000 rows 20.4, 16 at a time 19.6).
// One row of 64 sequences of up to 4096, 32 heads of 128 on 8: 99 us and 5 for
// the join, 5.4 TB/s in all; of 4 of up to 65536 157, 6.1 TB/s.
template <int HD, int NW>
struct FewShared {  // LDS of a group of NW waves
  static constexpr int HP = 17;  // merge row stride: [channel][row]
  static constexpr int TILES = NW * 64 * HD * 2, MERGE = NW * HD * HP * 4;
  unsigned char tiles[MERGE > TILES ? MERGE : TILES];
  float m[NW][16], l[NW][16];
};

// the work of group `block` of NW waves (if there is one), as its thread `tid`; all threads of the workgroup call it
template <int HD, int NW, bool HEAD>
__device__ __forceinline__ void few_rows(const PagedAttention& a, int block, bool there, int tid, FewShared<HD, NW>& shared) {
  constexpr int KK = HD / 32, CT = HD / 16, CPR = HD / 8;
  constexpr int RB = HD * 2, HALF = 32 * RB;    // a tile of 32 rows of K, or V
  constexpr int RPL = 1024 / RB, NL = 16 / RPL;  // rows a load, loads per 16 rows
  constexpr int HP = FewShared<HD, NW>::HP;
  unsigned char* smem = shared.tiles;
  auto& sm = shared.m;
  auto& sl = shared.l;
  const int Hkv = a.H / a.G, pair = block % (Hkv * a.B), st = block / (Hkv * a.B);
  const int g = pair % Hkv, b = pair / Hkv, tile = st % a.tiles, split = st / a.tiles;
  const Span sp = span_of(a, b);
  const int i0 = tile * kPagedFewRows;
  const bool live = there && i0 < sp.rows && sp.rows <= a.few_rows;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int quarter = lane >> 4, l16 = lane & 15;
  const int row = min(i0 + l16, sp.rows - 1);  // rows past the sequence are not stored
  // A common prefix in the same job (HEAD) comes first, filled up to whole steps: key
  // j below `head` is its row j, key j from there on row j - head of the
  // sequence's own
  const int head = HEAD ? (a.head_len + 31) & ~31 : 0, end = head + sp.len;
  auto seen = [&](int i) { return head + (a.causal ? max(min(sp.first + i / a.G, sp.len), 0) : sp.len); };
  const int lim = seen(row), lim0 = seen(i0);  // a lane's keys are those below lim; the tile's first row's
  const int last = seen(min(i0 + 15, sp.rows - 1));
  const int k0 = split * a.chunk, kend = live ? min(last, k0 + a.chunk) : 0;
  const float scale_log2 = a.scale * kLog2e;

  // K row r of a tile keeps its 16-byte chunk c at c ^ ksw(r), V row r at c ^ vsw(r) (k_attn.hip)
  auto ksw = [](int r) { return HD == 32 ? (r >> 2) & 3 : HD == 64 ? (r >> 1) & 7 : r & 15; };
  auto vsw = [](int r) { return HD == 32 ? 0 : HD == 64 ? ((r >> 1) & 1) << 2 : (r & 3) << 2; };
  const uint32_t rowb = static_cast<uint32_t>(a.at.kvd) * 4u;
  uint32_t koff[NL], voff[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int r = i * RPL + lane / CPR;
    koff[i] = r * rowb + (((lane % CPR) ^ ksw(r)) << 4);
    voff[i] = r * rowb + (((lane % CPR) ^ vsw(r)) << 4);
  }
  unsigned char* mine = smem + wave * (2 * HALF);
  const uint32_t lds0 = lds_address(smem) + wave * (2 * HALF);
  const scalar_ids table = scalar(sp.table), head_table = scalar(a.head_table);
  const char* pool = static_cast<const char*>(a.at.pool);
  // 16 rows from row j on, of page `page` (-1 where the sequence has ended): `col` bytes into a row
  auto resource = [&](int j, int page, uint32_t col) {
    const bool there = page >= 0 && page < a.at.n_pages;
    const uint32_t bytes = there ? static_cast<uint32_t>(min((HEAD && j < head ? a.head_len : end) - j, 16)) * rowb - col : 0u;
    u32x4 res = buffer_resource(pool + (there ? page : 0) * (a.at.page_stride * 2) +
                                    static_cast<uint32_t>((HEAD && j >= head ? j - head : j) & ((1 << a.at.shift) - 1)) * rowb + col,
                                bytes);
    // a load in asm may follow a vector instruction's write of its scalar operands by five states at least
    asm volatile("s_nop 4" : "+s"(res));
    return res;
  };
  // (the read does not wait for the length: up to the table's end it goes through)
  auto page_of = [&](int j) {
    const bool first = HEAD && j < head;
    const int p = (first ? j : j - head) >> a.at.shift, most = first ? (a.head_len - 1) >> a.at.shift : a.at.max_pages - 1;
    const int page = most >= 0 ? (first ? head_table : table)[min(p, most)] : -1;
    return j < (first ? a.head_len : end) ? page : -1;
  };
  const bool once = !HEAD && a.once && a.tiles == 1;  // this workgroup alone reads the rows
  const uint32_t kcol = g * RB, vcol = rowb / 2 + g * RB;
  auto load = [&](int j0, int pg0, int pg1, uint32_t lds, uint32_t col, const uint32_t (&off)[NL]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const u32x4 res = resource(j0 + 16 * h, h == 0 ? pg0 : pg1, col);
      if (once) {
#pragma unroll
        for (int i = 0; i < NL; ++i) lds_load16_once(lds + (h * NL + i) * 1024, off[i], res);
      } else {
#pragma unroll
        for (int i = 0; i < NL; ++i) lds_load16(lds + (h * NL + i) * 1024, off[i], res);
      }
    }
  };

  float m_run = -INFINITY, l_run = 0.f;  // of the raw scores; l_run: this lane's keys only
  const f32x4_t zero = {};
  f32x4_t o[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) o[ct] = zero;
  // fragment addresses: a transposing read gives group `quarter` of 16 lanes
  // the keys 4 quarter .. + 3 of 16 channels, one a lane
  const uint32_t vrow = 4 * quarter + (l16 >> 2);
  uint32_t kaddr[KK], vaddr[CT];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) kaddr[kk] = l16 * RB + (((4 * kk + quarter) ^ ksw(l16)) << 4);
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
    vaddr[ct] = HALF + vrow * RB + (lane & 1) * 8 + (((2 * ct + ((lane >> 1) & 1)) ^ vsw(vrow)) << 4);

  int j0 = k0 + wave * 32;
  int pg0 = page_of(j0), pg1 = page_of(j0 + 16);
  if (j0 < kend) {
    load(j0, pg0, pg1, lds0, kcol, koff);
    load(j0, pg0, pg1, lds0 + HALF, vcol, voff);
  }
  int nx0 = page_of(j0 + 32 * NW), nx1 = page_of(j0 + 32 * NW + 16);  // read a step before the loads that need them
  asm volatile("" : "+s"(nx0), "+s"(nx1));
  bf16x8_t qf[KK];
  if (j0 < kend) {
    const bf16_t* qp = static_cast<const bf16_t*>(a.q) + static_cast<int64_t>(sp.lo + row / a.G) * a.q_stride +
                       (g * a.G + row % a.G) * HD;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
      qf[kk] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4*>(qp + kk * 32 + quarter * 8));
    // here before the loop, which would otherwise wait for every load in it
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) asm volatile("" : "+v"(qf[kk]));
  }
  for (; j0 < kend; j0 += 32 * NW) {
    const int jn = j0 + 32 * NW;
    const bool more = jn < kend;
    pg0 = nx0;
    pg1 = nx1;
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NL) : "memory");  // K is here, V may be under way
    __builtin_amdgcn_sched_barrier(0);
    f32x4_t s[2];
    bf16x8_t kf[KK][2];  // all read before the products: one latency, not one a product
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        kf[kk][t] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4*>(mine + kaddr[kk] + 16 * t * RB));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kk][t], qf[kk], kk == 0 ? zero : s[t], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) load(jn, pg0, pg1, lds0, kcol, koff);
    nx0 = page_of(jn + 32 * NW);
    nx1 = page_of(jn + 32 * NW + 16);
    // s[t][r]: key j0 + 16 t + 4 quarter + r, packed row `row`
    if (j0 + 32 > (HEAD && j0 < head ? a.head_len : lim0)) {
      const int left = (HEAD && j0 < head ? a.head_len : lim) - j0;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (16 * t + 4 * quarter + r >= left) s[t][r] = -INFINITY;
    }
    const float mloc = quarter_swap_max(fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                                              fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3]))));
    // the reference maximum moves only when it has to (k_attn.hip)
    const float m_new = fmaxf(m_run, mloc);
    if (__builtin_amdgcn_ballot_w64(m_new == -INFINITY ? false : !((m_new - m_run) * scale_log2 <= 8.0f)) != 0) {
      const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m_run - m_new) * scale_log2);
      l_run *= alpha;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[ct][r] *= alpha;
      m_run = m_new;
    }
    // (the difference first: where a scaled score is rounded by many units of an
    // exponential, a product's rounding would be left in it)
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
    u32x4 hi, lo;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        const float p0 = __builtin_amdgcn_exp2f((s[t][r] - m_use) * scale_log2);
        const float p1 = __builtin_amdgcn_exp2f((s[t][r + 1] - m_use) * scale_log2);
        l_run += p0 + p1;
        s[t][r] = p0;
        s[t][r + 1] = p1;
        const uint32_t w = pack_bf16x2(p0, p1);
        hi[2 * t + (r >> 1)] = w;
        lo[2 * t + (r >> 1)] = pack_bf16x2(p0 - __uint_as_float(w << 16), p1 - __uint_as_float(w & 0xffff0000u));
      }
    if (more)
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NL) : "memory");  // V is here, the next K may be under way
    else
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    asm volatile("" : "+s"(nx0), "+s"(nx1));  // here: scalar loads under way make every wait for LDS one for all
    __builtin_amdgcn_sched_barrier(0);
    // A value that is not finite must not reach a row that does not see its
    // key, through the product with its zero probability: where the tile holds
    // hidden keys and such values, it goes through the vector ALU, key by key.
    bool odd = false;
    if ((!HEAD || j0 >= head) && lim0 < min(j0 + 32, end)) {
#pragma unroll
      for (int i = 0; i < 2 * NL; ++i) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(mine + HALF + i * 1024 + lane * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          odd |= (w[e] & 0x7f80u) == 0x7f80u || (w[e] & 0x7f800000u) == 0x7f800000u;
      }
      odd = __builtin_amdgcn_ballot_w64(odd) != 0;
    }
    if (!odd) {
      bf16x8_t vf[CT];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
        vf[ct] = __builtin_bit_cast(bf16x8_t, lds_read_columns(mine + vaddr[ct], mine + vaddr[ct] + 16 * RB));
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
        o[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[ct], __builtin_bit_cast(bf16x8_t, hi), o[ct], 0, 0, 0);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
        o[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bounded(vf[ct]), __builtin_bit_cast(bf16x8_t, lo), o[ct], 0, 0, 0);
    } else {
#pragma unroll
      for (int kk = 0; kk < 32; ++kk) {
        // key j0 + kk: register kk % 4 of tile kk / 16, lane quarter (kk / 4) % 4
        const float p = __shfl(s[kk >> 4][kk & 3], l16 + 16 * ((kk >> 2) & 3), 64);
        if (j0 + kk < lim) {
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            const int c = ct * 16 + 4 * quarter;
            const uint2 w = *reinterpret_cast<const uint2*>(mine + HALF + kk * RB + (((c >> 3) ^ vsw(kk)) << 4) + (c & 7) * 2);
            o[ct][0] = fmaf(p, __uint_as_float(w.x << 16), o[ct][0]);
            o[ct][1] = fmaf(p, __uint_as_float(w.x & 0xffff0000u), o[ct][1]);
            o[ct][2] = fmaf(p, __uint_as_float(w.y << 16), o[ct][2]);
            o[ct][3] = fmaf(p, __uint_as_float(w.y & 0xffff0000u), o[ct][3]);
          }
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) load(jn, pg0, pg1, lds0 + HALF, vcol, voff);
  }
  l_run = quarter_swap_sum(l_run);
  __syncthreads();  // every wave is past its tiles
  float* so = reinterpret_cast<float*>(smem);
  if (quarter == 0) {
    sm[wave][l16] = m_run == -INFINITY ? -INFINITY : m_run * scale_log2;
    sl[wave][l16] = l_run;
  }
  const int nr = live ? min(kPagedFewRows, sp.rows - i0) : 0;
  if (l16 < nr) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int r = 0; r < 4; ++r) so[(wave * HD + ct * 16 + 4 * quarter + r) * HP + l16] = o[ct][r];
  }
  __syncthreads();
  for (int it = tid; it < nr * (HD / 4); it += 64 * NW) {
    const int q = it / (HD / 4), c0 = (it % (HD / 4)) * 4, i = i0 + q;
    float m = sm[0][q];
#pragma unroll
    for (int w = 1; w < NW; ++w) m = fmaxf(m, sm[w][q]);
    float l = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      // a wave without keys for this row holds the empty sum
      if (sm[w][q] == -INFINITY && sl[w][q] == 0.f) continue;
      const float f = __builtin_amdgcn_exp2f(sm[w][q] - (m == -INFINITY ? 0.f : m));
      l = fmaf(f, sl[w][q], l);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = fmaf(f, so[(w * HD + c0 + e) * HP + q], v[e]);
    }
    const int t = sp.lo + i / a.G, h = g * a.G + i % a.G;
    const int64_t row0 = static_cast<int64_t>(t) * a.H + h;
    if (a.direct) {
      const float inv = l == 0.f ? 0.f : 1.0f / l;
      *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.out) + t * a.out_stride + h * HD + c0) =
          make_uint2(pack_bf16x2(v[0] * inv, v[1] * inv), pack_bf16x2(v[2] * inv, v[3] * inv));
      if (c0 == 0 && a.lse != nullptr)
        a.lse[static_cast<int64_t>(h) * a.T + t] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
      if (c0 == 0 && a.ml != nullptr) a.ml[row0] = make_float2(0.f, kDone);
    } else {
      const int64_t at = static_cast<int64_t>(split) * a.T * a.H + row0;
      if (c0 == 0) {
        a.ml[at] = make_float2(m, l);
        if (split == 0) empty_parts(a, at);
      }
      if (l != 0.f) *reinterpret_cast<float4*>(a.o + at * HD + c0) = make_float4(v[0], v[1], v[2], v[3]);
    }
  }
}

template <int HD, int NW, bool HEAD>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(HD <= 64 && NW == 4 ? 3 : 2))) void paged_few_kernel(
    PagedJobs jobs) {
  __shared__ __align__(1024) FewShared<HD, NW> shared;
  const int which = blockIdx.x >= jobs.first;
  const PagedAttention a = jobs.job[which];  // (a copy: what it holds stays in registers)
  few_rows<HD, NW, HEAD>(a, blockIdx.x - (which ? jobs.first : 0), true, threadIdx.x, shared);
}

// bf16, heads of 32, 64 and 128, many packed rows: bound by the products. A
// workgroup takes 32 QB NW packed rows of one (sequence, key/value head) and a
// split of its keys; all waves share the K and V tiles of 64 keys, three of
// them in LDS, loaded two ahead straight from the pages. A wave owns 32 QB rows
// and issues the products S(u + 1) = K Q^T and O += V P(u - 1) one at a time
// between the exponentials of step u, relative to a reference maximum that
// moves only when it must: the order of the work, the tile layout and the
// reasons are those of attn_wide_kernel (k_attn.hip). What differs is where a
// tile's rows come from and which keys a row sees.
//  * A load instruction covers rows of one page (4 of 128, 8 of 64, 16 of 32 columns);
//    its page id is in a register of all lanes that holds the next 64 ids of
//    the table, read 64 at a time: a scalar load would make every wait for LDS
//    a wait for all of it, a vector load one for the tiles under way.
//  * The resource ends with the sequence, so rows behind it read as zeros.
//  * The packed rows put the G query heads that share a key/value head into
//    one workgroup: its tiles are read once for all of them.
//  * A common prefix that the launch puts before the rows (HEAD) is filled up
//    to 32 keys, masked in the one step that holds them.
//  * P is rounded to bf16 for the second product, as there: half a step of
//    each probability, which the sums of many average out.
// 4 x 1024 new rows over up to 8024, 32 heads of 128 on 8, 361 us, 1.06 PFLOP/s
// (the few-row kernel 751); 4 x 1024 over 8192, 32 of 64, 303 us, 0.91.
template <int HD, int QB, int NW>
struct ManyShared {
  static constexpr int WQ = 32 * QB, BUF = 2 * 64 * HD * 2, NB = 3, OLD = HD + 8;
  unsigned char tiles[NB * BUF > NW * WQ * OLD * 2 ? NB * BUF : NW * WQ * OLD * 2];
};

template <int HD, int QB, int NW, bool HEAD>
__device__ __forceinline__ void many_rows(const PagedAttention& a, int block, ManyShared<HD, QB, NW>& shared) {
  constexpr int WQ = 32 * QB, BQ = WQ * NW, BK = 64;
  constexpr int KK = HD / 16, CT = HD / 32, CPR = HD / 8;
  constexpr int RB = HD * 2, HALF = BK * RB, BUF = 2 * HALF, OLD = HD + 8;
  constexpr int RPL = 1024 / RB, LPW = HALF / 1024 / NW;  // rows per load, loads per wave and operand
  static_assert(LPW * NW * 1024 == HALF && NW * RPL % 16 == 0 && BQ == kPagedManyRows, "tile split");
  unsigned char* smem = shared.tiles;

  // the row blocks of a pair (key/value head, sequence, split of the keys) run
  // on one XCD one after another, the last ones, which see most keys, first
  const int Hkv = a.H / a.G, pair = (block >> 3) / a.tiles * 8 + (block & 7);
  if (pair >= a.splits * Hkv * a.B) return;
  const int tile = a.tiles - 1 - (block >> 3) % a.tiles;
  const int split = pair / (Hkv * a.B), g = pair % Hkv, b = pair / Hkv % a.B;
  const Span sp = span_of(a, b);
  const int i0 = tile * BQ;
  if (i0 >= sp.rows || sp.rows <= a.few_rows) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const int wq0 = i0 + wave * WQ;  // the wave's first packed row
  const float scale_log2 = a.scale * kLog2e;
  // A common prefix in the same job (HEAD) comes first, as in few_rows
  const int head = HEAD ? (a.head_len + 31) & ~31 : 0, end = head + sp.len;
  // keys that packed row i sees
  auto seen = [&](int i) {
    const int n = a.causal ? min(sp.first + min(i, sp.rows - 1) / a.G, sp.len) : sp.len;
    return HEAD ? head + max(n, 0) : n;
  };
  const int k0 = split * a.chunk;
  const int kend = min(seen(i0 + BQ - 1), k0 + a.chunk);
  const int nt = max((kend - k0 + BK - 1) / BK, 0);
  // the wave's own tiles: none past its last row's last key
  const int wlast = min(seen(wq0 + WQ - 1), kend), wlim0 = seen(wq0);
  const int ntw = min(nt, (wlast - k0 + BK - 1) / BK);
  const bool busy = wq0 < sp.rows && wlast > k0;  // a wave without rows or keys only loads tiles

  const uint32_t rowb = static_cast<uint32_t>(a.at.kvd) * 4u;
  auto ksw = [](int r) { return HD == 32 ? (r >> 2) & 3 : HD == 64 ? (r >> 1) & 7 : r & 15; };
  auto vsw = [](int r) { return HD == 32 ? 0 : HD == 64 ? ((r >> 1) & 1) << 2 : (r & 3) << 2; };
  const int lrow = wave * RPL + lane / CPR;  // tile row of the wave's first load; the later ones are 16 n rows on
  const uint32_t koff = (lane / CPR) * rowb + (((lane % CPR) ^ ksw(lrow)) << 4);
  const uint32_t voff = (lane / CPR) * rowb + (((lane % CPR) ^ vsw(lrow)) << 4);
  const uint32_t lds0 = lds_address(smem) + wave * 1024;
  const char* pool = static_cast<const char*>(a.at.pool);
  // ids of the 64 pages from `idp` on, one a lane, and of the 64 after them
  // (the reads do not wait for the length: up to the table's end they go through)
  // (with a prefix its pages' ids and then the sequence's, as one list)
  const int most = a.at.max_pages - 1, hpages = HEAD ? (head + (1 << a.at.shift) - 1) >> a.at.shift : 0;
  auto place = [&](int j) { return HEAD && j >= head ? hpages + ((j - head) >> a.at.shift) : j >> a.at.shift; };
  int idp = place(k0);
  auto read_ids = [&](int from) {
    const int p = from + lane;
    if (HEAD && p < hpages) return a.head_table[min(p, (a.head_len - 1) >> a.at.shift)];
    return most >= 0 ? sp.table[min(p - hpages, most)] : -1;
  };
  int ids = read_ids(idp), idn = read_ids(idp + 64);
  auto load_rows = [&](int j, uint32_t lds) {  // K and V of RPL rows from row j on
    const int p = place(j), left = (HEAD && j < head ? a.head_len : end) - j;
    if (p >= idp + 64) {
      asm volatile("" : "+v"(idn));  // waited for here
      ids = idn;
      idp += 64;
      idn = read_ids(idp + 64);
    }
    const int page = __builtin_amdgcn_readlane(ids, p - idp);
    const bool there = left > 0 && page >= 0 && page < a.at.n_pages;
    const uint32_t bytes = there ? static_cast<uint32_t>(min(left, RPL)) * rowb - g * RB : 0u;
    const char* at = pool + (there ? page : 0) * (a.at.page_stride * 2) +
                     static_cast<uint32_t>((HEAD && j >= head ? j - head : j) & ((1 << a.at.shift) - 1)) * rowb + g * RB;
    u32x4 kres = buffer_resource(at, bytes), vres = buffer_resource(at + rowb / 2, there ? bytes - rowb / 2 : 0u);
    // a load in asm may follow a vector instruction's write of its scalar operands by five states at least
    asm volatile("s_nop 4" : "+s"(kres), "+s"(vres));
    lds_load16(lds, koff, kres);
    lds_load16(lds + HALF, voff, vres);
  };
  auto load_tile = [&](int t, int buf) {
#pragma unroll
    for (int i = 0; i < LPW; ++i)
      load_rows(k0 + t * BK + i * (NW * RPL) + wave * RPL, lds0 + buf * BUF + i * (NW * 1024));
  };

  float mu[QB], l_run[QB];  // reference max (scaled, exp2 units); sum over this lane's keys
  f32x16_t o[QB][CT], sa[QB], sb[QB];
  bf16x8_t pf[QB][2];  // P of the last step: [row block][16 keys]
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    l_run[qb] = 0.f;
    mu[qb] = kNoReference;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[qb][ct][r] = 0.f;
  }
  int lim[QB];
  const bf16_t* qrow[QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    // rows past the sequence are clamped, not zeroed: their outputs are not stored
    const int i = min(wq0 + 32 * qb + l32, sp.rows - 1);
    lim[qb] = seen(i);
    qrow[qb] = static_cast<const bf16_t*>(a.q) + static_cast<int64_t>(sp.lo + i / a.G) * a.q_stride +
               (g * a.G + i % a.G) * HD + half * 8;
  }
  bf16x8_t qf[QB][KK];
  const f32x16_t zero = {};

  if (nt > 0) {
    load_tile(0, 0);
    if (nt > 1) load_tile(1, 1);
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
        qf[qb][kk] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4*>(qrow[qb] + kk * 16));

    // fragment addresses within a tile: K rows l32 (+ 32), chunk 2 kk + half;
    // V key rows 4 half + r (+ 8, 16 ..), the channel runs of a transposing read
    const uint32_t kf0 = l32 * RB, vrow = 4 * half + ((lane & 15) >> 2);
    const int ks0 = ksw(l32), vs0 = vsw(vrow);
    const uint32_t vf0 = HALF + vrow * RB + (lane & 1) * 8;
    const int vch = 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
    uint32_t kaddr[KK], vaddr[CT];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) kaddr[kk] = kf0 + (((2 * kk + half) ^ ks0) << 4);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) vaddr[ct] = vf0 + (((4 * ct + vch) ^ vs0) << 4);
    auto read_k = [&](const unsigned char* base, int kk) {
      return __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4*>(base + kaddr[kk]));
    };
    auto read_v = [&](const unsigned char* base, int k, int ct) {
      const unsigned char* vr = base + vaddr[ct] + k * (16 * RB);
      return __builtin_bit_cast(bf16x8_t, lds_read_columns(vr, vr + 8 * RB));
    };
    auto row_max = [&](const f32x16_t& s) {
      float mx = fmaxf(fmaxf(s[0], s[1]), s[2]);
#pragma unroll
      for (int r = 3; r < 15; r += 2) mx = fmaxf(fmaxf(mx, s[r]), s[r + 1]);
      return half_swap_max(fmaxf(mx, s[15]));
    };
    auto mask = [&](int u, f32x16_t (&s)[QB]) {
      const int j0 = k0 + 32 * u;
      const bool fill = HEAD && j0 < head && j0 + 32 > a.head_len;
      if (j0 + 32 <= wlim0 && !fill) return;
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        int left = (fill ? a.head_len : lim[qb]) - j0 - 4 * half;  // keys from this lane's limit on are masked
        asm("" : "+v"(left));  // the comparisons stay here (hoisted, their masks fill the scalar registers)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (8 * (r >> 2) + (r & 3) >= left) s[qb][r] = -INFINITY;
      }
    };
    // one step: the exponentials of step u (scores s) beside the products of
    // O += V P(u - 1) and S(u + 1) = sn (the first step: alone)
    auto step = [&](int u, int bufn, int ksn, int bufp, int ksp, f32x16_t (&s)[QB], f32x16_t (&sn)[QB], auto first_c) {
      constexpr bool first = decltype(first_c)::value;
      if (!first) mask(u, s);
      constexpr int FA = 2;                                   // fragments in flight ahead of their use
      constexpr int NF = KK + 2 * CT, NS = QB * NF;           // operand fragments, matrix instructions
      constexpr int NU = 16 * QB;                             // pieces of vector work
      const unsigned char* kp = smem + bufn * BUF + ksn * (32 * RB);
      const unsigned char* vp = smem + bufp * BUF + ksp * (32 * RB);
      bf16x8_t fr[FA + 1];
      auto read = [&](int f) { fr[f % (FA + 1)] = f < KK ? read_k(kp, f) : read_v(vp, (f - KK) / CT, (f - KK) % CT); };
      auto product = [&](int i) {
        const int f = i / QB, qb = i % QB;
        if (f < KK)
          sn[qb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[f % (FA + 1)], qf[qb][f], f == 0 ? zero : sn[qb], 0, 0, 0);
        else
          o[qb][(f - KK) % CT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              fr[f % (FA + 1)], pf[qb][(f - KK) / CT], o[qb][(f - KK) % CT], 0, 0, 0);
      };
      float rsum[QB], a0 = 0.f, a1 = 0.f, p0 = 0.f, p1 = 0.f;
      u32x4 pn[QB][2];
      auto work = [&](int w) {
        const int qb = w >> 4, r = w & 14;
        if ((w & 1) == 0) {
          p0 = __builtin_amdgcn_exp2f(fmaf(s[qb][r], scale_log2, -mu[qb]));
          p1 = __builtin_amdgcn_exp2f(fmaf(s[qb][r + 1], scale_log2, -mu[qb]));
          asm volatile("" : "+v"(p0), "+v"(p1));  // computed here, beside this step's products
        } else {
          uint32_t pw = pack_bf16x2(p0, p1);
          a0 = r == 0 ? p0 : a0 + p0;
          a1 = r == 0 ? p1 : a1 + p1;
          asm volatile("" : "+v"(pw), "+v"(a0), "+v"(a1));
          pn[qb][r >> 3][(r >> 1) & 3] = pw;
          if (r == 14) rsum[qb] = a0 + a1;
        }
      };
      if constexpr (first) {
#pragma unroll
        for (int k = 0; k < NU; ++k) work(k);
      } else {
#pragma unroll
        for (int f = 0; f < FA; ++f) read(f);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          if (i % QB == 0 && i / QB + FA < NF) read(i / QB + FA);
          product(i);
#pragma unroll
          for (int k = NU * i / NS; k < NU * (i + 1) / NS; ++k) work(k);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      bool high = false;
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) high |= !(rsum[qb] <= 4096.f);
      if (!first && __builtin_amdgcn_ballot_w64(high) != 0) {
        // a score far above the reference, or the first key that a row sees:
        // move it, and redo this step's P
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          const float m_new = fmaxf(mu[qb], row_max(s[qb]) * scale_log2);
          const float alpha = __builtin_amdgcn_exp2f(mu[qb] - m_new);
          mu[qb] = m_new;
          l_run[qb] *= alpha;
#pragma unroll
          for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[qb][ct][r] *= alpha;
          rsum[qb] = 0.f;
#pragma unroll
          for (int r = 0; r < 16; r += 2) {
            const float e0 = __builtin_amdgcn_exp2f(fmaf(s[qb][r], scale_log2, -m_new));
            const float e1 = __builtin_amdgcn_exp2f(fmaf(s[qb][r + 1], scale_log2, -m_new));
            rsum[qb] += e0 + e1;
            pn[qb][r >> 3][(r >> 1) & 3] = pack_bf16x2(e0, e1);
          }
        }
      }
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        l_run[qb] += rsum[qb];
        pf[qb][0] = __builtin_bit_cast(bf16x8_t, pn[qb][0]);
        pf[qb][1] = __builtin_bit_cast(bf16x8_t, pn[qb][1]);
      }
    };

    int bp = 2, bc = 0, bn = 1;  // buffers of tiles t - 1, t, t + 1
    auto turn = [&]() {
      const int f = bp;
      bp = bc;
      bc = bn;
      bn = f;
    };
    turn_over();
    if (busy) {
      // the first tile's scores, and the reference: the max over its 64 keys
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        const bf16x8_t a0 = read_k(smem, kk), a1 = read_k(smem + 32 * RB, kk);
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          sa[qb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a0, qf[qb][kk], kk == 0 ? zero : sa[qb], 0, 0, 0);
          sb[qb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a1, qf[qb][kk], kk == 0 ? zero : sb[qb], 0, 0, 0);
        }
      }
      mask(0, sa);
      mask(1, sb);
#pragma unroll
      for (int qb = 0; qb < QB; ++qb)
        mu[qb] = fmaxf(fmaxf(row_max(sa[qb]), row_max(sb[qb])) * scale_log2, kNoReference);
      step(0, bc, 1, bp, 1, sa, sb, std::true_type());
    }
    if (nt > 2) load_tile(2, bp);
    if (busy) step(1, bn, 0, bc, 0, sb, sa, std::false_type());
    int t = 1;
    for (; t < (busy ? ntw : 0); ++t) {
      turn();
      step(2 * t, bc, 1, bp, 1, sa, sb, std::false_type());
      turn_over();
      if (t + 2 < nt) load_tile(t + 2, bp);
      step(2 * t + 1, bn, 0, bc, 0, sb, sa, std::false_type());
    }
    if (busy) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          const bf16x8_t v = read_v(smem + bc * BUF + 32 * RB, k, ct);
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
            o[qb][ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pf[qb][k], o[qb][ct], 0, 0, 0);
        }
    }
    for (; t < nt; ++t) {  // the tiles of the block's later rows
      turn();
      turn_over();
      if (t + 2 < nt) load_tile(t + 2, bp);
    }
    turn_over();  // every wave is past the tiles before the output staging reuses them
  }

#pragma unroll
  for (int qb = 0; qb < QB; ++qb) l_run[qb] = half_swap_sum(l_run[qb]);
  // A value that is not finite must not reach a row that does not see its key;
  // through the product with its zero probability it has, and left a NaN. And a
  // reference of 2^27 and more is rounded by 8 and more, which is left in the
  // exponents of a row, from 128 on as zeros and infinities. Where the wave's
  // tiles hold hidden keys and its results a NaN, or its references are that far,
  // its rows are computed again: the scores' difference to the maximum before
  // its scale, the second product on the vector ALU, key by key.
  if (busy) {
    bool odd = false;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) odd |= fabsf(mu[qb]) >= 0x1p27f && mu[qb] != kNoReference;
    if (wlim0 < min(end, k0 + ntw * BK)) {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int r = 0; r < 16; ++r) odd |= o[qb][ct][r] != o[qb][ct][r];
    }
    if (__builtin_amdgcn_ballot_w64(odd) != 0) {
      auto row_of = [&](int j) {  // row j's keys, or null
        const bool first = HEAD && j < head;
        const int i = first ? j : j - head;
        const int page = i < (first ? a.head_len : sp.len) ? (first ? a.head_table : sp.table)[i >> a.at.shift] : -1;
        return page < 0 || page >= a.at.n_pages
                   ? nullptr
                   : pool + page * (a.at.page_stride * 2) + static_cast<uint32_t>(i & ((1 << a.at.shift) - 1)) * rowb + g * RB;
      };
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        float m = kNoReference, l = 0.f;  // of the raw scores
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[qb][ct][r] = 0.f;
        for (int j0 = k0; j0 < wlast; j0 += 32) {
          const char* kr = row_of(j0 + l32);
          f32x16_t s = zero;
#pragma unroll
          for (int kk = 0; kk < KK; ++kk) {
            u32x4 k = {0u, 0u, 0u, 0u};
            if (kr != nullptr) k = *reinterpret_cast<const u32x4*>(kr + kk * 32 + half * 16);
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, k), qf[qb][kk], s, 0, 0, 0);
          }
          float mx = m;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int j = j0 + 8 * (r >> 2) + 4 * half + (r & 3);
            if (j >= lim[qb] || (HEAD && j < head && j >= a.head_len)) s[r] = -INFINITY;
            mx = fmaxf(mx, s[r]);
          }
          mx = half_swap_max(mx);
          const float alpha = __builtin_amdgcn_exp2f((m - mx) * scale_log2);
          m = mx;
          l *= alpha;
#pragma unroll
          for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[qb][ct][r] *= alpha;
          float part = 0.f;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f((s[r] - m) * scale_log2);
            part += s[r];
          }
          l += half_swap_sum(part);
#pragma unroll
          for (int kk = 0; kk < 32; ++kk) {
            // key j0 + kk: register (kk / 8) * 4 + kk % 4 of lane half (kk / 4) % 2
            const float p = __shfl(s[(kk >> 3) * 4 + (kk & 3)], l32 + 32 * ((kk >> 2) & 1), 64);
            const char* vr = j0 + kk < lim[qb] ? row_of(j0 + kk) : nullptr;
            if (vr != nullptr) {
#pragma unroll
              for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                  const uint2 w = *reinterpret_cast<const uint2*>(vr + rowb / 2 + (ct * 32 + 2 * r + 4 * half) * 2);
                  o[qb][ct][r] = fmaf(p, __uint_as_float(w.x << 16), o[qb][ct][r]);
                  o[qb][ct][r + 1] = fmaf(p, __uint_as_float(w.x & 0xffff0000u), o[qb][ct][r + 1]);
                  o[qb][ct][r + 2] = fmaf(p, __uint_as_float(w.y << 16), o[qb][ct][r + 2]);
                  o[qb][ct][r + 3] = fmaf(p, __uint_as_float(w.y & 0xffff0000u), o[qb][ct][r + 3]);
                }
            }
          }
        }
        mu[qb] = m * scale_log2;
        l_run[qb] = l;
      }
    }
  }

  // o[qb][ct][r] = O^T[channel ct*32 + 8 (r/4) + 4 half + r%4][packed row wq0 + 32 qb + l32]
  if (!a.direct) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const int i = wq0 + 32 * qb + l32;
      if (i >= sp.rows) continue;
      const int64_t at = (static_cast<int64_t>(split) * a.T + sp.lo + i / a.G) * a.H + g * a.G + i % a.G;
      if (half == 0) {
        a.ml[at] = make_float2(l_run[qb] == 0.f ? -INFINITY : mu[qb], l_run[qb]);
        if (split == 0) empty_parts(a, at);
      }
      if (l_run[qb] == 0.f) continue;
      float* op = a.o + at * HD + 4 * half;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          *reinterpret_cast<float4*>(op + ct * 32 + 2 * r) =
              make_float4(o[qb][ct][r], o[qb][ct][r + 1], o[qb][ct][r + 2], o[qb][ct][r + 3]);
    }
    return;
  }
  bf16_t* Os = reinterpret_cast<bf16_t*>(smem) + wave * WQ * OLD;
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const float inv_l = l_run[qb] == 0.f ? 0.f : 1.0f / l_run[qb];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const uint2 w = {pack_bf16x2(o[qb][ct][r] * inv_l, o[qb][ct][r + 1] * inv_l),
                         pack_bf16x2(o[qb][ct][r + 2] * inv_l, o[qb][ct][r + 3] * inv_l)};
        *reinterpret_cast<uint2*>(Os + (32 * qb + l32) * OLD + ct * 32 + 2 * r + 4 * half) = w;
      }
    const int i = wq0 + 32 * qb + l32;
    if (a.lse != nullptr && half == 0 && i < sp.rows)
      a.lse[static_cast<int64_t>(g * a.G + i % a.G) * a.T + sp.lo + i / a.G] =
          l_run[qb] == 0.f ? -INFINITY : (mu[qb] + log2f(l_run[qb])) * kLn2;
    if (a.ml != nullptr && half == 0 && i < sp.rows)
      a.ml[static_cast<int64_t>(sp.lo + i / a.G) * a.H + g * a.G + i % a.G] = make_float2(0.f, kDone);
  }
  // each wave stores its own rows: its LDS writes are in order before its reads
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  for (int c = lane; c < WQ * CPR; c += 64) {
    const int r = c / CPR, ch = (c % CPR) * 8, i = wq0 + r;
    if (i < sp.rows)
      *reinterpret_cast<u32x4*>(static_cast<bf16_t*>(a.out) + static_cast<int64_t>(sp.lo + i / a.G) * a.out_stride +
                                (g * a.G + i % a.G) * HD + ch) = *reinterpret_cast<const u32x4*>(Os + r * OLD + ch);
  }
}

// The many-row kernel, and the few-row one's work in the same launch: its
// workgroups fill the CUs that the first, longer ones leave.
template <int HD, int QB, int NW, bool HEAD>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_many_kernel(PagedJobs many,
                                                                                                      PagedJobs few) {
  constexpr int GROUPS = NW / 4;
  __shared__ __align__(1024) union {
    ManyShared<HD, QB, NW> many;
    FewShared<HD, 4> few[GROUPS];
  } shared;
  if (blockIdx.x < many.blocks) {
    const int which = blockIdx.x >= many.first;
    const PagedAttention a = many.job[which];  // (a copy: what it holds stays in registers)
    many_rows<HD, QB, NW, HEAD>(a, blockIdx.x - (which ? many.first : 0), shared.many);
  } else {
    const int group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
    const uint32_t block = (blockIdx.x - many.blocks) * GROUPS + group;
    const int which = block >= few.first;
    const PagedAttention a = few.job[which];
    few_rows<HD, 4, HEAD>(a, block - (which ? few.first : 0), block < few.blocks, threadIdx.x & 255, shared.few[group]);
  }
}

// fp32 storage, and bf16 at head dim 16: the few-row kernel with both
// products on the fp32 matrix instructions, fp32 operands and sums, for any
// number of packed rows, W = 16 or 32 at a time (one row costs what W do; one of
// 42 sequences of up to 867, 32 heads of 128 on 8, 81 us with 32, 63 with 16, and
// 57.7, 4.2 TB/s, now; 16 of up to 1024, 12 of 64, 19.4, loads' and products'
// latency in turn). K is read from LDS 16 bytes a lane, as the first
// operand has it; V one number a lane, W consecutive channels a row. The
// exponentials are expf (the fp32 attention in k_attn.hip says why).
template <typename T, int HD, int W, int NW>
struct F32Shared {
  static constexpr int HP = W + 1;  // merge row stride: [channel][row]
  static constexpr int TILES = NW * 64 * HD * sizeof(T), MERGE = NW * HD * HP * 4;
  unsigned char tiles[MERGE > TILES ? MERGE : TILES];
  float m[NW][W], l[NW][W];
};

template <typename T, int HD, int W, int NW, bool HEAD>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(HD == 128 ? 1 : HD == 64 || NW == 8 ? 2 : 3))) void paged_f32_kernel(
    PagedJobs jobs) {
  constexpr int E = sizeof(T);
  constexpr int NG = 64 / W, NT = 32 / W, NR = W * W / 64;  // lane groups, key tiles of a step, registers of a tile
  constexpr int KK = HD / (4 * NG);          // channels go 4 a lane and group
  constexpr int CT = HD < W ? 1 : HD / W;    // W-channel blocks of O (half empty at HD 16, W 32)
  typedef std::conditional_t<W == 32, f32x16_t, f32x4_t> acc_t;
  constexpr int RB = HD * E, HALF = 32 * RB, CPR = RB / 16;
  constexpr int RPL = 1024 / RB < 16 ? 1024 / RB : 16, NL = 16 / RPL;  // rows a load, loads per 16 rows
  constexpr int HP = F32Shared<T, HD, W, NW>::HP;
  __shared__ __align__(1024) F32Shared<T, HD, W, NW> shared;
  unsigned char* smem = shared.tiles;
  auto& sm = shared.m;
  auto& sl = shared.l;
  const int which = blockIdx.x >= jobs.first, block = blockIdx.x - (which ? jobs.first : 0);
  const PagedAttention a = jobs.job[which];  // (a copy: what it holds stays in registers)
  const int Hkv = a.H / a.G, pair = block % (Hkv * a.B), st = block / (Hkv * a.B);
  const int g = pair % Hkv, b = pair / Hkv, tile = st % a.tiles, split = st / a.tiles;
  const Span sp = span_of(a, b);
  const int i0 = tile * W;
  if (i0 >= sp.rows) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = lane / W, col = lane % W;
  const int row = min(i0 + col, sp.rows - 1);  // rows past the sequence are not stored
  // A common prefix in the same job (HEAD) comes first, filled up to whole steps: key
  // j below `head` is its row j, key j from there on row j - head of the
  // sequence's own
  const int head = HEAD ? (a.head_len + 31) & ~31 : 0, end = head + sp.len;
  auto seen = [&](int i) { return head + (a.causal ? max(min(sp.first + i / a.G, sp.len), 0) : sp.len); };
  const int lim = seen(row), lim0 = seen(i0);  // a lane's keys are those below lim; the tile's first row's
  const int last = seen(min(i0 + W - 1, sp.rows - 1));
  const int k0 = split * a.chunk, kend = min(last, k0 + a.chunk);

  // K row r of a tile keeps its 16-byte chunk c at c ^ ksw(r): the rows of a
  // read phase fall on all banks; V row r at c ^ vsw(r): rows four apart, which
  // the lane groups read at once, do
  auto ksw = [](int r) { return CPR >= 16 ? r & 15 : CPR == 8 ? (r >> 1) & 7 : CPR == 4 ? (r >> 2) & 3 : (r >> 3) & 1; };
  auto vsw = [](int r) { return CPR >= 16 ? ((r >> 2) & (NG - 1)) << (W == 32 ? 3 : 2) : CPR == 8 && W == 16 ? ((r >> 2) & 1) << 2 : 0; };
  const uint32_t rowb = static_cast<uint32_t>(a.at.kvd) * (2 * E);
  uint32_t koff[NL], voff[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int r = i * RPL + lane / CPR;
    koff[i] = r * rowb + (((lane % CPR) ^ ksw(r)) << 4);
    voff[i] = r * rowb + (((lane % CPR) ^ vsw(r)) << 4);
  }
  unsigned char* mine = smem + wave * (2 * HALF);
  const uint32_t lds0 = lds_address(smem) + wave * (2 * HALF);
  const scalar_ids table = scalar(sp.table), head_table = scalar(a.head_table);
  const char* pool = static_cast<const char*>(a.at.pool);
  // 16 rows from row j on, of page `page` (-1 where the sequence has ended): `col` bytes into a row
  auto resource = [&](int j, int page, uint32_t col) {
    const bool there = page >= 0 && page < a.at.n_pages;
    const uint32_t bytes = there ? static_cast<uint32_t>(min((HEAD && j < head ? a.head_len : end) - j, 16)) * rowb - col : 0u;
    u32x4 res = buffer_resource(pool + (there ? page : 0) * (a.at.page_stride * E) +
                                    static_cast<uint32_t>((HEAD && j >= head ? j - head : j) & ((1 << a.at.shift) - 1)) * rowb + col,
                                bytes);
    // a load in asm may follow a vector instruction's write of its scalar operands by five states at least
    asm volatile("s_nop 4" : "+s"(res));
    return res;
  };
  // (the read does not wait for the length: up to the table's end it goes through)
  auto page_of = [&](int j) {
    const bool first = HEAD && j < head;
    const int p = (first ? j : j - head) >> a.at.shift, most = first ? (a.head_len - 1) >> a.at.shift : a.at.max_pages - 1;
    const int page = most >= 0 ? (first ? head_table : table)[min(p, most)] : -1;
    return j < (first ? a.head_len : end) ? page : -1;
  };
  const bool once = !HEAD && a.once && a.tiles == 1;  // this workgroup alone reads the rows
  const uint32_t kcol = g * RB, vcol = rowb / 2 + g * RB;
  auto load = [&](int j0, int pg0, int pg1, uint32_t lds, uint32_t col, const uint32_t (&off)[NL]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const u32x4 res = resource(j0 + 16 * h, h == 0 ? pg0 : pg1, col);
      if (once) {
#pragma unroll
        for (int i = 0; i < NL; ++i)
          if (RPL * CPR == 64 || lane < RPL * CPR) lds_load16_once(lds + (h * NL + i) * (RPL * RB), off[i], res);
      } else {
#pragma unroll
        for (int i = 0; i < NL; ++i)
          if (RPL * CPR == 64 || lane < RPL * CPR) lds_load16(lds + (h * NL + i) * (RPL * RB), off[i], res);
      }
    }
  };

  float m_run = -INFINITY, l_run = 0.f;  // of the scaled scores; l_run: this lane's keys only
  const acc_t zero = {};
  acc_t o[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) o[ct] = zero;
  const bool vch = HD >= W || col < HD;  // lanes whose channel exists
  // the key of register r of tile t; the same of the channel of a register of O
  auto key = [&](int t, int r) { return t * W + 8 * (r >> 2) + 4 * group + (r & 3); };
  // fragment addresses: the lane's four channels of K row col, its channel of V
  // row 4 group, whose chunks are those of all its rows (vsw)
  uint32_t kaddr[KK], vaddr[CT];
#pragma unroll
  for (int c = 0; c < KK; ++c) {
    const int ch = 4 * (NG * c + group) * E;
    kaddr[c] = col * RB + (((ch >> 4) ^ ksw(col)) << 4) + (ch & 15);
  }
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int ch = (ct * W + (HD < W ? col % HD : col)) * E;
    vaddr[ct] = HALF + 4 * group * RB + (((ch >> 4) ^ vsw(4 * group)) << 4) + (ch & 15);
  }
  auto mfma = [](float x, float y, acc_t c) {
    if constexpr (W == 32) return __builtin_amdgcn_mfma_f32_32x32x2f32(x, y, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x4f32(x, y, c, 0, 0, 0);
  };
  int j0 = k0 + wave * 32;
  int pg0 = page_of(j0), pg1 = page_of(j0 + 16);
  if (j0 < kend) {
    load(j0, pg0, pg1, lds0, kcol, koff);
    load(j0, pg0, pg1, lds0 + HALF, vcol, voff);
  }
  int nx0 = page_of(j0 + 32 * NW), nx1 = page_of(j0 + 32 * NW + 16);  // read a step before the loads that need them
  asm volatile("" : "+s"(nx0), "+s"(nx1));
  float4 qf[KK];
  if (j0 < kend) {
    const T* qp = static_cast<const T*>(a.q) + static_cast<int64_t>(sp.lo + row / a.G) * a.q_stride + (g * a.G + row % a.G) * HD;
#pragma unroll
    for (int s = 0; s < KK; ++s) qf[s] = load4<T>(qp + 4 * (NG * s + group));
    // here before the loop, which would otherwise wait for every load in it
#pragma unroll
    for (int s = 0; s < KK; ++s) asm volatile("" : "+v"(qf[s].x), "+v"(qf[s].y), "+v"(qf[s].z), "+v"(qf[s].w));
  }
  for (; j0 < kend; j0 += 32 * NW) {
    const int jn = j0 + 32 * NW;
    const bool more = jn < kend;
    pg0 = nx0;
    pg1 = nx1;
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NL) : "memory");  // K is here, V may be under way
    __builtin_amdgcn_sched_barrier(0);
    acc_t s[NT];
    float4 kf[KK][NT];  // all read before the products: one latency, not one a product
#pragma unroll
    for (int c = 0; c < KK; ++c)
#pragma unroll
      for (int t = 0; t < NT; ++t) kf[c][t] = load4<T>(reinterpret_cast<const T*>(mine + kaddr[c] + t * W * RB));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int c = 0; c < KK; ++c) {
#pragma unroll
      for (int t = 0; t < NT; ++t) s[t] = mfma(kf[c][t].x, qf[c].x, c == 0 ? zero : s[t]);
#pragma unroll
      for (int t = 0; t < NT; ++t) s[t] = mfma(kf[c][t].y, qf[c].y, s[t]);
#pragma unroll
      for (int t = 0; t < NT; ++t) s[t] = mfma(kf[c][t].z, qf[c].z, s[t]);
#pragma unroll
      for (int t = 0; t < NT; ++t) s[t] = mfma(kf[c][t].w, qf[c].w, s[t]);
    }
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) load(jn, pg0, pg1, lds0, kcol, koff);
    nx0 = page_of(jn + 32 * NW);
    nx1 = page_of(jn + 32 * NW + 16);
    const bool edge = j0 + 32 > (HEAD && j0 < head ? a.head_len : lim0);
    const int left = (HEAD && j0 < head ? a.head_len : lim) - j0;
    float mloc = -INFINITY;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        s[t][r] = edge && key(t, r) >= left ? -INFINITY : s[t][r] * a.scale;
        mloc = fmaxf(mloc, s[t][r]);
      }
    mloc = W == 32 ? half_swap_max(mloc) : quarter_swap_max(mloc);
    const float m_new = fmaxf(m_run, mloc);
    if (__builtin_amdgcn_ballot_w64(m_new > m_run) != 0) {
      const float alpha = m_new == -INFINITY ? 1.0f : expf(m_run - m_new);
      l_run *= alpha;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int r = 0; r < NR; ++r) o[ct][r] *= alpha;
      m_run = m_new;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        s[t][r] = expf(s[t][r] - m_use);
        l_run += s[t][r];
      }
    if (more)
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NL) : "memory");  // V is here, the next K may be under way
    else
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    asm volatile("" : "+s"(nx0), "+s"(nx1));  // here: scalar loads under way make every wait for LDS one for all
    __builtin_amdgcn_sched_barrier(0);
    // hidden keys' values that are not finite: key by key (few_rows)
    bool odd = false;
    if ((!HEAD || j0 >= head) && lim0 < min(j0 + 32, end)) {
#pragma unroll
      for (int i = 0; i < HALF / 1024; ++i) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(mine + HALF + i * 1024 + lane * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          odd |= (w[e] & 0x7f800000u) == 0x7f800000u || (E == 2 && (w[e] & 0x7f80u) == 0x7f80u);
      }
      odd = __builtin_amdgcn_ballot_w64(odd) != 0;
    }
    if (!odd) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r0 = 0; r0 < NR; r0 += 4) {
          float vf[4][CT];
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
              vf[r][ct] = to_f32(*reinterpret_cast<const T*>(mine + vaddr[ct] + (t * W + 2 * r0 + r) * RB));
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) o[ct] = mfma(vch ? vf[r][ct] : 0.f, s[t][r0 + r], o[ct]);
        }
    } else {
#pragma unroll
      for (int kk = 0; kk < 32; ++kk) {
        const int w = kk % W;  // key j0 + kk: its register, and its lane group
        const float p = __shfl(s[kk / W][W == 32 ? (w >> 3) * 4 + (w & 3) : w & 3], col + W * ((w >> 2) & (NG - 1)), 64);
        if (j0 + kk < lim) {
#pragma unroll
          for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int r = 0; r < NR; r += 4) {
              const int c = ct * W + 2 * r + 4 * group, ch = c * E;
              if (c >= HD) continue;
              const float4 v = load4<T>(reinterpret_cast<const T*>(mine + HALF + kk * RB + (((ch >> 4) ^ vsw(kk)) << 4) + (ch & 15)));
              o[ct][r] = fmaf(p, v.x, o[ct][r]);
              o[ct][r + 1] = fmaf(p, v.y, o[ct][r + 1]);
              o[ct][r + 2] = fmaf(p, v.z, o[ct][r + 2]);
              o[ct][r + 3] = fmaf(p, v.w, o[ct][r + 3]);
            }
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) load(jn, pg0, pg1, lds0 + HALF, vcol, voff);
  }
  l_run = W == 32 ? half_swap_sum(l_run) : quarter_swap_sum(l_run);
  __syncthreads();  // every wave is past its tiles
  float* so = reinterpret_cast<float*>(smem);
  if (group == 0) {
    sm[wave][col] = m_run;
    sl[wave][col] = l_run;
  }
  const int nr = min(W, sp.rows - i0);
  if (col < nr) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int r = 0; r < NR; ++r)
        if (key(ct, r) < HD) so[(wave * HD + key(ct, r)) * HP + col] = o[ct][r];
  }
  __syncthreads();
  for (int it = tid; it < nr * (HD / 4); it += 64 * NW) {
    const int q = it / (HD / 4), c0 = (it % (HD / 4)) * 4, i = i0 + q;
    float m = sm[0][q];
#pragma unroll
    for (int w = 1; w < NW; ++w) m = fmaxf(m, sm[w][q]);
    float l = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      // a wave without keys for this row holds the empty sum
      if (sm[w][q] == -INFINITY && sl[w][q] == 0.f) continue;
      const float f = expf(sm[w][q] - (m == -INFINITY ? 0.f : m));
      l = fmaf(f, sl[w][q], l);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = fmaf(f, so[(w * HD + c0 + e) * HP + q], v[e]);
    }
    const int t = sp.lo + i / a.G, h = g * a.G + i % a.G;
    const int64_t row0 = static_cast<int64_t>(t) * a.H + h;
    if (a.direct) {
      const float inv = l == 0.f ? 0.f : 1.0f / l;
      T* op = static_cast<T*>(a.out) + t * a.out_stride + h * HD + c0;
#pragma unroll
      for (int e = 0; e < 4; ++e) op[e] = from_f32<T>(v[e] * inv);
      if (c0 == 0 && a.lse != nullptr) a.lse[static_cast<int64_t>(h) * a.T + t] = l == 0.f ? -INFINITY : m + logf(l);
    } else {
      const int64_t at = static_cast<int64_t>(split) * a.T * a.H + row0;
      if (c0 == 0) {
        a.ml[at] = make_float2(m, l);
        if (split == 0) empty_parts(a, at);
      }
      if (l != 0.f) *reinterpret_cast<float4*>(a.o + at * HD + c0) = make_float4(v[0], v[1], v[2], v[3]);
    }
  }
}

// The parts of every row, joined: M = max m, L = sum l exp(m - M), out = sum o
// exp(m - M) / L. A part without keys has l = 0 and no o. (The bf16 matrix
// kernels' maxima are in units of log 2, as they used them.) HD / 4 threads
// take four channels each of a row's parts sub, sub + per, ...; `per` such
// groups a row, whose sums are added in their order. Few rows of many parts
// need them: 128 rows of 62 parts with one group 39.7 us.
template <typename T, int HD>
__global__ __launch_bounds__(256) void paged_join_kernel(const float2* __restrict__ ml,
                                                         const float* __restrict__ o, int parts, int rows,
                                                         int H, int Trows, T* __restrict__ out,
                                                         int64_t out_stride, float* __restrict__ lse, int per) {
  constexpr int LPR = HD / 4, U = 4;
  constexpr bool LOG2 = sizeof(T) == 2 && HD >= 32;
  __shared__ float sv[256][4];
  __shared__ float2 sml[256 / LPR];
  const int group = threadIdx.x / LPR, lane = threadIdx.x % LPR, sub = group % per, c = 4 * lane;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * (256 / LPR / per) + group / per;
  const bool live = i < rows && ml[i].y != kDone;
  float M = -INFINITY, L = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
  if (live) {
    for (int s = sub + lane * per; s < parts; s += per * LPR) M = fmaxf(M, ml[static_cast<int64_t>(s) * rows + i].x);
#pragma unroll
    for (int off = 1; off < LPR; off <<= 1) M = fmaxf(M, __shfl_xor(M, off, 64));
    const float m0 = M == -INFINITY ? 0.f : M;
    for (int s0 = sub; s0 < parts; s0 += per * U) {
      float2 p[U];
      float4 w[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t at = static_cast<int64_t>(min(s0 + u * per, parts - 1)) * rows + i;
        p[u] = ml[at];
        w[u] = *reinterpret_cast<const float4*>(o + at * HD + c);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (s0 + u * per >= parts || p[u].y == 0.f) continue;
        const float f = LOG2 ? __builtin_amdgcn_exp2f(p[u].x - m0) : expf(p[u].x - m0);
        L = fmaf(p[u].y, f, L);
        v[0] = fmaf(w[u].x, f, v[0]);
        v[1] = fmaf(w[u].y, f, v[1]);
        v[2] = fmaf(w[u].z, f, v[2]);
        v[3] = fmaf(w[u].w, f, v[3]);
      }
    }
  }
  if (per > 1) {
    if (lane == 0) sml[group] = make_float2(M, L);
#pragma unroll
    for (int e = 0; e < 4; ++e) sv[threadIdx.x][e] = v[e];
    __syncthreads();
    if (sub != 0) return;
    for (int k = 0; k < per; ++k) M = fmaxf(M, sml[group + k].x);
    const float m0 = M == -INFINITY ? 0.f : M;
    L = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = 0.f;
    for (int k = 0; k < per; ++k) {
      const float2 p = sml[group + k];
      if (p.y == 0.f) continue;
      const float f = LOG2 ? __builtin_amdgcn_exp2f(p.x - m0) : expf(p.x - m0);
      L = fmaf(p.y, f, L);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = fmaf(sv[threadIdx.x + k * LPR][e], f, v[e]);
    }
  }
  if (!live) return;
  const int t = static_cast<int>(i / H), h = static_cast<int>(i - static_cast<int64_t>(t) * H);
  const float inv = L == 0.f ? 0.f : 1.0f / L;
  T* op = out + t * out_stride + h * HD + c;
#pragma unroll
  for (int e = 0; e < 4; ++e) op[e] = from_f32<T>(v[e] * inv);
  if (c == 0 && lse != nullptr)
    lse[static_cast<int64_t>(h) * Trows + t] = L == 0.f ? -INFINITY : LOG2 ? (M + log2f(L)) * kLn2 : M + logf(L);
}

template <typename T, int HD, int W, bool HEAD>
hipError_t f32_launch(hipStream_t s, const PagedJobs& jobs) {
  if constexpr (W == 16)
    if (jobs.job[0].waves == 1)
      return launch(K_ATTENTION, paged_f32_kernel<T, HD, W, 1, HEAD>, dim3(jobs.blocks), dim3(64), 0, s, jobs);
  if constexpr (W == 16 && HD * sizeof(T) <= 256)
    if (jobs.job[0].waves == 8)
      return launch(K_ATTENTION, paged_f32_kernel<T, HD, W, 8, HEAD>, dim3(jobs.blocks), dim3(512), 0, s, jobs);
  return launch(K_ATTENTION, paged_f32_kernel<T, HD, W, 4, HEAD>, dim3(jobs.blocks), dim3(256), 0, s, jobs);
}

template <typename T, int W, bool HEAD>
hipError_t f32_dispatch(hipStream_t s, const PagedJobs& jobs) {
  if (jobs.job[0].hd == 16) return f32_launch<T, 16, W, HEAD>(s, jobs);
  if constexpr (sizeof(T) == 4) {
    if (jobs.job[0].hd == 32) return f32_launch<T, 32, W, HEAD>(s, jobs);
    if (jobs.job[0].hd == 64) return f32_launch<T, 64, W, HEAD>(s, jobs);
    if (jobs.job[0].hd == 128) return f32_launch<T, 128, W, HEAD>(s, jobs);
  }
  return hipErrorInvalidValue;
}

template <int HD, bool HEAD>
hipError_t few_launch(hipStream_t s, const PagedJobs& jobs) {
  if (jobs.job[0].waves == 1)
    return launch(K_ATTENTION, paged_few_kernel<HD, 1, HEAD>, dim3(jobs.blocks), dim3(64), 0, s, jobs);
  if (jobs.job[0].waves == 8)
    return launch(K_ATTENTION, paged_few_kernel<HD, 8, HEAD>, dim3(jobs.blocks), dim3(512), 0, s, jobs);
  return launch(K_ATTENTION, paged_few_kernel<HD, 4, HEAD>, dim3(jobs.blocks), dim3(256), 0, s, jobs);
}

template <bool HEAD>
hipError_t few_dispatch(hipStream_t s, int dtype, const PagedJobs& jobs) {
  const PagedAttention& a = jobs.job[0];
  if (paged_matrix(dtype, a.hd)) {
    if (a.hd == 32) return few_launch<32, HEAD>(s, jobs);
    return a.hd == 64 ? few_launch<64, HEAD>(s, jobs) : few_launch<128, HEAD>(s, jobs);
  }
  if (a.tile == 32) return dtype == 1 ? f32_dispatch<bf16_t, 32, HEAD>(s, jobs) : f32_dispatch<float, 32, HEAD>(s, jobs);
  return dtype == 1 ? f32_dispatch<bf16_t, 16, HEAD>(s, jobs) : f32_dispatch<float, 16, HEAD>(s, jobs);
}

template <typename T>
hipError_t join_dispatch(hipStream_t s, const float2* ml, const float* o, int parts, int rows, int H, int T_,
                         int hd, void* out, int64_t os, float* lse) {
  // groups of threads a row: until they number four a SIMD, or take few parts each
  const int groups = 256 / (hd / 4);
  int per = 1;
  while (per < groups && 4 * per < parts && static_cast<int64_t>(rows) * per < 16 * device_cu_count()) per *= 2;
  const int rpb = groups / per;
  const dim3 g(static_cast<uint32_t>((rows + rpb - 1) / rpb)), block(256);
  T* op = static_cast<T*>(out);
  switch (hd) {
    case 16: return launch(K_ATTENTION, paged_join_kernel<T, 16>, g, block, 0, s, ml, o, parts, rows, H, T_, op, os, lse, per);
    case 32: return launch(K_ATTENTION, paged_join_kernel<T, 32>, g, block, 0, s, ml, o, parts, rows, H, T_, op, os, lse, per);
    case 64: return launch(K_ATTENTION, paged_join_kernel<T, 64>, g, block, 0, s, ml, o, parts, rows, H, T_, op, os, lse, per);
    case 128: return launch(K_ATTENTION, paged_join_kernel<T, 128>, g, block, 0, s, ml, o, parts, rows, H, T_, op, os, lse, per);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t launch_paged_append(hipStream_t s, int dtype, const PagedAppend& a) {
  if (a.T == 0) return hipSuccess;
  // few rows: one a workgroup, so that they spread over the CUs; many: about
  // 1024 items
  const int per16 = dtype == 1 ? 8 : 4, kv = a.Hkv * a.hd / per16;
  const int items = a.pos != nullptr ? ((a.q != nullptr ? a.H : 0) + a.Hkv) * a.hd / (2 * per16) + kv : 2 * kv;
  const int rows = std::max(1, std::min({kAppendRows, a.T / (4 * device_cu_count()), 1024 / items}));
  const dim3 grid((a.T + rows - 1) / rows), block(256);
  if (dtype == 1) return launch(K_MISC, paged_append_kernel<bf16_t>, grid, block, 0, s, a, rows);
  return launch(K_MISC, paged_append_kernel<float>, grid, block, 0, s, a, rows);
}

template <bool HEAD>
static hipError_t many_dispatch(hipStream_t s, int hd, const PagedJobs& many, const PagedJobs& few) {
  const dim3 grid(many.blocks + (hd == 128 ? (few.blocks + 1) / 2 : few.blocks));
  if (hd == 32) return launch(K_ATTENTION, paged_many_kernel<32, 2, 4, HEAD>, grid, dim3(256), 0, s, many, few);
  if (hd == 64) return launch(K_ATTENTION, paged_many_kernel<64, 2, 4, HEAD>, grid, dim3(256), 0, s, many, few);
  return launch(K_ATTENTION, paged_many_kernel<128, 1, 8, HEAD>, grid, dim3(512), 0, s, many, few);
}

hipError_t launch_paged_attention(hipStream_t s, int dtype, const PagedAttention* few, int fews,
                                  const PagedAttention* many, int manys) {
  PagedJobs w[2] = {};
  for (int k = 0; k < 2; ++k) {
    const PagedAttention* job = k ? many : few;
    const int n = k ? manys : fews;
    if (n == 0) continue;
    w[k].job[0] = job[0];
    w[k].job[1] = job[n - 1];
    w[k].first = static_cast<uint32_t>(paged_blocks(job[0], k != 0));
    w[k].blocks = w[k].first + (n > 1 ? static_cast<uint32_t>(paged_blocks(job[1], k != 0)) : 0u);
  }
  const int hd = (manys > 0 ? many : few)[0].hd;
  if (manys > 0)
    return many[0].head_len > 0 ? many_dispatch<true>(s, hd, w[1], w[0]) : many_dispatch<false>(s, hd, w[1], w[0]);
  return few[0].head_len > 0 ? few_dispatch<true>(s, dtype, w[0]) : few_dispatch<false>(s, dtype, w[0]);
}

hipError_t launch_paged_join(hipStream_t s, int dtype, const float2* ml, const float* o, int parts, int T, int H,
                             int hd, void* out, int64_t out_stride, float* lse) {
  if (dtype == 1) return join_dispatch<bf16_t>(s, ml, o, parts, T * H, H, T, hd, out, out_stride, lse);
  return join_dispatch<float>(s, ml, o, parts, T * H, H, T, hd, out, out_stride, lse);
}

}  // namespace zsa
